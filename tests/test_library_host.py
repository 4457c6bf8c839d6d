"""CPU-side checks of the CUDA library: it loads, exports everything the header declares,
and its host-only entry points agree with the oracle.  No kernel runs here."""
import ctypes as C
import os
import re
import struct

import numpy as np
import pytest

import oracle
import workloads
import paper_2505_02380_b200 as E
from paper_2505_02380_b200 import build as build_mod

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "entro.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(entro_[a-z0-9_]+)\s*\(", header))
    assert declared, "no declarations found"
    L = C.CDLL(E.LIB_PATH)
    for name in sorted(declared):
        assert hasattr(L, name), name
    assert declared == set(E.EXPORTS)


def test_golden_lengths_and_codes():
    from test_oracle_huffman import _golden_cases
    for counts, lengths in _golden_cases():
        cb = E.entro_build_codebook(counts)
        assert cb.lengths().tolist() == lengths
        assert cb.max_len == max(lengths)


def test_codebook_matches_oracle_bit_exactly():
    rng = np.random.default_rng(2024)
    for t in range(600):
        n = [16, 256, int(rng.integers(1, 257))][t % 3]
        hi = [1, 3, 60, 10**7][t % 4]
        counts = rng.integers(0, hi + 1, size=n)
        if counts.sum() == 0:
            counts[int(rng.integers(0, n))] = 1
        cb = E.entro_build_codebook(counts)
        ln = oracle.huffman_lengths(counts)
        assert np.array_equal(cb.lengths(), ln), counts
        assert np.array_equal(cb.codes(), oracle.canonical_codes(ln))
        assert cb.max_len == int(ln.max())


def test_limited_codebook_matches_oracle_bit_exactly():
    rng = np.random.default_rng(12)
    cases = [[1, 1, 2, 3, 5, 8], [5, 5, 5, 5], [1, 1, 1, 1, 1, 1, 1], [0, 3, 0, 9, 1]]
    for _ in range(40):
        n = int(rng.integers(2, 257))
        c = rng.integers(0, 1000, n)
        c[rng.integers(0, n)] = 10 ** 6          # a dominant symbol makes long tails
        cases.append(c.tolist())
    for bits in (4, 8):
        w = workloads.make_values(1 << 18, 0.02, 70 + bits).numpy()
        q, _ = oracle.quantize_tensor(w, bits)
        cases.append(oracle.histogram(q, 1 << bits).tolist())
    for counts in cases:
        used = sum(1 for c in counts if c)
        for cap in (32, 16, 12, 10, 8):
            if used > 1 and (1 << cap) < used:
                continue
            ref = oracle.length_limited_lengths(counts, cap)
            cb = E.entro_build_codebook_limited(counts, cap)
            assert cb.lengths().tolist() == ref.tolist(), (counts[:8], cap)
            assert cb.codes().tolist() == oracle.canonical_codes(ref).tolist()
            assert cb.max_len == int(ref.max())
    with pytest.raises(E.EntroError) as e:
        E.entro_build_codebook_limited([1] * 9, 3)
    assert e.value.status == E.ERR_CODE_TOO_LONG


def test_codebook_errors():
    fib = [1, 1]
    while len(fib) < 40:
        fib.append(fib[-1] + fib[-2])
    with pytest.raises(E.EntroError) as e:
        E.entro_build_codebook(fib)
    assert e.value.status == E.ERR_CODE_TOO_LONG
    with pytest.raises(E.EntroError) as e:
        E.entro_build_codebook([0, 0, 0])
    assert e.value.status == E.ERR_INVALID_ARG
    fib33 = fib[:33]        # depth 32: the longest supported code
    assert E.entro_build_codebook(fib33).max_len == 32


def test_size_helpers():
    assert E.entro_index_bytes(1 << 20, 4096) == 8 * 257 + 64 * 256
    assert E.entro_index_bytes(4097, 4096) == 8 * 3 + 64 * 2
    assert E.entro_index_bytes(100, 48) == 0          # not a multiple of 32
    assert E.entro_index_bytes(100, 32768) == 0       # above the maximum
    counts = [5, 0, 3, 9]
    cb = E.entro_build_codebook(counts)
    bits = sum(c * l for c, l in zip(counts, cb.lengths().tolist()))
    assert E.entro_stream_words(counts, cb) == (bits + 31) // 32 + E.STREAM_SLACK_WORDS
    assert E.entro_encode_bound_words(1000, cb) == (1000 * cb.max_len + 31) // 32 + E.STREAM_SLACK_WORDS
    assert E.status_string(E.ERR_CORRUPT_STREAM) and E.status_string(E.OK) == "ok"


def test_argument_errors_are_found_before_any_launch():
    """Null pointers and bad sizes are refused on the host (no device is touched)."""
    L = E.lib()
    cb = E.entro_build_codebook([1, 2, 3, 4])
    qp = E.QParams()
    assert L.entro_quantize_tensor(None, 16, 8, 0, None, C.byref(qp), None) == E.ERR_INVALID_ARG
    assert L.entro_quantize_tensor(16, 16, 5, 0, 16, C.byref(qp), None) == E.ERR_INVALID_ARG
    counts = (C.c_uint64 * 256)()
    assert L.entro_histogram(None, 16, 8, counts, None) == E.ERR_INVALID_ARG
    total = C.c_uint64()
    assert L.entro_encode(None, 16, C.byref(cb), 4096, None, 0, None, 0, C.byref(total), None) == E.ERR_INVALID_ARG
    assert L.entro_encode(16, 16, C.byref(cb), 100, 16, 64, 16, 4096, C.byref(total), None) == E.ERR_INVALID_ARG
    # symbols that do not start on a 16-byte boundary (an offset view of a tensor: q[1:]) are refused
    assert L.entro_encode(17, 16, C.byref(cb), 4096, 16, 64, 16, 4096, C.byref(total), None) == E.ERR_INVALID_ARG
    assert L.entro_decode_dequant(None, 0, None, 16, 4096, C.byref(cb), 1.0, 0, None, None) == E.ERR_INVALID_ARG
    assert L.entro_decode_dequant(16, 100, 16, 16, 4096, C.byref(cb), 1.0, 0, 24, None) == E.ERR_INVALID_ARG  # misaligned out
    bad = E.Codebook.from_lengths([1, 1, 1, 0])        # over-subscribed lengths
    assert L.entro_decode_dequant(16, 100, 16, 16, 4096, C.byref(bad), 1.0, 0, 32, None) == E.ERR_INVALID_ARG
    assert L.entro_decode_dequant_batched(None, 3, None) == E.ERR_INVALID_ARG
    assert L.entro_decode_dequant_batched(None, 0, None) == E.OK


def _kv_cache(**changes):
    """An entro_kv_cache block with made-up addresses (no call that passes its checks is made with it)."""
    f = dict(codes=4096, scales=4096, table=4096, lens=4096, refs=4096, work=4096, work_bytes=1 << 30, pages=100, heads=8, page=16,
             dim=64, slots=10, width=20)
    f.update(changes)
    buf = C.create_string_buffer(128)
    struct.pack_into("=7Q6I", buf, 0, *f.values())
    return buf


def test_kv_cache_refusals_before_any_launch():
    L = E.lib()
    batch = struct.pack("=2I2Q", 2, 2, 4096, 0)
    rows = struct.pack("=2Q4q2i", 4096, 4096, 512, 64, 512, 64, 0, 0)
    query = struct.pack("=3Q4q4Ifi", 4096, 4096, 0, 512, 64, 512, 64, 8, 0, 0, 0, 0.0, 0)

    def calls(cache, batch=batch, rows=rows, query=query):
        return [L.entro_kv_reserve(cache, batch, None), L.entro_kv_append(cache, batch, rows, None),
                L.entro_kv_read(cache, batch, rows, None), L.entro_kv_attention(cache, batch, query, None)]

    for change in (dict(codes=0), dict(codes=4100), dict(scales=0), dict(scales=4098), dict(table=0), dict(lens=0), dict(refs=0),
                   dict(work=0), dict(work=4104), dict(pages=0), dict(heads=0), dict(slots=0), dict(width=0), dict(pages=1 << 31)):
        cache = _kv_cache(**change)
        assert set(calls(cache)) == {E.ERR_INVALID_ARG}, change
        assert L.entro_kv_free(cache, 4096, 1, None) == E.ERR_INVALID_ARG
        assert L.entro_kv_fork(cache, 4096, 4096, 1, None) == E.ERR_INVALID_ARG
        assert L.entro_kv_trim(cache, 4096, 1, 8, 0, None) == E.ERR_INVALID_ARG
        assert L.entro_kv_compact(cache, None) == E.ERR_INVALID_ARG
    for change in (dict(page=17), dict(page=256), dict(page=8), dict(dim=80), dict(dim=256), dict(dim=32)):
        assert set(calls(_kv_cache(**change))) == {E.ERR_UNSUPPORTED}, change
        assert L.entro_kv_work_bytes(_kv_cache(**change)) == 0
    assert set(calls(_kv_cache(work_bytes=4096))) == {E.ERR_BUFFER_TOO_SMALL}
    assert set(calls(None)) == {E.ERR_INVALID_ARG} and L.entro_kv_work_bytes(None) == 0
    good = _kv_cache()
    # more sequences than slots, rows that do not fit one row each, unaligned lists
    for b in (struct.pack("=2I2Q", 11, 11, 4096, 0), struct.pack("=2I2Q", 2, 3, 4096, 0), struct.pack("=2I2Q", 2, 2, 4097, 0),
              struct.pack("=2I2Q", 2, 9, 4096, 4098), struct.pack("=2I2Q", 2, 1 << 31, 4096, 4096)):
        assert set(calls(good, batch=b)) == {E.ERR_INVALID_ARG}
    assert set(calls(good, batch=None)) == {E.ERR_INVALID_ARG}
    for r in ((0, 4096, 512, 64, 512, 64, 0, 0), (4096, 0, 512, 64, 512, 64, 0, 0), (4104, 4096, 512, 64, 512, 64, 0, 0),
              (4096, 4096, 513, 64, 512, 64, 0, 0), (4096, 4096, 512, 64, 512, 65, 0, 0), (4096, 4096, 512, 64, 512, 64, 2, 0),
              (4096, 4096, 512, 64, 512, 64, 0, 1)):
        r = struct.pack("=2Q4q2i", *r)
        assert L.entro_kv_append(good, batch, r, None) == L.entro_kv_read(good, batch, r, None) == E.ERR_INVALID_ARG
    for q in ((0, 4096, 0, 512, 64, 512, 64, 8, 0, 0, 0, 0.0, 0), (4096, 0, 0, 512, 64, 512, 64, 8, 0, 0, 0, 0.0, 0),
              (4096, 4096, 2, 512, 64, 512, 64, 8, 0, 0, 0, 0.0, 0), (4096, 4096, 0, 512, 63, 512, 64, 8, 0, 0, 0, 0.0, 0),
              (4096, 4096, 0, 512, 64, 511, 64, 8, 0, 0, 0, 0.0, 0), (4096, 4096, 0, 512, 64, 512, 64, 0, 0, 0, 0, 0.0, 0),
              (4096, 4096, 0, 512, 64, 512, 64, 12, 0, 0, 0, 0.0, 0), (4096, 4096, 0, 512, 64, 512, 64, 8, 0, 0, 0, -1.0, 0),
              (4096, 4096, 0, 512, 64, 512, 64, 8, 0, 0, 0, float("nan"), 0),
              (4096, 4096, 0, 512, 64, 512, 64, 8, 0, 0, 0, float("inf"), 0), (4096, 4096, 0, 512, 64, 512, 64, 8, 0, 0, 0, 0.0, 2)):
        assert L.entro_kv_attention(good, batch, struct.pack("=3Q4q4Ifi", *q), None) == E.ERR_INVALID_ARG, q
    assert L.entro_kv_fork(good, None, 4096, 1, None) == L.entro_kv_fork(good, 4096, 4096, 11, None) == E.ERR_INVALID_ARG
    assert L.entro_kv_free(good, None, 1, None) == L.entro_kv_free(good, 4098, 1, None) == E.ERR_INVALID_ARG
    assert L.entro_kv_trim(good, 4096, 11, 8, 0, None) == E.ERR_INVALID_ARG
    # nothing to do is not an error
    nothing = struct.pack("=2I2Q", 0, 0, 0, 0)
    assert set(calls(good, batch=nothing)) == {E.OK}
    assert L.entro_kv_free(good, None, 0, None) == L.entro_kv_fork(good, None, None, 0, None) == E.OK
    assert "page" in E.status_string(E.ERR_NO_PAGES)
