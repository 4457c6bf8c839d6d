"""The paged 8-bit key/value cache on the GPU: writing and reading bit for bit against NumPy float32,
page operations against lists, attention against 64 bits within a derived bound (kv_reference.py)."""
import math

import numpy as np
import pytest
import torch

import paper_2505_02380_b200 as E
from kv_reference import ZERO, Pages, append, assert_attention, ints, make_cache, sequence, starts

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------- writing and reading

def _numpy(kv):
    return kv.codes.cpu().numpy().copy(), kv.scales.cpu().numpy().copy(), kv.table.cpu().numpy(), kv.lens.cpu().numpy()


def _append_and_compare(kv, slots, rows, k, v, single=False):
    codes, scales, table, lens = _numpy(kv)
    odd = append(codes, scales, table, lens, slots, rows, k.float().cpu().numpy(), v.float().cpu().numpy())
    E.entro_kv_append(kv, k, v, slots=ints(slots), row_start=None if single else starts(rows))
    assert E.entro_kv_status(kv) == (E.ERR_NONFINITE if odd else E.OK)
    assert np.array_equal(kv.scales.cpu().numpy(), scales)
    assert np.array_equal(kv.codes.cpu().numpy(), codes)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,dim,page", [(1, 64, 16), (3, 96, 32), (8, 128, 64), (2, 128, 128), (32, 64, 64), (2, 96, 128)])
def test_append_matches_float32_bit_for_bit(dtype, heads, dim, page):
    lens = [1, page, page + 1, 3 * page - 1, 2 * page + 7, 5, 4 * page]
    rows = [1, page, 1, 2 * page, page + 9, 3, 0]
    kv = make_cache(lens, heads, dim, page, seed=dim + page)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(sum(rows), 4 * heads, dim, device="cuda", generator=g).to(dtype)      # k and v as slices: strided
    x[3::5] *= 7
    slots = [3, 0, 6, 2, 4, 1, 5]
    kv.lens[:] = ints([lens[slots.index(s)] for s in range(7)])
    table = kv.table.clone()
    order = torch.argsort(ints(slots).long())
    kv.table.copy_(table[order])
    _append_and_compare(kv, slots, rows, x[:, heads:2 * heads], x[:, 3 * heads:])


def test_append_single_rows_growing_and_not_growing_scales():
    lens, heads, dim, page = [1, 16, 17, 40, 64, 33], 4, 128, 16
    kv = make_cache(lens, heads, dim, page, seed=5)
    for step, size in enumerate((0.01, 30.0, 1.0, 1e-4, 1000.0)):
        k = torch.randn(len(lens), heads, dim, device="cuda", generator=torch.Generator(device="cuda").manual_seed(step)).half()
        _append_and_compare(kv, list(range(len(lens))), [1] * len(lens), k * size, (k * 0.5).flip(0).contiguous(), single=True)


def test_append_zeros_tiny_huge_and_non_finite_values():
    heads, dim, page = 2, 64, 16
    kv = make_cache([40, 40, 40, 40], heads, dim, page)
    k = torch.randn(160, heads, dim, device="cuda").bfloat16()
    v = k.clone()
    k[:40] = 0
    v[:40] *= 1e-30
    k[40:80] *= 1e30
    k[85, 1, 3] = math.inf
    k[86, 0, 5] = -math.inf
    v[90, 1, 7] = math.nan
    v[100] = math.nan
    k[130:] = math.inf
    _append_and_compare(kv, [0, 1, 2, 3], [40] * 4, k, v)


def test_append_skips_absent_pages_slots_and_positions():
    heads, dim, page = 2, 64, 16
    kv = make_cache([40, 20, 10], heads, dim, page)
    kv.table[0, 1] = -1
    kv.table[1, 0] = 10 ** 6
    before = kv.codes.clone()
    k = torch.randn(40 + 20 + 5 + 25, heads, dim, device="cuda").half()
    codes, scales, table, lens = _numpy(kv)
    table = np.where((table >= 0) & (table < kv.pages), table, -1)
    append(codes, scales, table, lens, [0, 1], [40, 20], k[:60].float().cpu().numpy(), k[:60].float().cpu().numpy())
    # a slot that is not there, and a sequence with more rows than tokens: its first rows have no position
    append(codes, scales, table, lens, [2], [10], k[80:].float().cpu().numpy(), k[80:].float().cpu().numpy())
    kv2 = E.KvCache(kv.codes, kv.scales, torch.cat([kv.table, torch.full_like(kv.table[:1], -1)]),
                    torch.cat([kv.lens, kv.lens[:1] * 0]), kv.refs)
    E.entro_kv_append(kv2, k, k, slots=ints([0, 1, 99, 2]), row_start=starts([40, 20, 5, 25]))
    torch.cuda.synchronize()
    assert np.array_equal(kv.codes.cpu().numpy(), codes) and not torch.equal(kv.codes, before)
    assert np.array_equal(kv.scales.cpu().numpy(), scales)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,dim,page", [(1, 64, 16), (5, 96, 32), (8, 128, 64), (3, 128, 128)])
def test_read_returns_the_values_the_codes_stand_for(dtype, heads, dim, page):
    lens, rows, slots = [page + 3, 1, 2 * page, 7], [page + 1, 3, 2 * page, 0], [2, 0, 3, 1]
    kv = make_cache(lens, heads, dim, page, seed=3)
    kv.table[2, 1] = -1
    out = torch.empty(sum(rows), 3 * heads, dim, dtype=dtype, device="cuda")
    E.entro_kv_read(kv, slots=ints(slots), row_start=starts(rows), k=out[:, :heads], v=out[:, 2 * heads:])
    torch.cuda.synchronize()
    row = 0
    for slot, r in zip(slots, rows):
        for which, got in ((0, out[:, :heads]), (1, out[:, 2 * heads:])):
            n = lens[slot]
            for h in range(heads):
                # code * scale needs at most 32 bits: the 64-bit product rounded to 32 is the float32 product
                ref = sequence(kv, slot, which, h, n).float().nan_to_num(0.0).to(dtype)[max(0, n - r):]
                pad = r - ref.shape[0]
                assert (got[row:row + pad, h] == 0).all()
                assert torch.equal(got[row + pad:row + r, h], ref)
        row += r


# ----------------------------------------------------------------------------- attention

DIMS = [(1, 1, 64, 16), (4, 4, 96, 32), (8, 2, 128, 64), (32, 8, 128, 16), (6, 2, 64, 128), (7, 1, 96, 16), (16, 1, 128, 128),
        (24, 1, 64, 32)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,kv_heads,dim,page", DIMS)
def test_attention_of_single_tokens(heads, kv_heads, dim, page, dtype):
    lens = [1, 2, 15, 16, 17, 31, 33, 64, 65, 127, 128, 129, 255, 500, 1025, 0]
    kv = make_cache(lens, kv_heads, dim, page, seed=dim)
    slots = list(np.random.default_rng(dim).permutation(len(lens)))
    q = torch.randn(len(lens), heads, dim, device="cuda").to(dtype)
    assert_attention(kv, q, slots, [1] * len(lens))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (16, 16), (100, 33), (64, 0), (4096, 4), (2 ** 31, 0), (50, 2 ** 31)])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (96, 128)])
def test_attention_window_and_sinks(window, sinks, dim, page):
    lens = [1, 5, 40, 64, 130, 300, 777, 0]
    kv = make_cache(lens, 2, dim, page, seed=window % 1000 + sinks % 100)
    q = torch.randn(len(lens), 6, dim, device="cuda").half()
    assert_attention(kv, q, list(range(len(lens))), [1] * len(lens), window, sinks)
    rows = [1, 2, 40, 3, 129, 200, 300, 5]
    q = torch.randn(sum(rows), 6, dim, device="cuda").half()
    assert_attention(kv, q, list(range(len(lens))), rows, window, sinks)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,kv_heads,dim,page", DIMS)
def test_attention_of_prompts(heads, kv_heads, dim, page, dtype):
    lens = [1, 3, 128, 129, 257, 300, 700, 64, 511]
    rows = [1, 3, 128, 127, 130, 2, 333, 0, 511]
    kv = make_cache(lens, kv_heads, dim, page, seed=page)
    q = torch.randn(sum(rows), heads + 3, dim, device="cuda").to(dtype)[:, 1:1 + heads]      # strided
    assert_attention(kv, q, list(range(len(lens)))[::-1], rows[::-1])


def test_attention_rows_without_a_visible_token():
    """More rows than tokens, an empty sequence, a slot that is not there, pages that are not there."""
    kv = make_cache([10, 0, 40, 70], 2, 128, 16)
    kv.table[2, :] = -1
    kv.table[3, 1] = -1
    for rows in ([1, 1, 1, 1], [30, 2, 3, 70], [150, 9, 40, 64]):
        q = torch.randn(sum(rows), 8, 128, device="cuda").half()
        out, lse = assert_attention(kv, q, [0, 1, 2, 3], rows)
        assert (out[rows[0]:rows[0] + rows[1]] == 0).all() and torch.isinf(lse[rows[0]:rows[0] + rows[1]]).all()
    kv = make_cache([10, 12, 14], 2, 128, 16)
    q = torch.randn(3, 8, 128, device="cuda").half()
    assert_attention(kv, q, [0, 9, 2], [1, 1, 1])
    assert_attention(kv, q, [0, -1, 2], [1, 1, 1])


def test_attention_ignores_what_lies_behind_the_length():
    """Codes at the ends of the range and scales that are NaN or infinite where nothing visible lies."""
    for rows in ([1, 1, 1], [20, 100, 33]):
        kv = make_cache([37, 130, 64], 2, 64, 32, table_extra=3)
        q = torch.randn(sum(rows), 4, 64, device="cuda").half()
        a = assert_attention(kv, q, [0, 1, 2], rows)
        live = kv.table[kv.table >= 0].long()
        free = torch.ones(kv.pages, dtype=torch.bool, device="cuda")
        free[live] = False
        kv.scales[free] = math.nan
        kv.codes[free] = 255
        kv.table[0, 2:] = int(free.nonzero()[0])
        kv.codes[kv.table[0, 1], :, :, 5:] = 0          # the rest of the last page
        kv.codes[kv.table[1, 4], :, :, 2:] = 255
        b = E.entro_kv_attention(kv, q, slots=ints([0, 1, 2]), row_start=None if len(rows) == sum(rows) else starts(rows), return_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("rows", [1, 60])
def test_attention_with_scales_of_very_different_size(rows):
    """Pages whose scales lie 2^40 apart, large scores, and a softmax that sits on one token."""
    kv = make_cache([200, 333], 2, 128, 16, key_width=30.0)
    factors = torch.tensor([2.0 ** -20, 1.0, 2.0 ** 20, 2.0 ** -8], device="cuda")
    kv.scales[:, 1] *= factors[torch.arange(kv.pages, device="cuda") % 4][:, None]
    q = torch.randn(2 * rows, 4, 128, device="cuda").bfloat16()
    for scale in (None, 1e-3, 0.5):
        assert_attention(kv, q, [0, 1], [rows, rows], scale=scale)
    kv.scales[:] = 2.0 ** -60          # as an empty page of zeros has it
    assert_attention(kv, q, [0, 1], [rows, rows])


@pytest.mark.parametrize("rows", [1, 40])
def test_attention_of_queries_beyond_the_range_of_fp16(rows):
    kv = make_cache([150, 90], 1, 64, 16)
    q = torch.randn(2 * rows, 8, 64, device="cuda")
    q[0] *= 1e30
    q[1] *= 1e-30
    q[:, 2] = 0
    kv.scales[:, 0] *= 1e-3
    assert_attention(kv, q.bfloat16(), [0, 1], [rows, rows], scale=1e-30)
    q = q.clamp(-60000, 60000).half()
    assert_attention(kv, q, [0, 1], [rows, rows], scale=1e-4)


@pytest.mark.parametrize("rows", [1, 30])
def test_attention_nan_and_infinity_in_a_query_stay_in_their_row(rows):
    kv = make_cache([150, 90], 1, 64, 16)
    for dtype in (torch.float16, torch.bfloat16):
        q = torch.randn(2 * rows, 8, 64, device="cuda").to(dtype)
        q2 = q.clone()
        q2[0, 3, 5] = math.nan
        q2[rows, 6, 1] = math.inf
        start = None if rows == 1 else starts([rows, rows])
        a = E.entro_kv_attention(kv, q, slots=ints([0, 1]), row_start=start)
        b = E.entro_kv_attention(kv, q2, slots=ints([0, 1]), row_start=start)
        same = torch.ones(2 * rows, 8, dtype=torch.bool, device="cuda")
        same[0, 3] = same[rows, 6] = False
        assert torch.equal(a[same], b[same])
        assert b[0, 3].isnan().all() and b[rows, 6].isnan().all()


@pytest.mark.parametrize("seqs,length,kv_heads,group,dim,page,rows", [
    (1, 20001, 1, 8, 128, 64, 1), (1, 9001, 8, 4, 128, 16, 1), (3, 5003, 2, 1, 96, 128, 1), (2, 6000, 1, 4, 64, 32, 4),
    (1, 4100, 2, 16, 64, 16, 1), (1, 9000, 1, 4, 128, 64, 100), (2, 3000, 2, 2, 96, 16, 700), (1, 2500, 1, 1, 64, 128, 2500)])
def test_attention_split_over_a_long_axis(seqs, length, kv_heads, group, dim, page, rows):
    lens = [length - 17 * i for i in range(seqs)]
    kv = make_cache(lens, kv_heads, dim, page, seed=length)
    q = torch.randn(seqs * rows, kv_heads * group, dim, device="cuda").half()
    a = assert_attention(kv, q, list(range(seqs)), [rows] * seqs)
    b = assert_attention(kv, q, list(range(seqs)), [rows] * seqs)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])          # no order of arrival in the result
    assert_attention(kv, q, list(range(seqs)), [rows] * seqs, window=1111, sinks=5)


def test_attention_mixed_batch_with_and_without_the_bound_on_rows():
    lens, rows = [900, 300, 1500, 64, 5, 800], [1, 300, 1, 64, 2, 9]
    kv = make_cache(lens, 2, 128, 32)
    q = torch.randn(sum(rows), 8, 128, device="cuda").half()
    a = assert_attention(kv, q, list(range(6)), rows)
    b = assert_attention(kv, q, list(range(6)), rows, max_rows=300)
    assert torch.equal(a[0], b[0])
    rows = [1, 3, 2, 1, 2, 1]
    q = torch.randn(sum(rows), 8, 128, device="cuda").half()
    assert_attention(kv, q, list(range(6)), rows, max_rows=3)
    assert_attention(kv, q, list(range(6)), rows)


def test_attention_writes_strided_outputs_and_nothing_else():
    kv = make_cache([100, 40], 2, 96, 16)
    for rows in ([1, 1], [50, 40]):
        q = torch.randn(sum(rows), 4, 96, device="cuda").half()
        whole = torch.full((sum(rows), 7, 96 + 16), 5.0, dtype=torch.float16, device="cuda")
        out = whole[:, 1:5, 8:104]
        E.entro_kv_attention(kv, q, slots=ints([0, 1]), row_start=None if rows[0] == 1 else starts(rows), out=out)
        ref = E.entro_kv_attention(kv, q, slots=ints([0, 1]), row_start=None if rows[0] == 1 else starts(rows))
        assert torch.equal(out, ref)
        whole[:, 1:5, 8:104] = 5.0
        assert (whole == 5.0).all()


def test_attention_many_sequences():
    rng = np.random.default_rng(7)
    lens = rng.integers(0, 90, 700).tolist()
    kv = make_cache(lens, 1, 64, 16)
    slots = rng.permutation(700).tolist()
    q = torch.randn(700, 2, 64, device="cuda").half()
    assert_attention(kv, q, slots, [1] * 700)
    rows = [min(n, int(r)) for n, r in zip([lens[s] for s in slots], rng.integers(0, 20, 700))]
    q = torch.randn(sum(rows), 2, 64, device="cuda").half()
    assert_attention(kv, q, slots, rows)


def test_cache_larger_than_32_bits():
    """Pages whose bytes start behind 2^32: write, read, attend and move there."""
    heads, dim, page = 8, 128, 128
    pages = (1 << 32) // (2 * heads * dim * page) + 40
    kv = E.entro_kv_create(pages, heads, dim, page, 3, 2000)
    lens = [700, 300, 0]
    kv.lens[:] = ints(lens)
    kv.table[0, :6] = torch.arange(pages - 1, pages - 7, -1, device="cuda").to(torch.int32)
    kv.table[1, :3] = ints([pages - 20, 3, pages - 30])
    for p in kv.table[kv.table >= 0].tolist():
        kv.refs[p] = 1
    k = torch.randn(1000, heads, dim, device="cuda").half()
    v = torch.randn(1000, heads, dim, device="cuda").half()
    E.entro_kv_append(kv, k, v, slots=ints([0, 1]), row_start=starts([700, 300]))
    a, b = E.entro_kv_read(kv, 1000, slots=ints([0, 1]), row_start=starts([700, 300]))
    assert (a - k).abs().max() < 0.03 and (b - v).abs().max() < 0.03
    for rows in ([1, 1], [200, 100]):
        q = torch.randn(sum(rows), 16, dim, device="cuda").half()
        before = assert_attention(kv, q, [0, 1], rows)
        E.entro_kv_fork(kv, ints([0]), ints([2]))
        assert kv.lens.tolist() == [700, 300, 700]
        E.entro_kv_compact(kv)
        assert int(kv.table.max()) == 9
        after = E.entro_kv_attention(kv, q, slots=ints([2, 1]), row_start=None if rows[0] == 1 else starts(rows))
        assert torch.equal(before[0], after)


def test_calls_on_another_stream_and_in_a_graph():
    lens = [100, 31, 64]
    kv = make_cache(lens, 2, 128, 32)
    q, k, v = (torch.randn(3, h, 128, device="cuda").half() for h in (8, 2, 2))
    slots = ints([0, 1, 2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.zeros(3, 8, 128, dtype=torch.float16, device="cuda")

    def step(stream=None):
        E.entro_kv_reserve(kv, slots=slots, stream=stream)
        E.entro_kv_append(kv, k, v, slots=slots, stream=stream)
        E.entro_kv_attention(kv, q, slots=slots, out=out, stream=stream)

    step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert kv.lens.tolist() == [101, 32, 65]
    assert torch.equal(out, assert_attention(kv, q, [0, 1, 2], [1, 1, 1])[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    assert kv.lens.tolist() == [101, 32, 65]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert kv.lens.tolist() == [104, 35, 68] and E.entro_kv_status(kv) == E.OK
    assert torch.equal(out, assert_attention(kv, q, [0, 1, 2], [1, 1, 1])[0])


# ----------------------------------------------------------------------------- page operations

def _random_pool(seed, page=16, pages=61, slots=9, width=9):
    kv = E.entro_kv_create(pages, 2, 64, page, slots, width * page)
    kv.codes.random_(0, 256)
    kv.scales.uniform_(0.5, 2.0)
    return kv, Pages(kv), np.random.default_rng(seed)


def _values(kv, slot):
    n = int(kv.lens[slot])
    return torch.stack([sequence(kv, slot, w, h, n) for w in range(2) for h in range(2)]) if n else None


@pytest.mark.parametrize("seed", range(6))
def test_page_operations_against_lists(seed):
    kv, ref, rng = _random_pool(seed, pages=[61, 40, 200, 30, 3000, 64][seed])
    for step in range(60):
        op = rng.integers(0, 6)
        some = rng.permutation(kv.slots)[:rng.integers(1, kv.slots + 1)].tolist()
        before = {s: _values(kv, s) for s in range(kv.slots)}
        if op <= 1:
            room = [kv.table_width * kv.page_tokens - ref.lens[s] for s in some]
            rows = [int(min(r, rng.integers(0, 50))) for r in room]
            E.entro_kv_reserve(kv, slots=ints(some), row_start=starts(rows))
            ref.reserve(some, rows)
            some = list(range(kv.slots))          # contents of what was added are not defined
        elif op == 2:
            E.entro_kv_free(kv, ints(some))
            ref.free(some)
        elif op == 3:
            src = rng.integers(0, kv.slots, len(some)).tolist()
            E.entro_kv_fork(kv, ints(src), ints(some))
            ref.fork(src, some)
            for s, d in zip(src, some):
                if not ref.short:
                    a, b = before[s], _values(kv, d)
                    assert (a is None and b is None) or torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))
        elif op == 4:
            E.entro_kv_compact(kv)
            ref.compact()
            some = []
        else:
            window, sinks = int(rng.integers(0, 80)), int(rng.integers(0, 20))
            E.entro_kv_trim(kv, ints(some), window, sinks)
            ref.trim(some, window, sinks)
        torch.cuda.synchronize()
        ref.assert_same(kv)
        for s in range(kv.slots):
            if s not in some and before[s] is not None:
                assert torch.equal(before[s].nan_to_num(7.0), _values(kv, s).nan_to_num(7.0))
        assert E.entro_kv_status(kv) == (E.ERR_NO_PAGES if ref.short else E.OK)
        if ref.short:
            everything = list(range(kv.slots))
            E.entro_kv_free(kv, ints(everything))
            ref.free(everything)
            ref.short = False
            ref.assert_same(kv)


def test_single_rows_reserve_across_page_ends():
    kv, ref, _ = _random_pool(1)
    for _ in range(40):
        E.entro_kv_reserve(kv, slots=ints([4, 2, 7]))
        ref.reserve([4, 2, 7], [1, 1, 1])
        ref.assert_same(kv)


def test_large_pool_with_many_sequences():
    pages, slots, width = 20000, 900, 30
    kv = E.entro_kv_create(pages, 1, 64, 16, slots, width * 16)
    ref, rng = Pages(kv), np.random.default_rng(3)
    order = rng.permutation(slots).tolist()
    rows = rng.integers(0, 400, slots).tolist()
    E.entro_kv_reserve(kv, slots=ints(order), row_start=starts(rows))
    ref.reserve(order, rows)
    ref.assert_same(kv)
    E.entro_kv_free(kv, ints(order[:300]))
    ref.free(order[:300])
    src = rng.integers(0, slots, 500).tolist()
    E.entro_kv_fork(kv, ints(src), ints(order[:500]))
    ref.fork(src, order[:500])
    ref.assert_same(kv)
    E.entro_kv_compact(kv)
    ref.compact()
    ref.assert_same(kv)
    assert E.entro_kv_status(kv) == E.OK


def test_trimmed_cache_gives_the_same_windowed_attention():
    for rows in (1, 5, 60):
        kv = make_cache([500, 333, 64], 2, 64, 16)
        q = torch.randn(3 * rows, 4, 64, device="cuda").half()
        start = None if rows == 1 else starts([rows] * 3)
        a = E.entro_kv_attention(kv, q, slots=ints([0, 1, 2]), row_start=start, window=100, sinks=20)
        E.entro_kv_trim(kv, ints([0, 1, 2]), 100 + rows - 1, 20)
        assert int((kv.refs == 0).sum()) > 20
        kv.codes[kv.refs == 0] = 255
        b = E.entro_kv_attention(kv, q, slots=ints([0, 1, 2]), row_start=start, window=100, sinks=20)
        assert torch.equal(a, b)
