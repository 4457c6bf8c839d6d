"""Plain restatements of the key/value cache operators for the tests: attention in 64 bits with a
bound on what the kernel may differ by, quantised writing in IEEE float32 (NumPy), and the page
bookkeeping as Python lists.  Written from include/entro.h."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2505_02380_b200 as E

ZERO = 128


def make_cache(lens, kv_heads, dim, page, seed=0, spare=3, extra_slots=0, key_width=2.5, table_extra=1, pages=None):
    """A cache whose sequences (slot i has lens[i] tokens) lie on scattered pages."""
    g = torch.Generator().manual_seed(seed)
    used = [-(-n // page) for n in lens]
    pages = sum(used) + spare if pages is None else pages
    kv = E.entro_kv_create(pages, kv_heads, dim, page, len(lens) + extra_slots, max(1, (max(used) + table_extra) * page))
    kv.codes.copy_((torch.randn(kv.codes.shape, generator=g) * 36).round().clamp(-127, 127) + ZERO)
    kv.scales.copy_((0.7 + 0.7 * torch.rand(kv.scales.shape, generator=g)) * torch.tensor([key_width / 36, 1 / 36])[None, :, None])
    order = torch.randperm(pages, generator=g).to(torch.int32)
    at = 0
    for i, n in enumerate(used):
        kv.table[i, :n] = order[at:at + n].cuda()
        at += n
    kv.refs[order[:at].long().cuda()] = 1
    kv.lens[:len(lens)] = torch.tensor(lens, dtype=torch.int32)
    return kv


def sequence(kv, slot, which, head, n):
    """The first n tokens of a sequence in 64 bits [n, dim]; tokens without a page are NaN."""
    page = kv.page_tokens
    ids = kv.table[slot, :-(-n // page)].long()
    x = (kv.codes[ids.clamp_min(0), which, head].double() - ZERO) * kv.scales[ids.clamp_min(0), which, head].double()[:, None, None]
    x[ids < 0] = math.nan
    return x.reshape(-1, kv.head_dim)[:n]


def attention(kv, q, slots, rows, window, sinks, scale=None):
    """-> out, lse in 64 bits, and how far the kernel's may be from them: (out64, lse64, out_bound, lse_bound).

    The kernel's score is a float32 sum of dim exact products (bound dim * 2^-23 of the sum of their
    magnitudes, whatever the order and rounding of the sum), times float32 factors, and goes through an
    exp2 whose argument and result are good to about 2^-20 together.  A probability is rounded to fp16:
    2^-11 of itself, or 2^-25 of the largest term.  The result is rounded once to the output's type.
    """
    total, heads, dim = q.shape
    per = heads // kv.kv_heads
    scale = dim ** -0.5 if scale is None else scale
    out = torch.zeros(total, heads, dim, dtype=torch.float64, device=q.device)
    lse = torch.full((total, heads), -math.inf, dtype=torch.float64, device=q.device)
    out_bound, lse_bound = torch.zeros_like(out), torch.zeros(total, heads, dtype=torch.float64, device=q.device)
    unit = 2.0 ** (-11 if q.dtype == torch.float16 else -8)
    lens = kv.lens.tolist()
    row = 0
    for slot, r in zip(slots, rows):
        n = lens[slot] if 0 <= slot < kv.slots else 0
        if n == 0 or r == 0:
            row += r
            continue
        p = torch.arange(n - r, n, device=q.device)[:, None]
        j = torch.arange(n, device=q.device)[None]
        sees = (j <= p)
        if window:
            sees &= (j > p - window) | (j < sinks)
        for h in range(heads):
            k, v = sequence(kv, slot, 0, h // per, n), sequence(kv, slot, 1, h // per, n)
            there = ~k.isnan().any(1)
            k, v = k.nan_to_num(0.0), v.nan_to_num(0.0)
            ok = sees & there[None]
            x = q[row:row + r, h].double()
            s = (x @ k.T * scale).masked_fill(~ok, -math.inf)
            some = ok.any(1)
            size = ((x.abs() @ k.abs().T) * scale * ok).amax(1)
            ds = dim * 2.0 ** -23 * size + 2.0 ** -20 * (1 + size)
            w = torch.softmax(s, 1).nan_to_num(0.0)
            out[row:row + r, h] = w @ v
            lse[row:row + r, h] = torch.logsumexp(s, 1)
            spread = w @ v.abs()
            out_bound[row:row + r, h] = (2.0 ** -11 + 2 * ds)[:, None] * spread + n * 2.0 ** -25 * v.abs().amax() \
                + unit * (out[row:row + r, h].abs() + 2.0 ** -14)
            lse_bound[row:row + r, h] = torch.where(some, ds + 2.0 ** -21 * lse[row:row + r, h].abs(), 0.0)
        row += r
    return out, lse, out_bound, lse_bound


def assert_attention(kv, q, slots, rows, window=0, sinks=0, scale=None, **kw):
    """Runs the kernel and holds it to the bound.  -> (out, lse)"""
    start = None if all(r == 1 for r in rows) and kw.pop("single", True) else starts(rows)
    kw.pop("single", None)
    out, lse = E.entro_kv_attention(kv, q, slots=ints(slots), row_start=start, window=window, sinks=sinks,
                                    softmax_scale=0.0 if scale is None else scale, return_lse=True, **kw)
    torch.cuda.synchronize()
    ref, ref_lse, bound, lse_bound = attention(kv, q, slots, rows, window, sinks, scale)
    finite = ref_lse > -math.inf
    assert torch.equal(lse > -math.inf, finite)
    d = (lse.double() - ref_lse)[finite].abs()
    assert (d <= lse_bound[finite]).all(), (d / lse_bound[finite]).max()
    d = (out.double() - ref).abs()
    assert (d <= bound).all(), (d / bound).nan_to_num(math.inf).max()
    assert (out[~finite] == 0).all()
    return out, lse


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def starts(rows):
    return ints([0] + np.cumsum(rows).tolist())


def append(codes, scales, table, lens, slots, rows, k, v):
    """Writes rows into NumPy copies of the cache (codes uint8, scales float32), in float32 arithmetic.
    k, v float32 [rows, heads, dim].  -> whether a value was not finite."""
    page = codes.shape[3]
    row, odd = 0, False
    for slot, r in zip(slots, rows):
        n = int(lens[slot])
        begin = max(0, n - r)
        for block in range(begin // page, -(-n // page)):
            lo, hi = max(begin, block * page), min(n, (block + 1) * page)
            at = table[slot, block] if block < table.shape[1] else -1
            if at < 0:
                continue
            for which, x in ((0, k), (1, v)):
                new = x[row + lo - (n - r):row + hi - (n - r)]                 # [tokens, heads, dim]
                finite = np.isfinite(new)
                odd |= not finite.all()
                top = np.where(finite, np.abs(new), np.float32(0)).max((0, 2)).astype(np.float32)
                old = scales[at, which] if lo > block * page else np.zeros_like(top)
                s = np.maximum(np.maximum(old, top / np.float32(127)), np.float32(2.0 ** -60)).astype(np.float32)
                kept = codes[at, which, :, :lo - block * page].astype(np.float32) - np.float32(ZERO)
                ratio = (old / s).astype(np.float32)
                codes[at, which, :, :lo - block * page] = (np.rint(kept * ratio[:, None, None]) + ZERO).astype(np.uint8)
                with np.errstate(over="ignore", invalid="ignore"):
                    y = np.rint(new / s[None, :, None]).clip(-127, 127)
                y = np.where(np.isnan(new), np.float32(0), y)
                codes[at, which, :, lo - block * page:hi - block * page] = (y + ZERO).astype(np.uint8).transpose(1, 0, 2)
                scales[at, which] = s
        row += r
    return odd


class Pages:
    """The bookkeeping of tables, lengths and counts as Python lists."""

    def __init__(self, kv):
        self.table, self.lens, self.refs = kv.table.tolist(), kv.lens.tolist(), kv.refs.tolist()
        self.page, self.width, self.moves, self.short = kv.page_tokens, kv.table_width, [], False

    def blocks(self, n):
        return min(self.width, -(-n // self.page))

    def take(self):
        for p, r in enumerate(self.refs):
            if r <= 0:
                self.refs[p] = 1
                return p
        self.short = True
        return -1

    def reserve(self, slots, rows):
        for s, r in zip(slots, rows):
            n = self.lens[s] + r
            if n > self.width * self.page:
                self.short = True
            for e in range(self.blocks(self.lens[s]), self.blocks(n)):
                self.table[s][e] = self.take()
            self.lens[s] = n

    def free(self, slots):
        for s in slots:
            for e in range(self.blocks(self.lens[s])):
                if self.table[s][e] >= 0:
                    self.refs[self.table[s][e]] -= 1
                self.table[s][e] = -1
            self.lens[s] = 0

    def trim(self, slots, window, sinks):
        for s in slots:
            for e in range(self.blocks(self.lens[s])):
                if e * self.page >= sinks and (e + 1) * self.page <= self.lens[s] - window and window:
                    if self.table[s][e] >= 0:
                        self.refs[self.table[s][e]] -= 1
                    self.table[s][e] = -1

    def fork(self, src, dst):
        pairs = [(s, d) for s, d in zip(src, dst) if s != d]
        new = [(list(self.table[s]), self.lens[s]) for s, _ in pairs]
        tails = []
        for row, n in new:
            for p in row[:self.blocks(n)]:
                if p >= 0:
                    self.refs[p] += 1
        for _, d in pairs:
            for p in self.table[d][:self.blocks(self.lens[d])]:
                if p >= 0:
                    self.refs[p] -= 1
        for row, n in new:
            e = n // self.page
            if n % self.page and e < self.width and row[e] >= 0:
                tails.append((row, e, row[e]))
        for row, e, old in tails:
            row[e] = self.take()
            if row[e] >= 0:
                self.moves.append((old, row[e]))
        for _, _, old in tails:
            self.refs[old] -= 1
        for (_, d), (row, n) in zip(pairs, new):
            self.table[d] = row[:self.blocks(n)] + [-1] * (self.width - self.blocks(n))
            self.lens[d] = n

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] <= 0]
        movers = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.moves.append((a, b))
        self.table = [[to.get(p, p) for p in row] for row in self.table]

    def assert_same(self, kv):
        assert kv.table.tolist() == self.table
        assert kv.lens.tolist() == self.lens
        assert kv.refs.tolist() == self.refs
