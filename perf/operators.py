"""Cases for the operators on the paged 8-bit key/value cache, and their plain forms in elementary torch operations.

Cache layout (include/entro.h, entro_kv_cache): codes uint8 [pages, 2, kv_heads, page, dim], value = scale * (code - 128) with
one float32 scale per [page, K or V, kv_head]; table int32 [slots, width] of page numbers (-1: none), lens int32 [slots],
refs int32 [pages] (table entries that name a page).  The rows given for a sequence are its last rows.
"""
import math
import random

import torch

own = False

ZERO = 128          # code of the value 0
FLOOR = 2.0 ** -60  # smallest scale


# ----------------------------------------------------------------------------- cases

def _attend(name, **kw):
    case = dict(name=name, op="attend", type="float16", heads=32, kv_heads=8, dim=128, page=64, seqs=1, len_min=1, len_max=1024,
                rows_min=1, rows_max=1, window=0, sinks=0, mix=1)
    case.update(kw)
    return case


def _append(name, **kw):
    case = dict(name=name, op="append", type="float16", heads=32, kv_heads=8, dim=128, page=64, seqs=1, len_min=1, len_max=1024,
                rows_min=1, rows_max=1, mix=1)
    case.update(kw)
    return case


def listed():
    return [
        # one user, one new token, a short conversation: what counts is latency (mistral-shaped heads)
        _attend("token_one", page=16, len_min=777, len_max=777),
        # a server's ragged batch, one new token each, from a first token to 8192
        _attend("token_batch", type="bfloat16", seqs=64, len_min=1, len_max=8192, mix=2),
        # a few very long documents: the largest cache, bound by memory alone
        _attend("token_long", seqs=8, len_min=131072, len_max=131072, mix=3),
        # phi3-shaped heads (as many key/value heads as queries, 96 wide), sliding window with four sinks
        _attend("token_window", kv_heads=32, dim=96, page=32, seqs=16, len_min=900, len_max=4001, window=2047, sinks=4, mix=4),
        # a short first prompt (smolLM-shaped heads), an odd number of tokens
        _attend("prompt_short", kv_heads=32, dim=64, page=16, len_min=173, len_max=173, rows_min=173, rows_max=173, mix=5),
        # a whole long prompt at once: the largest amount of arithmetic
        _attend("prompt_whole", type="bfloat16", len_min=8192, len_max=8192, rows_min=8192, rows_max=8192, mix=6),
        # prompts fed in chunks behind long contexts, window and sinks, beside sequences that bring few rows
        _attend("prompt_chunks", page=128, seqs=4, len_min=5003, len_max=16001, rows_min=9, rows_max=1024, window=4096, sinks=4, mix=7),
        # the new token of every sequence of a batch goes into the cache
        _append("append_step", seqs=64, len_min=2, len_max=4096, mix=8),
        # several prompts go into the cache together, the first tokens of some already there
        _append("append_prompts", type="bfloat16", kv_heads=32, dim=96, page=32, seqs=5, len_min=701, len_max=5001, rows_min=700,
                rows_max=4096, mix=9),
        # beam search: surviving beams are carried on in the places of the others
        dict(name="fork_beams", op="fork", kv_heads=8, dim=128, page=64, groups=16, beams=4, len_min=100, len_max=4000, mix=10),
        # sequences come and go in a small pool
        dict(name="churn_small", op="churn", kv_heads=4, dim=64, page=16, groups=3, seqs=2, len_min=5, len_max=300, mix=11),
        # the same in a large pool: a quarter of it is freed, the rest moved together, the quarter filled again
        dict(name="churn_large", op="churn", kv_heads=8, dim=128, page=64, groups=4, seqs=16, len_min=500, len_max=6000, mix=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["token", "token", "token", "prompt", "prompt", "append", "append", "fork", "churn"])
    kv, group = rng.choice([(1, 8), (2, 7), (4, 3), (8, 1), (8, 2), (8, 4), (8, 8), (32, 1)])
    base = dict(heads=kv * group, kv_heads=kv, dim=rng.choice([64, 96, 128]), page=rng.choice([16, 32, 64, 128]), mix=rng.randrange(1 << 20))
    real = rng.choice(["float16", "bfloat16"])
    if op == "token":
        seqs = _log(rng, 1, 128)
        most = max(64, min(131072, (1 << 20) * 8 // (seqs * kv)))
        top = _log(rng, 1, most)
        windowed = rng.random() < 0.4
        return dict(base, op="attend", type=real, seqs=seqs, len_min=_log(rng, 1, top), len_max=top, rows_min=1, rows_max=1,
                    window=_log(rng, 1, 8192) if windowed else 0, sinks=rng.choice([0, 1, 4, 33]) if windowed else 0)
    if op == "prompt":
        seqs = rng.choice([1, 1, 2, 3, 6])
        most = int(math.sqrt(8192 * 8192 * 32 / (seqs * kv * group)))
        rows = _log(rng, 2, min(8192, most))
        top = max(rows, _log(rng, rows, max(rows, min(32768, 8192 * 8192 * 16 // (seqs * kv * group * rows)))))
        windowed = rng.random() < 0.4
        return dict(base, op="attend", type=real, seqs=seqs, len_min=rows, len_max=top, rows_min=_log(rng, 1, rows), rows_max=rows,
                    window=_log(rng, 1, 8192) if windowed else 0, sinks=rng.choice([0, 1, 4, 33]) if windowed else 0)
    if op == "append":
        seqs = _log(rng, 1, 128)
        rows = rng.choice([1, _log(rng, 1, max(2, 16384 // seqs))])
        return dict(base, op="append", type=real, seqs=seqs, len_min=rows, len_max=rows + _log(rng, 1, 4096), rows_min=_log(rng, 1, rows),
                    rows_max=rows)
    top = _log(rng, 2, 4096)
    del base["heads"]
    if op == "fork":
        return dict(base, op="fork", groups=_log(rng, 1, 32), beams=rng.choice([2, 3, 4, 8]), len_min=_log(rng, 1, top), len_max=top)
    return dict(base, op="churn", groups=rng.choice([2, 3, 4, 6]), seqs=_log(rng, 1, 16), len_min=_log(rng, 1, top), len_max=top)


def _spread(rng, lo, hi, n):
    """n whole numbers from lo to hi, spread over their logarithm, both ends among them."""
    got = [_log(rng, lo, hi) for _ in range(n)]
    got[0] = hi
    if n > 1:
        got[1] = lo
    return got


def _lens_rows(case):
    """Tokens and rows of every sequence: part of the case, the same for every seed."""
    rng = random.Random(case["mix"])
    rows = _spread(rng, case["rows_min"], case["rows_max"], case["seqs"])
    lens = [max(length, r) for length, r in zip(_spread(rng, case["len_min"], case["len_max"], case["seqs"]), rows)]
    return lens, rows


def _blocks(tokens, page):
    return -(-tokens // page)


def _seen(length, rows, window, sinks):
    """(tokens that some row sees, pairs of row and token that it sees)"""
    pairs = 0
    first = length - rows
    if not window:
        pairs = rows * first + rows * (rows + 1) // 2
        return length, pairs
    for p in range(first, length):
        near = max(0, p - window + 1)
        pairs += p + 1 - near + min(sinks, near)
    near = max(0, first - window + 1)
    return length - near + min(sinks, near), pairs


def work(case):
    h, d, page = case["kv_heads"], case["dim"], case["page"]
    page_bytes = 2 * h * page * d
    if case["op"] == "attend":
        lens, rows = _lens_rows(case)
        seen = [_seen(n, r, case["window"], case["sinks"]) for n, r in zip(lens, rows)]
        tokens, pairs, total = sum(s[0] for s in seen), sum(s[1] for s in seen), sum(rows)
        scales = sum(_blocks(s[0], page) for s in seen) * 2 * h * 4
        return {"bytes": tokens * 2 * h * d + scales + total * case["heads"] * (4 * d + 4), "flops": 4 * d * case["heads"] * pairs}
    if case["op"] == "append":
        lens, rows = _lens_rows(case)
        total = sum(rows)
        back = _back(case) * case["seqs"]
        # new values in (2 bytes), codes out (1), then the values that come back: codes in (1), values out (2)
        return {"bytes": total * 2 * h * d * 3 + back * 2 * h * d * 3, "flops": 4 * total * 2 * h * d}
    if case["op"] == "fork":
        lens, parents = _fork_plan(case)
        moved = sum(1 for i, p in enumerate(parents) if p != i and lens[i // case["beams"]] % page)
        entries = sum(_blocks(lens[i // case["beams"]], page) for i, p in enumerate(parents) if p != i)
        return {"bytes": moved * 2 * page_bytes + entries * 16, "flops": 0}
    lens = _churn_lens(case)
    pages = [sum(_blocks(n, page) for n in g) for g in lens]
    moved = sum(min(p, sum(pages) - p) for p in pages) / len(pages)
    return {"bytes": moved * 2 * page_bytes + sum(pages) * 8, "flops": 0}


# ----------------------------------------------------------------------------- inputs

def _back(case):
    """Rows per sequence that an append case reads back: at least a whole page, so that a rescaled page is seen whole."""
    return max(case["rows_max"], case["page"])


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _random_codes(gen, pages, h, page, d):
    """Codes as quantising bell-shaped values leaves them: a spread of about 36 steps."""
    codes = torch.empty(pages, 2, h, page, d, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (2 * h * page * d))
    for at in range(0, pages, step):
        part = codes[at:at + step]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(36).round_().clamp_(-127, 127).add_(ZERO))
    return codes


def _cache(gen, case, lens_of_slots, spare, width):
    """A pool in which every slot's pages lie scattered."""
    page, h, d = case["page"], case["kv_heads"], case["dim"]
    used = [_blocks(n, page) for n in lens_of_slots]
    pages = sum(used) + spare
    codes = _random_codes(gen, pages, h, page, d)
    # keys about 2.5 wide (scores of a few units), values about 1 wide, each page and head with a scale of its own
    scales = torch.empty(pages, 2, h, device="cuda").uniform_(0.7, 1.4, generator=gen)
    scales *= torch.tensor([2.5 / 36, 1.0 / 36], device="cuda")[None, :, None]
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    start = torch.tensor([sum(used[:i]) for i in range(len(used))], device="cuda")
    count = torch.tensor(used, device="cuda")
    block = torch.arange(width, device="cuda")
    held = block[None] < count[:, None]
    table = torch.where(held, order[(start[:, None] + block[None]).clamp_max(pages - 1)], -1).to(torch.int32).contiguous()
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[table[held].long()] = 1
    lens = torch.tensor(lens_of_slots, dtype=torch.int32, device="cuda")
    return dict(codes=codes, scales=scales, table=table, lens=lens, refs=refs)


def _starts(rows):
    at = [0]
    for r in rows:
        at.append(at[-1] + r)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = _generator(seed)
    page, h, d = case["page"], case["kv_heads"], case["dim"]
    if case["op"] in ("attend", "append"):
        real = getattr(torch, case["type"])
        lens, rows = _lens_rows(case)
        st = _cache(gen, case, lens, 3, max(_blocks(n, page) for n in lens) + 1)
        st["slots"] = torch.randperm(len(lens), generator=gen, device="cuda").to(torch.int32)   # sequences in any order
        inverse = torch.argsort(st["slots"].long())
        st["table"], st["lens"] = st["table"][inverse].contiguous(), st["lens"][inverse].contiguous()
        # queries, keys and values of the new rows as one projection leaves them: side by side
        qkv = torch.randn(sum(rows), case["heads"] + 2 * h, d, generator=gen, device="cuda").to(real)
        st["q"], st["k"], st["v"] = qkv.split([case["heads"], h, h], dim=1)
        st["k"].mul_(2.5)
        st["row_start"] = None if max(rows) == 1 else _starts(rows)
        st["max_rows"], st["max_len"] = max(rows), max(lens)
        if case["op"] == "attend":      # a server keeps the places its results go to
            st["out"] = torch.empty(sum(rows), case["heads"], d, dtype=real, device="cuda")
            st["lse"] = torch.empty(sum(rows), case["heads"], device="cuda")
        if case["op"] == "append":
            st["back_start"] = _starts([_back(case)] * len(rows))
            st["back_rows"] = _back(case) * len(rows)
    elif case["op"] == "fork":
        lens, parents = _fork_plan(case)
        w = case["beams"]
        slots = [n for n in lens for _ in range(w)]
        width = max(_blocks(n, page) for n in lens) + 1
        st = _cache(gen, case, slots, len(slots) + 2, width)
        pairs = [(p, i) for i, p in enumerate(parents)]
        st["src"] = torch.tensor([p for p, _ in pairs], dtype=torch.int32, device="cuda")
        st["dst"] = torch.tensor([i for _, i in pairs], dtype=torch.int32, device="cuda")
    else:
        lens = _churn_lens(case)
        flat = [n for g in lens for n in g]
        st = _cache(gen, case, flat, max(2, sum(_blocks(n, page) for n in flat) // 16), max(_blocks(n, page) for n in flat) + 1)
        n = case["seqs"]
        st["groups"] = [(torch.arange(g * n, (g + 1) * n, dtype=torch.int32, device="cuda"), _starts(lens[g])) for g in range(case["groups"])]
        st["turn"] = 0
    st["case"] = case
    return st


def _fork_plan(case):
    """Length of every group, and the parent slot of every beam; survivors are their own parents."""
    rng = random.Random(case["mix"])
    lens = _spread(rng, case["len_min"], case["len_max"], case["groups"])
    w, parents = case["beams"], []
    for g in range(case["groups"]):
        keep = rng.sample(range(w), rng.randint(1, w - 1))
        parents += [g * w + (i if i in keep else rng.choice(keep)) for i in range(w)]
    return lens, parents


def _churn_lens(case):
    rng = random.Random(case["mix"])
    flat = _spread(rng, case["len_min"], case["len_max"], case["groups"] * case["seqs"])
    rng.shuffle(flat)
    return [flat[g * case["seqs"]:(g + 1) * case["seqs"]] for g in range(case["groups"])]


# ----------------------------------------------------------------------------- one pass

def run(st):
    op = st["case"]["op"]
    if own:
        import paper_2505_02380_b200 as E
        kv = st.get("kv")
        if kv is None:
            kv = st["kv"] = E.KvCache(st["codes"], st["scales"], st["table"], st["lens"], st["refs"])
        if op == "attend":
            c = st["case"]
            return E.entro_kv_attention(kv, st["q"], slots=st["slots"], row_start=st["row_start"], max_rows=st["max_rows"],
                                        window=c["window"], sinks=c["sinks"], out=st["out"], lse=st["lse"])
        if op == "append":
            E.entro_kv_append(kv, st["k"], st["v"], slots=st["slots"], row_start=st["row_start"])
            k, v = E.entro_kv_read(kv, st["back_rows"], slots=st["slots"], row_start=st["back_start"], dtype=st["k"].dtype)
            return k, v, st["scales"]
        if op == "fork":
            E.entro_kv_fork(kv, st["src"], st["dst"])
        else:
            slots, starts = st["groups"][st["turn"] % len(st["groups"])]
            st["turn"] += 1
            E.entro_kv_free(kv, slots)
            E.entro_kv_compact(kv)
            E.entro_kv_reserve(kv, slots=slots, row_start=starts)
    elif op == "attend":
        return _plain_attend(st)
    elif op == "append":
        _plain_append(st)
        return _plain_read(st)
    elif op == "fork":
        _plain_fork(st)
    else:
        _plain_churn(st)
    return st["table"], st["lens"], st["refs"], st["codes"], st["scales"]


# ----------------------------------------------------------------------------- plain forms

def _row_map(starts, n, most):
    """Row numbers [n, most] of the sequences' rows, and which of them are there."""
    if starts is None:
        return torch.arange(n, device="cuda")[:, None], torch.ones(n, 1, dtype=torch.bool, device="cuda")
    r = torch.arange(most, device="cuda")
    rows = (starts[1:] - starts[:-1]).long()
    there = r[None] < rows[:, None]
    return torch.where(there, starts[:-1].long()[:, None] + r[None], 0), there


def _plain_attend(st):
    c = st["case"]
    h, d, page = c["kv_heads"], c["dim"], c["page"]
    n, g = st["slots"].numel(), c["heads"] // h
    nb = _blocks(st["max_len"], page)
    slots = st["slots"].long()
    pages = st["table"][slots, :nb].long().clamp_min(0)
    lens = st["lens"][slots].long()
    k = (st["codes"][:, 0][pages].float() - ZERO) * st["scales"][:, 0][pages][..., None, None]
    k = k.transpose(1, 2).reshape(n, h, nb * page, d)
    v = (st["codes"][:, 1][pages].float() - ZERO) * st["scales"][:, 1][pages][..., None, None]
    v = v.transpose(1, 2).reshape(n, h, nb * page, d)
    index, there = _row_map(st["row_start"], n, st["max_rows"])
    most = index.shape[1]
    rows = there.sum(1)
    q = st["q"].float()[index].reshape(n, most, h, g, d).permute(0, 2, 3, 1, 4).reshape(n, h, g * most, d)
    s = torch.matmul(q, k.transpose(2, 3)).mul_(d ** -0.5).view(n, h, g, most, nb * page)
    p = (lens - rows)[:, None] + torch.arange(most, device="cuda")[None]
    j = torch.arange(nb * page, device="cuda")
    sees = (j[None, None] <= p[..., None]) & there[..., None]
    if c["window"]:
        sees &= (j[None, None] > p[..., None] - c["window"]) | (j < c["sinks"])[None, None]
    s.masked_fill_(~sees[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = s.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(n, h, g * most, nb * page), v).view(n, h, g, most, d) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).squeeze(-1)
    back = lambda x: x.permute(0, 3, 1, 2, *range(4, x.dim())).reshape(n, most, h * g, *x.shape[4:])[there]  # noqa: E731
    return back(o).to(st["q"].dtype), back(lse)


def _plain_append(st):
    """Every page that gets a token, whole: [n, touched pages, 2, heads, page, dim]."""
    c = st["case"]
    page = c["page"]
    slots = st["slots"].long()
    n, most = slots.numel(), st["max_rows"]
    lens = st["lens"][slots].long()
    starts = st["row_start"]
    rows = torch.ones_like(lens) if starts is None else (starts[1:] - starts[:-1]).long()
    row0 = torch.arange(n, device="cuda") if starts is None else starts[:-1].long()
    first = lens - rows                                              # position of the first new token
    nb = _blocks(most + page - 1, page)
    block = first[:, None] // page + torch.arange(nb, device="cuda")[None]
    touched = block * page < lens[:, None]
    pages = st["table"][slots].long().gather(1, torch.where(touched, block, 0))
    position = block[..., None] * page + torch.arange(page, device="cuda")
    new = (position >= first[:, None, None]) & (position < lens[:, None, None])
    at = torch.where(new, position - first[:, None, None] + row0[:, None, None], 0)
    kv = torch.stack([st["k"], st["v"]], 1).float()                  # [rows, 2, heads, dim]
    x = kv[at].permute(0, 1, 3, 4, 2, 5) * new[:, :, None, None, :, None]
    old_scale = torch.where((block * page < first[:, None])[..., None, None], st["scales"][pages], 0.0)
    scale = torch.maximum(old_scale, x.abs().amax((-1, -2)) / 127.0).clamp_min(FLOOR)
    old = st["codes"][pages].float() - ZERO
    kept = torch.round(old * (old_scale / scale)[..., None, None])
    kept = torch.where((position < first[:, None, None])[:, :, None, None, :, None], kept, old)
    fresh = torch.round(x / scale[..., None, None]).clamp_(-127, 127)
    codes = (torch.where(new[:, :, None, None, :, None], fresh, kept) + ZERO).to(torch.uint8)
    st["codes"][pages[touched]] = codes[touched]
    st["scales"][pages[touched]] = scale[touched]


def _plain_read(st):
    c = st["case"]
    page, slots = c["page"], st["slots"].long()
    most = _back(c)
    lens = st["lens"][slots].long()
    position = lens[:, None] - most + torch.arange(most, device="cuda")[None]
    there = position >= 0
    position = position.clamp_min(0)
    pages = st["table"][slots].long().gather(1, position // page)
    codes = st["codes"][pages, :, :, position % page].float() - ZERO    # [n, rows, 2, heads, dim]
    x = torch.where(there[..., None, None, None], codes * st["scales"][pages][..., None], 0.0).to(st["k"].dtype)
    x = x.reshape(-1, *x.shape[2:])
    return x[:, 0].contiguous(), x[:, 1].contiguous(), st["scales"]


def _lowest_free(refs, count):
    """The `count` lowest free pages, in order."""
    rank = torch.cumsum(refs == 0, 0)
    return torch.searchsorted(rank, torch.arange(1, count + 1, device="cuda"))


def _plain_fork(st):
    page, pages = st["case"]["page"], st["refs"].numel()
    ahead = (st["src"] != st["dst"]).nonzero().squeeze(1)
    src, dst = st["src"][ahead].long(), st["dst"][ahead].long()
    table, lens, refs = st["table"], st["lens"], st["refs"]
    block = torch.arange(table.shape[1], device="cuda")
    new, n = table[src], lens[src].long()
    full, tail = (n // page)[:, None] > block, ((n // page)[:, None] == block) & (n % page != 0)[:, None]
    live = lambda t, m: t[m & (t >= 0)].long()  # noqa: E731
    held = table[dst]
    refs += torch.bincount(live(new, full | tail), minlength=pages).to(refs.dtype)
    refs -= torch.bincount(live(held, _blocks_of(lens[dst], page)[:, None] > block), minlength=pages).to(refs.dtype)
    copied = tail & (new >= 0)
    old = new[copied].long()
    fresh = _lowest_free(refs, old.numel())
    refs -= torch.bincount(old, minlength=pages).to(refs.dtype)
    refs[fresh] = 1
    new = torch.where(full | copied, new, -1)
    new[copied] = fresh.to(new.dtype)
    st["codes"][fresh], st["scales"][fresh] = st["codes"][old], st["scales"][old]
    table[dst], lens[dst] = new, n.to(lens.dtype)


def _blocks_of(n, page):
    return (n.long() + page - 1) // page


def _plain_churn(st):
    slots, starts = st["groups"][st["turn"] % len(st["groups"])]
    st["turn"] += 1
    page, table, lens, refs = st["case"]["page"], st["table"], st["lens"], st["refs"]
    slots, pages = slots.long(), refs.numel()
    block = torch.arange(table.shape[1], device="cuda")
    # free
    held = table[slots][(_blocks_of(lens[slots], page)[:, None] > block) & (table[slots] >= 0)].long()
    refs -= torch.bincount(held, minlength=pages).to(refs.dtype)
    table[slots], lens[slots] = -1, 0
    # compact: the live pages behind the first `live` places go, in order, to the free ones among them
    used = refs > 0
    live = used.sum()
    number = torch.arange(pages, device="cuda")
    holes = (~used & (number < live)).nonzero().squeeze(1)
    movers = (used & (number >= live)).nonzero().squeeze(1)
    st["codes"][holes], st["scales"][holes] = st["codes"][movers], st["scales"][movers]
    refs[holes], refs[movers] = refs[movers], 0
    to = number.clone()
    to[movers] = holes
    table.copy_(torch.where(table >= 0, to[table.clamp_min(0).long()], -1))
    # reserve: the lowest free pages, sequence after sequence
    lens[slots] = (starts[1:] - starts[:-1])
    need = _blocks_of(lens[slots], page)[:, None] > block
    got = _lowest_free(refs, int(need.sum()))
    refs[got] = 1
    mine = table[slots]
    mine[need] = got.to(table.dtype)
    table[slots] = mine


# ----------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    if case["op"] not in ("attend", "append"):
        return None     # page numbers, counts and moved bytes: nothing is computed
    st = prepare(case, seed)
    lens, rows = _lens_rows(case)
    table, codes, scales = st["table"].cpu(), st["codes"], st["scales"].double()
    slots, page, h = st["slots"].tolist(), case["page"], case["kv_heads"]
    starts = [sum(rows[:i]) for i in range(len(rows))]

    def values(b, which, head, lo, hi):
        """[hi - lo, dim] in 64 bits, pages lo // page on"""
        ids = table[slots[b], lo // page:_blocks(hi, page)].long().cuda()
        x = (codes[ids, which, head].double() - 128.0) * scales[ids, which, head][:, None, None]
        return x.reshape(-1, case["dim"])[lo - lo // page * page:][:hi - lo]

    if case["op"] == "attend":
        if 8 * max(lens) * max(rows) * 3 > 60e9 or sum(r * n for r, n in zip(rows, lens)) * case["heads"] * case["dim"] * 4 > 8e13:
            return None
        out = torch.zeros(sum(rows), case["heads"], case["dim"], dtype=torch.float64, device="cuda")
        lse = torch.full((sum(rows), case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
        per = case["heads"] // h
        for b, (n, r) in enumerate(zip(lens, rows)):
            p = torch.arange(n - r, n, device="cuda")[:, None]
            j = torch.arange(n, device="cuda")[None]
            hidden = j > p
            if case["window"]:
                hidden |= (j <= p - case["window"]) & (j >= case["sinks"])
            for head in range(h):
                k, v = values(b, 0, head, 0, n), values(b, 1, head, 0, n)
                for query in range(head * per, (head + 1) * per):
                    x = st["q"][starts[b]:starts[b] + r, query].double()
                    s = (x @ k.T / math.sqrt(case["dim"])).masked_fill(hidden, -math.inf)
                    lse[starts[b]:starts[b] + r, query] = torch.logsumexp(s, 1)
                    out[starts[b]:starts[b] + r, query] = torch.softmax(s, 1) @ v
        return out, lse
    back, d = _back(case), case["dim"]
    values_out = [torch.zeros(back * len(lens), h, d, dtype=torch.float64, device="cuda") for _ in range(2)]
    for b, (n, r) in enumerate(zip(lens, rows)):
        first, lo = n - r, max(0, n - back)
        whole = lo // page * page
        for which, name in ((0, "k"), (1, "v")):
            new = st[name][starts[b]:starts[b] + r].double()
            x = torch.stack([values(b, which, head, whole, n) for head in range(h)], 1)
            x[max(first, whole) - whole:] = new[max(0, whole - first):]
            for at in range(first // page, _blocks(n, page)):
                t0, t1 = at * page, min(n, at * page + page)
                page_id = int(table[slots[b], at])
                s = new[max(0, t0 - first):t1 - first].abs().amax((0, 2)) / 127.0
                if t0 < first:
                    s = torch.maximum(s, scales[page_id, which])
                s = s.clamp_min(FLOOR)
                if t1 > whole:
                    y = x[t0 - whole:t1 - whole]
                    x[t0 - whole:t1 - whole] = (y / s[:, None]).round().clamp(-127, 127) * s[:, None]
                scales[page_id, which] = s
            values_out[which][b * back + back - (n - lo):(b + 1) * back] = x[lo - whole:]
    return values_out[0], values_out[1], scales
