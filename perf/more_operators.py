"""Timed cases of what a paged cache needs around its attention: new keys and values with the position rotation applied on the way,
a cache held in 4 bits with the attention that reads it, and attention over a few pages that a cheap score picks for each query.

All of them work on the pools, block tables and lengths of `wkv_paged` (see perf/operators.py for the attention over whole caches).
Shapes come from the library's named workloads: 32 x 128 heads, 32 query heads on 8 kv heads, 4 x 64 heads in fp32; prompts to 32768
tokens; 508 recent and 4 first tokens kept.

`run` computes an operator in its plain form, or calls the library where `own` is true.

Rows in 4 bits.  32 neighbouring channels share a scale s and a zero point z; a code n in 0..15 stands for s (n - z).  With lo = min(0,
least) and hi = max(0, largest): s is (hi - lo) / 15 rounded up to four significant bits (2^-17 .. 4096), z = rint(-lo / s), n =
rint(x / s) + z; everything in 32 bits, the quotients as products with 1 / s.  Such a value is a bfloat16 number.  A row of a page is
d / 2 bytes of codes, and behind the page's rows stand d / 32 pairs (scale byte, zero byte) per row.  Their order inside a row is the
library's (include/wkv.h).

Bounds of a page, per kv head: the largest and the least key of every channel in steps of page_scale = (largest magnitude) / 127,
rounded outwards.  A query's cheap score of a page is the bound on q.k that they give, with q in steps of 1 / 127 of its largest
channel, summed over the query heads of the kv head: a whole number, times page_scale.
"""
import math

import torch

own = False

NEG = float("-inf")
GROUP = 32                     # channels of a scale


# ---------------------------------------------------------------- cases

def _append(name, batch, hq, hk, d, dtype, page, lo, hi, new_lo, new_hi, rot, paired=False, bounds=False, shift=0, pad=0):
    return dict(name=name, op="append", batch=batch, hq=hq, hk=hk, d=d, dtype=dtype, page=page, lo=lo, hi=hi, new_lo=new_lo,
                new_hi=new_hi, rot=rot, paired=paired, bounds=bounds, shift=shift, pad=pad)


def _pack(name, batch, hq, hk, d, page, lo, hi, new_lo, new_hi, rot, paired=False, pad=0):
    return dict(name=name, op="pack", batch=batch, hq=hq, hk=hk, d=d, dtype="4bit", page=page, lo=lo, hi=hi, new_lo=new_lo,
                new_hi=new_hi, rot=rot, paired=paired, bounds=False, shift=0, pad=pad)


def _decode4(name, batch, hq, hk, d, page, lo, hi, window=0, sink=0, pad=0):
    return dict(name=name, op="decode4", batch=batch, hq=hq, hk=hk, d=d, dtype="4bit", page=page, lo=lo, hi=hi, window=window,
                sink=sink, pad=pad)


def _sparse(name, batch, hq, hk, d, dtype, page, lo, hi, n_select, recent, sink, pad=0):
    return dict(name=name, op="sparse", batch=batch, hq=hq, hk=hk, d=d, dtype=dtype, page=page, lo=lo, hi=hi, n_select=n_select,
                recent=recent, sink=sink, pad=pad)


def listed():
    return [
        # a decode step of the serving batch, grouped heads: one token a sequence, bounds kept for page selection; three padded rows
        _append("append_step", 19, 32, 8, 128, "bf16", 16, 1499, 16383, 1, 1, 128, bounds=True, pad=3),
        # ragged prompts into an empty cache, one kv head per query head, bounds kept
        _append("append_prompt", 4, 32, 32, 128, "bf16", 32, 0, 0, 2048, 8191, 128, bounds=True),
        # fp32 rows of the small workload, neighbouring channels rotated, half of the head; positions run ahead of the entries, as
        # they do in a cache that evicted some
        _append("append_f32", 3, 4, 4, 64, "f32", 16, 0, 131, 37, 256, 32, paired=True, shift=1024, pad=2),
        # one user's next token into a cache in 4 bits, its 611 entries spread out for a few drafted tokens' attention
        _pack("pack_single", 1, 32, 8, 128, 16, 610, 610, 1, 1, 128),
        # chunks of 17 to 61 tokens behind contexts of 1638 to 8192, 4 bits; the contexts spread out for the chunk's attention
        _pack("pack_chunk", 8, 32, 8, 128, 64, 1638, 8192, 17, 61, 128, pad=5),
        # one user's chat early on in 4 bits: latency is all
        _decode4("decode4_single", 1, 32, 8, 128, 16, 611, 611),
        # the serving batch in 4 bits: 16 ragged sequences of 8192 to 16384 tokens, one kv head per query head
        _decode4("decode4_serving", 16, 32, 32, 128, 32, 8192, 16384),
        # long grouped sequences in 4 bits, the whole of them seen; the batch is padded by three empty rows
        _decode4("decode4_long", 19, 32, 8, 128, 64, 12000, 32768, pad=3),
        # streaming caches in 4 bits: the newest 508 and the first 4 tokens of sequences to 32768
        _decode4("decode4_window", 32, 32, 8, 128, 16, 1500, 32768, window=508, sink=4),
        # one user's long document: 64 of 2048 pages read
        _sparse("sparse_single", 1, 32, 8, 128, "bf16", 16, 32761, 32761, 64, 2, 1),
        # the serving batch, 64 of up to 512 pages a kv head read
        _sparse("sparse_serving", 16, 32, 32, 128, "bf16", 32, 8192, 16384, 64, 4, 1),
        # the same batch in 4 bits with grouped heads, 37 pages of 64 read; two padded rows
        _sparse("sparse_4bit", 18, 32, 8, 128, "4bit", 64, 8192, 32768, 37, 2, 1, pad=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.499)))))


def draw(rng):
    """A case of the ranges above: any operator, head layout, type and page size; lengths from one token to 32768."""
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), work(c)["bytes"])
    while True:
        op = rng.choice(["append", "pack", "decode4", "decode4", "sparse", "sparse"])
        hq, hk, d = rng.choice([(32, 32, 128), (32, 8, 128), (32, 4, 128), (16, 8, 64), (4, 4, 64), (8, 1, 128)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        page = rng.choice([16, 32, 64])
        batch = _log_int(rng, 1, 40)
        pad = rng.choice([0, 0, 1, 3])
        if op in ("append", "pack"):
            new_hi = rng.choice([1, _log_int(rng, 1, 8192)])
            new_lo = rng.randint(1, new_hi)
            hi = rng.choice([0, _log_int(rng, 1, 16384)])
            rot, paired = rng.choice([d, d, 16 * rng.randint(1, d // 16)]), rng.random() < 0.4
            if op == "append":
                c = _append(None, batch, hq, hk, d, dtype, page, rng.randint(0, hi), hi, new_lo, new_hi, rot, paired,
                            rng.random() < 0.5, rng.choice([0, rng.randint(1, 4000)]), pad)
            else:
                c = _pack(None, batch, hq, hk, d, page, rng.randint(0, hi), hi, new_lo, new_hi, rot, paired, pad)
        else:
            hi = _log_int(rng, 1, 32768)
            lo = rng.randint(1, hi)
            if op == "decode4":
                window = rng.choice([0, 0, _log_int(rng, 1, 2048)])
                c = _decode4(None, batch, hq, hk, d, page, lo, hi, window, rng.choice([0, rng.randint(1, 70)]) if window else 0, pad)
            else:
                n_select = _log_int(rng, 1, 200)
                recent = rng.randint(1, min(4, n_select))
                c = _sparse(None, batch, hq, hk, d, rng.choice([dtype, "4bit"]), page, lo, hi, n_select, recent,
                            rng.randint(0, min(2, n_select - recent)), pad)
        del c["name"]
        lens, _ = _lengths(c)
        # a drawn case costs no more than the largest listed one of its operator, its pool included
        if work(c)["bytes"] > most[op] or sum(lens) * hk * d > 900_000_000:
            continue
        return c


# ---------------------------------------------------------------- sizes

def _spread(n, lo, hi):
    """n whole numbers in [lo, hi], the first of them hi: the ragged lengths of a batch, the same for every seed."""
    return [hi if i == 0 else lo + int((hi - lo) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _step(case):
    """Does the call bring one token per sequence, row b for sequence b?"""
    return case["op"] in ("decode4", "sparse") or case["new_hi"] == 1


def _lengths(case):
    """Entries of every sequence after the call's tokens have joined it, and the number of those tokens."""
    empty = min(case["pad"], case["batch"] - 1) if _step(case) else 0
    n = case["batch"] - empty
    lens = _spread(n, case["lo"], case["hi"])
    if case["op"] in ("decode4", "sparse"):
        return lens + [0] * empty, [0] * case["batch"]
    new = _spread(n, case["new_lo"], case["new_hi"])
    return [c + t for c, t in zip(lens, new)] + [0] * empty, new + [0] * empty


def _row(case):
    """Bytes of one token's keys, or values, of one kv head in the pool."""
    d = case["d"]
    return {"bf16": 2 * d, "f32": 4 * d, "4bit": d // 2 + d // 16}[case["dtype"]]


def work(case):
    lens, new = _lengths(case)
    hq, hk, d, page, row = case["hq"], case["hk"], case["d"], case["page"], _row(case)
    e = 4 if case["dtype"] == "f32" else 2
    pages = [-(-n // page) for n in lens]
    rows = sum(1 for n in lens if n)
    if case["op"] in ("append", "pack"):
        T = sum(new)
        # q in and out, k and v in, their rows out, the angles
        b = T * (2 * hq * d * e + 2 * hk * d * e + 2 * hk * row + case["rot"] * 4)
        flops = 3 * T * (hq + hk) * case["rot"]
        if case["op"] == "pack":
            b += sum(lens) * hk * (2 * row + 4 * d) + 2 * 4 * sum(pages)
            flops += T * hk * d * 6 + sum(lens) * hk * d * 4
        else:
            b += 4 * sum(pages)
            if case["bounds"]:
                for n, t in zip(lens, new):
                    old = n - t
                    touched = -(-n // page) - old // page if t else 0
                    # entries that are in the first page already are read, the touched pages' bounds written
                    b += hk * ((old % page if t else 0) * d * e + touched * (2 * d + 4))
                flops += 2 * T * hk * d
        return {"bytes": b, "flops": flops}
    if case["op"] == "decode4":
        w = case["window"]
        seen = sum(n if not w or n <= w else w + min(case["sink"], n - w) for n in lens)
        # every visible row once; a query in, its output and log-sum out
        return {"bytes": 2 * hk * row * seen + rows * hq * (4 * d + 4) + 4 * sum(pages), "flops": 4 * d * hq * seen}
    read = entries = 0
    for n, p in zip(lens, pages):
        take = min(case["n_select"], p)
        entries += take * page - (p * page - n) if n else 0
        read += p
    # bounds of every page, the chosen pages' rows, scores and choice out; a query in, its output and log-sum out
    return {"bytes": read * hk * (2 * d + 4 + 4) + rows * hk * case["n_select"] * 4 + 2 * hk * row * entries
            + rows * hq * (2 * d * e + 4) + 4 * sum(pages), "flops": 4 * d * hq * entries + 4 * d * hk * read}


# ---------------------------------------------------------------- rows in 4 bits

_ORDER = {}


def _order(kind, d, device):
    """Where the codes of a row lie: for each swizzle, the channel in the low and in the high half of every byte, and its inverse:
    byte and shift of every channel."""
    key = (kind, d, str(device))
    if key not in _ORDER:
        nb, groups = d // 2, d // GROUP
        at = torch.zeros(4, d, 2, dtype=torch.long)                  # [swizzle][channel] -> byte, shift
        for sw in range(4):
            for c in range(d):
                g, cc = divmod(c, GROUP)
                if kind == "k":
                    bit = (cc % 8 // 2) * 4 + (cc % 2) * 16
                    byte = ((g ^ (sw % groups)) * 16) + cc // 8 * 4 + bit // 8
                    at[sw, c, 0], at[sw, c, 1] = byte, bit % 8
                else:
                    byte = (cc // 4) * 2 * groups + 2 * g + (cc % 4) // 2
                    at[sw, c, 0], at[sw, c, 1] = (byte ^ 32 if d == 128 and sw % 2 else byte), cc % 2 * 4
        lo, hi = torch.zeros(4, nb, dtype=torch.long), torch.zeros(4, nb, dtype=torch.long)
        for sw in range(4):
            for c in range(d):
                (hi if at[sw, c, 1] else lo)[sw, at[sw, c, 0]] = c
        _ORDER[key] = lo.to(device), hi.to(device), at[..., 0].to(device), at[..., 1].to(device)
    return _ORDER[key]


def _swizzle(kind, d, i):
    """Swizzle of row i of a page."""
    return (i >> 1) & 3 if d == 128 else (i >> 2) & 1 if kind == "k" else torch.zeros_like(i)


def _to_codes(x):
    """x [..., d] in 32 bits -> codes [..., d], scale bytes and zero bytes [..., d / 32]."""
    x = x.unflatten(-1, (-1, GROUP))
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    r = (hi - lo) * torch.tensor(1.0 / 15.0, dtype=torch.float32, device=x.device)
    e = torch.frexp(r).exponent.clamp(-13, 14)
    step = torch.ldexp(torch.ones_like(r), e - 4)
    s = (torch.ceil(r / step) * step).clamp(2.0 ** -17, 4096.0)      # quotients and products with powers of two are exact
    inv = 1.0 / s
    z = torch.round(-lo * inv).clamp(0, 15)
    n = (torch.round(x * inv[..., None]) + z[..., None]).clamp(0, 15)
    sbyte = (s.half().view(torch.int16) >> 7).to(torch.uint8)
    return n.flatten(-2).to(torch.uint8), sbyte, z.to(torch.uint8)


def _scales(sbyte):
    return (sbyte.to(torch.int16) << 7).view(torch.float16).float()


def _put4(kind, pool, pages, i, x):
    """Rows x [N, hk, d] become row i[n] of page pages[n] of the 4-bit pool [pages, hk, bytes]."""
    d = x.shape[-1]
    page = pool.shape[-1] // (d // 2 + d // 16)
    lo, hi, _, _ = _order(kind, d, x.device)
    n, s, z = _to_codes(x)
    sw = _swizzle(kind, d, i)
    put = lambda idx: n.gather(-1, idx[sw][:, None].expand(-1, x.shape[1], -1))
    codes = put(lo) | put(hi) << 4
    b = torch.arange(d // 2, device=x.device)
    pool[pages[:, None], :, i[:, None] * (d // 2) + b] = codes.transpose(1, 2)
    sz = torch.stack([s, z], -1).flatten(-2)
    b = torch.arange(d // 16, device=x.device)
    pool[pages[:, None], :, page * (d // 2) + i[:, None] * (d // 16) + b] = sz.transpose(1, 2)


def _get4(kind, blocks, d, dtype=torch.float32):
    """Blocks [..., bytes] of pages -> values [..., page, d]."""
    page = blocks.shape[-1] // (d // 2 + d // 16)
    _, _, byte, shift = _order(kind, d, blocks.device)
    i = torch.arange(page, device=blocks.device)
    sw = _swizzle(kind, d, i)
    codes = blocks[..., :page * (d // 2)].unflatten(-1, (page, d // 2))
    n = codes.gather(-1, byte[sw].expand(*codes.shape[:-1], d)) >> shift[sw].to(torch.uint8) & 15
    sz = blocks[..., page * (d // 2):].unflatten(-1, (page, d // GROUP, 2))
    s, z = _scales(sz[..., 0]).to(dtype), sz[..., 1].to(dtype)
    return ((n.to(dtype).unflatten(-1, (-1, GROUP)) - z[..., None]) * s[..., None]).flatten(-2)


def _values(case, kind, pool, pages):
    """Pages of the layer's pool in 32 bits: [..., hk, page, d]."""
    x = pool[0][pages]
    return _get4(kind, x, case["d"]) if case["dtype"] == "4bit" else x.float()


# ---------------------------------------------------------------- bounds of pages and the cheap score

def _bounds(k, valid):
    """Bounds of keys k [..., page, d] over the valid rows [..., page]: codes int8 [..., 2, d] (largest, least) and scales [...]."""
    hi = k.masked_fill(~valid[..., None], NEG).amax(-2)
    lo = k.masked_fill(~valid[..., None], -NEG).amin(-2)
    most = torch.maximum(hi.abs(), lo.abs()).amax(-1)
    scale = most * torch.tensor(1.0 / 127.0, dtype=torch.float32, device=k.device)
    inv = torch.where(scale >= 2.0 ** -100, 1.0 / scale, 0.0)[..., None]
    up, down = torch.ceil(hi * inv).clamp(max=127.0), torch.floor(lo * inv).clamp(min=-127.0)
    return torch.stack([up, down], -2).to(torch.int8), scale


def _query_codes(q, hk):
    """q [B, hq, d] -> [B, hk, 2, d]: the query heads' positive and negative parts summed, in steps of 1 / 127 of the largest."""
    q = q.float().unflatten(1, (hk, -1))
    up, down = q[:, :, 0].clamp(min=0.0), q[:, :, 0].clamp(max=0.0)
    for g in range(1, q.shape[2]):
        up, down = up + q[:, :, g].clamp(min=0.0), down + q[:, :, g].clamp(max=0.0)
    x = torch.stack([up, down], 2)
    step = x.abs().amax((-1, -2)) * torch.tensor(1.0 / 127.0, dtype=torch.float32, device=q.device)
    inv = torch.where(step >= 2.0 ** -100, 1.0 / step, 0.0)
    return torch.round(x * inv[..., None, None]).clamp(-127.0, 127.0)


# ---------------------------------------------------------------- inputs

def _angles(rows, dim, device):
    """cos | sin of the positions' angles [rows, dim]."""
    f = 10000.0 ** (-torch.arange(dim // 2, dtype=torch.float64, device=device) * 2.0 / dim)
    a = torch.arange(rows, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([a.cos(), a.sin()], -1).float()


def _fill(pool, kind, d, four, loud, g):
    """Random rows; keys of a page share a direction, as neighbouring tokens' do, and have a few loud channels."""
    n, hk = pool.shape[1], pool.shape[2]
    page = pool.shape[3] // (d // 2 + d // 16) if four else pool.shape[3]
    some = max(1, 2 ** 25 // (hk * page * d))
    i = torch.arange(page, device=pool.device)
    for a in range(0, n, some):
        m = min(some, n - a)
        x = torch.randn(m, hk, page, d, generator=g, device=pool.device)
        if kind == "k":
            x = (x + 0.7 * torch.randn(m, hk, 1, d, generator=g, device=pool.device)) * loud
        if four:
            which = torch.arange(a, a + m, device=pool.device).repeat_interleave(page)
            _put4(kind, pool[0], which, i.repeat(m), x.transpose(1, 2).flatten(0, 1))
        else:
            pool[0, a:a + m] = x


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    lens, new = _lengths(case)
    B, hq, hk, d, page = case["batch"], case["hq"], case["hk"], case["d"], case["page"]
    four = case["dtype"] == "4bit"
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    used = [-(-n // page) for n in lens]
    width = max(used)
    n_pages = sum(used) + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    loud = torch.ones(d, device=dev)
    loud[torch.randperm(d, generator=g, device=dev)[:4]] = 3.0
    if four:
        pools = [torch.zeros(1, n_pages, hk, page * _row(case), device=dev, dtype=torch.uint8) for _ in "kv"]
    else:
        pools = [torch.zeros(1, n_pages, hk, page, d, device=dev, dtype=dt) for _ in "kv"]
    if case["hi"]:
        _fill(pools[0], "k", d, four, loud, g)
        _fill(pools[1], "v", d, four, loud, g)
    s = dict(case=dict(case), width=width, k_pool=pools[0], v_pool=pools[1], table=_table(order, 0, used, width, dev),
             seq_lens=torch.tensor(lens, dtype=torch.int32, device=dev))
    if case["op"] in ("append", "pack"):
        T = B if _step(case) else sum(new) + case["pad"]
        qkv = torch.randn(T, hq + 2 * hk, d, generator=g, device=dev, dtype=dt)      # a projection's output, side by side
        qkv[:, hq:hq + hk].mul_(loud.to(dt))
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        s["q_out"] = torch.zeros(T, hq, d, device=dev, dtype=dt)
        s["rope"] = _angles(max(lens) + case["shift"], case["rot"], dev)
        s["q_start"], s["positions"] = None, None
        row, entry = [], []
        for b, (n, t) in enumerate(zip(lens, new)):
            row += [b] * t
            entry += range(n - t, n)
        s["seq"], s["entry"] = torch.tensor(row, device=dev), torch.tensor(entry, device=dev)
        if not _step(case):
            starts = [0]
            for t in new:
                starts.append(starts[-1] + t)
            s["q_start"] = torch.tensor(starts, dtype=torch.int32, device=dev)
            s["at"] = torch.arange(sum(new), device=dev)
        else:
            s["at"] = s["seq"]
        if case["shift"]:
            s["positions"] = torch.zeros(T, dtype=torch.int32, device=dev)
            s["positions"][s["at"]] = (s["entry"] + case["shift"]).int()
        if case["bounds"]:
            s["page_bounds"] = torch.zeros(1, n_pages, hk, 2, d, dtype=torch.int8, device=dev)
            s["page_scale"] = torch.zeros(1, n_pages, hk, device=dev)
            s["first_touched"] = torch.tensor([(n - t) // page for n, t in zip(lens, new)], device=dev)
        if case["op"] == "pack":
            # bf16 pages for the values, in another order
            s["wide_table"] = _table(torch.randperm(n_pages, generator=g, device=dev).to(torch.int32), 0, used, width, dev)
            s["wide_k"] = torch.zeros(1, n_pages, hk, page, d, device=dev, dtype=dt)
            s["wide_v"] = torch.zeros(1, n_pages, hk, page, d, device=dev, dtype=dt)
    else:
        s["q"] = torch.randn(B, hq, d, generator=g, device=dev, dtype=dt)
        s["out"] = torch.zeros(B, hq, d, device=dev, dtype=dt)
        s["lse"] = torch.zeros(B, hq, device=dev)
    if case["op"] == "sparse":
        bounds = torch.zeros(1, n_pages, hk, 2, d, dtype=torch.int8, device=dev)
        scale = torch.zeros(1, n_pages, hk, device=dev)
        fill = torch.zeros(n_pages, dtype=torch.long, device=dev)
        col = torch.arange(width, device=dev)
        there = col < torch.tensor(used, device=dev)[:, None]
        n = (s["seq_lens"].long()[:, None] - col * page).clamp(0, page)
        fill[s["table"][there].long()] = n[there]
        some = max(1, 2 ** 25 // (hk * page * d))
        for a in range(0, n_pages, some):
            k = _values(case, "k", s["k_pool"], torch.arange(a, min(a + some, n_pages), device=dev))
            ok = torch.arange(page, device=dev) < fill[a:a + some, None].clamp(min=1)
            bounds[0, a:a + some], scale[0, a:a + some] = _bounds(k, ok[:, None].expand(-1, hk, -1))
        s["page_bounds"], s["page_scale"] = bounds, scale
        s["page_scores"] = torch.zeros(B, hk, width, device=dev)
        s["pages"] = torch.zeros(B, hk, case["n_select"], dtype=torch.int32, device=dev)
    if own:
        from paper_2503_01330_b200 import binding
        kind = {"bf16": binding.WKV_BF16, "f32": binding.WKV_F32, "4bit": binding.WKV_KV4}[case["dtype"]]
        s["cache"] = binding.PagedCache(1, n_pages, page, hq, hk, d, max_batch=B, max_pages=width, dtype=kind, device=dev,
                                        k_pool=s["k_pool"], v_pool=s["v_pool"])
        if case["op"] == "pack":
            s["wide"] = binding.PagedCache(1, n_pages, page, hq, hk, d, max_batch=B, max_pages=width, dtype=binding.WKV_BF16,
                                           device=dev, k_pool=s["wide_k"], v_pool=s["wide_v"])
    return s


def _table(order, first, counts, width, dev):
    """Block table [sequences, width]: consecutive runs of the shuffled pages; 0 behind a sequence's last page."""
    n = torch.tensor(counts, device=dev)
    at = torch.cumsum(n, 0) - n + first
    col = torch.arange(width, device=dev)
    idx = (at[:, None] + col).clamp_(max=order.numel() - 1)
    return torch.where(col < n[:, None], order[idx], 0).to(torch.int32).contiguous()


# ---------------------------------------------------------------- one pass

def run(s):
    return (_RUN_OWN if own else _RUN_PLAIN)[s["case"]["op"]](s, s["case"])


def _append_out(s, c):
    out = {"q_out": s["q_out"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    if c["bounds"]:
        out["page_bounds"], out["page_scale"] = s["page_bounds"], s["page_scale"]
    return out


def _own_append(s, c):
    s["cache"].wkv_paged_append(0, s["q"], s["k"], s["v"], s["table"], s["seq_lens"], q_start=s["q_start"], rope=s["rope"],
                                paired=c["paired"], positions=s["positions"], q_out=s["q_out"],
                                page_bounds=s.get("page_bounds"), page_scale=s.get("page_scale"))
    return _append_out(s, c)


def _own_pack(s, c):
    _own_append(s, c)
    s["cache"].wkv_paged_expand(0, s["table"], s["seq_lens"], s["wide"], 0, s["wide_table"])
    return {"q_out": s["q_out"], "k": s["wide_k"], "v": s["wide_v"]}


def _own_decode4(s, c):
    s["cache"].wkv_paged_decode(0, s["q"], None, None, s["table"], s["seq_lens"], s["out"], window=c["window"], sink=c["sink"],
                                lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_sparse(s, c):
    s["cache"].wkv_paged_select(0, s["q"], s["table"], s["seq_lens"], s["page_bounds"], s["page_scale"], s["page_scores"],
                                s["pages"], recent=c["recent"], sink=c["sink"])
    s["cache"].wkv_paged_decode_pages(0, s["q"], s["table"], s["seq_lens"], s["pages"], s["out"], lse=s["lse"])
    return {"page_scores": s["page_scores"], "pages": s["pages"], "out": s["out"], "lse": s["lse"]}


_RUN_OWN = {"append": _own_append, "pack": _own_pack, "decode4": _own_decode4, "sparse": _own_sparse}


def _rotate(x, angles, paired):
    """x [N, heads, d], angles [N, dim]: the first dim channels turned, in x's type."""
    dim = angles.shape[-1]
    c, w = angles[:, None, :dim // 2], angles[:, None, dim // 2:]
    a, b = (x[..., 0:dim:2], x[..., 1:dim:2]) if paired else (x[..., :dim // 2], x[..., dim // 2:dim])
    y0, y1 = a * c - b * w, b * c + a * w
    y = torch.stack([y0, y1], -1).flatten(-2) if paired else torch.cat([y0, y1], -1)
    return torch.cat([y, x[..., dim:]], -1)


def _plain_append(s, c):
    at, page = s["at"], c["page"]
    pos = s["entry"] if s["positions"] is None else s["positions"][at].long()
    angles = s["rope"][pos]
    s["q_out"][at] = _rotate(s["q"][at].float(), angles, c["paired"]).to(s["q_out"].dtype)
    k, v = _rotate(s["k"][at].float(), angles, c["paired"]), s["v"][at].float()
    pages, i = s["table"][s["seq"], s["entry"] // page].long(), s["entry"] % page
    if c["dtype"] == "4bit":
        _put4("k", s["k_pool"][0], pages, i, k)
        _put4("v", s["v_pool"][0], pages, i, v)
        return None
    s["k_pool"][0][pages, :, i] = k.to(s["k_pool"].dtype)
    s["v_pool"][0][pages, :, i] = v.to(s["v_pool"].dtype)
    if c["bounds"]:
        col = torch.arange(s["width"], device=at.device)
        n = s["seq_lens"].long()[:, None] - col * page
        b, j = ((n > 0) & (col >= s["first_touched"][:, None])).nonzero(as_tuple=True)
        which = s["table"][b, j].long()
        ok = torch.arange(page, device=at.device) < n[b, j][:, None]
        s["page_bounds"][0, which], s["page_scale"][0, which] = _bounds(s["k_pool"][0][which].float(),
                                                                        ok[:, None].expand(-1, c["hk"], -1))
    return _append_out(s, c)


def _plain_pack(s, c):
    _plain_append(s, c)
    page = c["page"]
    i = torch.arange(s["width"] * page, device=s["q"].device)
    b, e = (i < s["seq_lens"][:, None]).nonzero(as_tuple=True)
    col = torch.arange(s["width"], device=i.device)
    bp, j = (col * page < s["seq_lens"][:, None]).nonzero(as_tuple=True)
    place = torch.zeros(s["table"].shape, dtype=torch.long, device=i.device)
    place[bp, j] = torch.arange(bp.numel(), device=i.device)
    for kind, pool, wide in (("k", s["k_pool"], s["wide_k"]), ("v", s["v_pool"], s["wide_v"])):
        x = _values(c, kind, pool, s["table"][bp, j].long()).to(wide.dtype)
        wide[0][s["wide_table"][b, e // page].long(), :, e % page] = x[place[b, e // page], :, e % page]
    return {"q_out": s["q_out"], "k": s["wide_k"], "v": s["wide_v"]}


def _softmax_sum(s, c, K, V, see):
    """One query row per sequence against keys K [B, hk, L, d] where see [B, 1 or hk, L]."""
    B, hq, d = s["q"].shape
    G = hq // c["hk"]
    q = s["q"].float().view(B, c["hk"], G, d)
    x = (q @ K.transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).masked_fill_(~see[:, :, None], NEG)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == NEG, 0.0, m)
    x.sub_(m).exp_()
    z = x.sum(-1, keepdim=True)
    x.mul_(torch.where(z > 0, 1.0 / z, 0.0))
    s["out"].copy_((x @ V).view(B, hq, d))
    s["lse"].copy_((m + z.log()).view(B, hq))


def _plain_decode4(s, c):
    lens = s["seq_lens"].long()
    K, V = (_values(c, kind, pool, s["table"].long()).transpose(1, 2).flatten(2, 3) for kind, pool in (("k", s["k_pool"]), ("v", s["v_pool"])))
    j = torch.arange(K.shape[2], device=lens.device)
    see = j < lens[:, None]
    if c["window"]:
        see &= (j >= lens[:, None] - c["window"]) | (j < c["sink"])
    _softmax_sum(s, c, K, V, see[:, None])
    return {"out": s["out"], "lse": s["lse"]}


def _plain_sparse(s, c):
    lens, page, n_select = s["seq_lens"].long(), c["page"], c["n_select"]
    dev = lens.device
    n = (lens + page - 1) // page
    col = torch.arange(s["width"], device=dev)
    code = _query_codes(s["q"], c["hk"])
    bounds = s["page_bounds"][0][s["table"].long()].float()              # [B, width, hk, 2, d]
    whole = (bounds * code[:, None]).sum((-1, -2))                       # whole numbers below 2^24
    score = (whole * s["page_scale"][0][s["table"].long()]).transpose(1, 2)
    live = (col < n[:, None])[:, None].expand_as(score)
    s["page_scores"].copy_(torch.where(live, score, s["page_scores"]))
    # the first and the newest pages are always taken, then the best scores, of equal ones the lowest page
    forced = ((col < c["sink"]) | (col >= n[:, None] - c["recent"]))[:, None]
    rank = score.masked_fill(forced, -NEG).masked_fill(~live, NEG)
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :n_select]
    if best.shape[-1] < n_select:
        best = torch.nn.functional.pad(best, (0, n_select - best.shape[-1]))
    taken = torch.arange(n_select, device=dev) < n[:, None, None]
    best = torch.sort(torch.where(taken, best, s["width"]), dim=-1).values
    s["pages"].copy_(torch.where(taken, best, -1))
    b = torch.arange(lens.numel(), device=dev)[:, None, None]
    h = torch.arange(c["hk"], device=dev)[:, None]
    which = s["table"][b, torch.where(taken, best, 0)].long()
    i = best[..., None] * page + torch.arange(page, device=dev)
    see = (taken[..., None] & (i < lens[:, None, None, None])).flatten(2)
    rows = []
    for kind, pool in (("k", s["k_pool"]), ("v", s["v_pool"])):
        x = pool[0][which, h]
        rows.append((_get4(kind, x, c["d"]) if c["dtype"] == "4bit" else x.float()).flatten(2, 3))
    _softmax_sum(s, c, rows[0], rows[1], see)
    return {"page_scores": s["page_scores"], "pages": s["pages"], "out": s["out"], "lse": s["lse"]}


_RUN_PLAIN = {"append": _plain_append, "pack": _plain_pack, "decode4": _plain_decode4, "sparse": _plain_sparse}


# ---------------------------------------------------------------- the definition in 64 bits

def _turned(x, s, rows, positions, paired):
    """Rows of x in 64 bits, each channel's pair by a product of complex numbers."""
    dim = s["rope"].shape[1]
    a = s["rope"][positions].double()
    turn = torch.complex(a[:, :dim // 2], a[:, dim // 2:])[:, None]
    x = x[rows].double()
    y = x.clone()
    if paired:
        z = torch.view_as_complex(x[..., :dim].unflatten(-1, (-1, 2)).contiguous()) * turn
        y[..., :dim] = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(x[..., :dim // 2], x[..., dim // 2:dim]) * turn
        y[..., :dim // 2], y[..., dim // 2:dim] = z.real, z.imag
    return y


def exact(case, seed):
    """One sequence and one kv head at a time, in 64 bits.  None for copies, whole numbers, and values that stand in 4 bits."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f8 = torch.float64
    lens, new = _lengths(case)
    hk, G, d, page = case["hk"], case["hq"] // case["hk"], case["d"], case["page"]
    if case["op"] in ("append", "pack"):
        out = {}
        pos = s["entry"] + case["shift"]
        out["q_out"] = s["q_out"].to(f8)
        out["q_out"][s["at"]] = _turned(s["q"], s, s["at"], pos, case["paired"])
        if case["op"] == "pack":
            out["k"] = out["v"] = None
            return out
        k = _turned(s["k"], s, s["at"], pos, case["paired"])
        out["k_pool"] = s["k_pool"].to(f8)
        stored = s["k_pool"].to(f8)
        for b, (n, t) in enumerate(zip(lens, new)):
            mine = (s["seq"] == b).nonzero()[:, 0]
            for p in range((n - t) // page, -(-n // page)) if t else ():
                of = mine[s["entry"][mine] // page == p]
                at = int(s["table"][b, p])
                i = s["entry"][of] % page
                out["k_pool"][0, at, :, i] = k[of].transpose(0, 1)
                stored[0, at, :, i] = k[of].to(s["k_pool"].dtype).to(f8).transpose(0, 1)
                if case["bounds"]:
                    # as the rows are stored
                    s["page_scale"][0, at] = (stored[0, at, :, :n - p * page].abs().amax((-1, -2)) / 127.0).float()
        out["v_pool"] = None
        if case["bounds"]:
            out["page_bounds"], out["page_scale"] = None, s["page_scale"].to(f8)
        return out
    res, lse = s["out"].to(f8), s["lse"].to(f8)
    score = None
    if case["op"] == "sparse":
        score, code = s["page_scores"].to(f8), _query_codes(s["q"], hk).to(f8)
    for b, n in enumerate(lens):
        if n == 0:
            res[b], lse[b] = 0.0, NEG
            continue
        pages = s["table"][b, :-(-n // page)].long()
        for h in range(hk):
            idx = torch.arange(n, device="cuda")
            which = pages
            if case["op"] == "sparse":
                sc = torch.einsum("pwd,wd->p", s["page_bounds"][0, pages, h].to(f8), code[b, h]) * s["page_scale"][0, pages, h].to(f8)
                score[b, h, :pages.numel()] = sc
                order = sc.float().clone()
                order[:case["sink"]] = math.inf
                order[max(0, pages.numel() - case["recent"]):] = math.inf
                take = torch.argsort(order, descending=True, stable=True)[:case["n_select"]].sort().values
                idx = (take[:, None] * page + torch.arange(page, device="cuda")).flatten()
                which = pages[take]
            elif case["window"]:
                idx = idx[(idx >= n - case["window"]) | (idx < case["sink"])]
                keep = torch.unique(idx // page)
                which = pages[keep]
                idx = (keep[:, None] * page + torch.arange(page, device="cuda")).flatten()
            else:
                idx = torch.arange(pages.numel() * page, device="cuda")
            hidden = idx >= n
            if case["op"] == "decode4" and case["window"]:
                hidden |= (idx < n - case["window"]) & (idx >= case["sink"])
            if case["dtype"] == "4bit":
                keys, vals = (_get4(kind, pool[0, which, h], d, f8).flatten(0, 1) for kind, pool in (("k", s["k_pool"]), ("v", s["v_pool"])))
            else:
                keys, vals = s["k_pool"][0, which, h].flatten(0, 1).to(f8), s["v_pool"][0, which, h].flatten(0, 1).to(f8)
            logit = s["q"][b, h * G:h * G + G].to(f8) @ keys.T / d ** 0.5
            logit[:, hidden] = NEG
            norm = torch.logsumexp(logit, -1)
            res[b, h * G:h * G + G] = torch.exp(logit - norm[:, None]) @ vals
            lse[b, h * G:h * G + G] = norm
    if case["op"] == "sparse":
        return {"page_scores": score, "pages": None, "out": res, "lse": lse}
    return {"out": res, "lse": lse}
