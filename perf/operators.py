"""Timed cases of the paged-cache operators: decode attention, prompt attention and eviction over a cache kept in pages.

These are the uncompressed and the evicting caches that a compressed one is weighed against: every token kept (decode and prompt
attention without a window), first and newest tokens kept (window + sink), and heavy hitters kept (accumulated attention weight,
then eviction).  All three read one cache: pages of `page` entries, pool [layers, pages, kv heads, page, head dim], one block
table row per sequence.  Shapes come from the library's named workloads (32 x 128 heads, 32 query heads on 8 kv heads, 4 x 64
heads in fp32; prompts to 32768 tokens; 508 / 124 recent and 4 first tokens kept).

`run` computes an operator in its plain form, or calls the library where `own` is true.
"""
import math

import torch

own = False

NEG = float("-inf")


# ---------------------------------------------------------------- cases

def _decode(name, batch, hq, hk, d, dtype, page, lo, hi, window=0, sink=0, scores=False, pad=0):
    return dict(name=name, op="decode", batch=batch, hq=hq, hk=hk, d=d, dtype=dtype, page=page, lo=lo, hi=hi, window=window,
                sink=sink, scores=scores, pad=pad)


def _prefill(name, batch, hq, hk, d, dtype, page, ctx_lo, ctx_hi, new_lo, new_hi, window=0, sink=0, scores=False, pad=0):
    return dict(name=name, op="prefill", batch=batch, hq=hq, hk=hk, d=d, dtype=dtype, page=page, lo=ctx_lo, hi=ctx_hi,
                new_lo=new_lo, new_hi=new_hi, window=window, sink=sink, scores=scores, pad=pad)


def _evict(name, batch, hq, hk, d, dtype, page, lo, hi, budget, recent, sink):
    return dict(name=name, op="evict", batch=batch, hq=hq, hk=hk, d=d, dtype=dtype, page=page, lo=lo, hi=hi, budget=budget,
                recent=recent, sink=sink)


def listed():
    return [
        # one user's chat early on: a single sequence of some 600 tokens, grouped heads; latency is all
        _decode("decode_single", 1, 32, 8, 128, "bf16", 16, 611, 611),
        # the serving batch with its whole prompts kept: 16 ragged sequences of 8192 to 16384 tokens, one kv head per query head
        _decode("decode_serving", 16, 32, 32, 128, "bf16", 32, 8192, 16384),
        # streaming caches: the newest 508 and the first 4 tokens of sequences to 32768; the batch is padded by three empty rows
        _decode("decode_window", 32, 32, 8, 128, "bf16", 16, 1500, 32768, window=508, sink=4, pad=3),
        # a heavy-hitter cache between two evictions: attention weights are added up
        _decode("decode_scores", 8, 32, 32, 128, "bf16", 64, 4096, 4351, scores=True),
        # fp32 rows, 4 heads x 64, short ragged sequences, weights added up
        _decode("decode_f32", 4, 4, 4, 64, "f32", 16, 37, 512, scores=True),
        # fp32 prompt of the small workload, weights added up
        _prefill("prefill_f32", 2, 4, 4, 64, "f32", 16, 0, 0, 131, 256, scores=True),
        # chunks of 17 to 61 tokens behind contexts of 1638 to 8192, grouped heads; a few rows behind the last sequence
        _prefill("prefill_chunk", 8, 32, 8, 128, "bf16", 64, 1638, 8192, 17, 61, pad=5),
        # ragged prompts under a window of 508 with 4 sinks, grouped heads
        _prefill("prefill_window", 4, 32, 8, 128, "bf16", 16, 0, 0, 2048, 8191, window=508, sink=4),
        # one whole prompt of 8192 tokens, one kv head per query head
        _prefill("prefill_prompt", 1, 32, 32, 128, "bf16", 32, 0, 0, 8192, 8192),
        # prompts whose attention weights decide what is kept
        _prefill("prefill_scores", 2, 32, 32, 128, "bf16", 64, 0, 0, 1638, 4096, scores=True),
        # one sequence grown by its recent window past a cache of 1024
        _evict("evict_step", 1, 32, 32, 128, "bf16", 16, 1148, 1148, 1024, 508, 4),
        # prompts of 8192 to 32768 cut to 3277 entries a head, grouped heads
        _evict("evict_prompt", 16, 32, 8, 128, "bf16", 64, 8192, 32768, 3277, 128, 4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.499)))))


def draw(rng):
    """A case of the ranges above: any operator, head layout, type and page size; lengths from one token to 32768."""
    most = {}
    for c in listed():
        w, m = work(c), most.setdefault(c["op"], [0, 0])
        m[0], m[1] = max(m[0], w["bytes"]), max(m[1], w["flops"])
    while True:
        op = rng.choice(["decode", "prefill", "evict"])
        hq, hk, d = rng.choice([(32, 32, 128), (32, 8, 128), (32, 4, 128), (16, 8, 64), (4, 4, 64), (8, 1, 128)])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        page = rng.choice([16, 32, 64])
        batch = _log_int(rng, 1, 40)
        if op == "decode":
            hi = _log_int(rng, 1, 32768)
            lo = rng.randint(1, hi)
            window = rng.choice([0, _log_int(rng, 1, 2048)])
            c = _decode(None, batch, hq, hk, d, dtype, page, lo, hi, window, rng.choice([0, rng.randint(1, 70)]) if window else 0,
                        rng.random() < 0.4, rng.choice([0, 0, 1]))
        elif op == "prefill":
            new_hi = _log_int(rng, 1, 8192 if dtype == "bf16" else 700)
            new_lo = rng.randint(1, new_hi)
            ctx_hi = rng.choice([0, _log_int(rng, 1, 16384)])
            window = rng.choice([0, _log_int(rng, 1, 2048)])
            c = _prefill(None, min(batch, 12), hq, hk, d, dtype, page, rng.randint(0, ctx_hi), ctx_hi, new_lo, new_hi, window,
                         rng.choice([0, rng.randint(1, 70)]) if window else 0, rng.random() < 0.4, rng.choice([0, 3]))
        else:
            hi = _log_int(rng, 2, 32768)
            budget = rng.randint(1, hi)
            sink = rng.randint(0, min(8, budget - 1))
            c = _evict(None, batch, hq, hk, d, dtype, page, rng.randint(1, hi), hi, budget, rng.randint(1, budget - sink), sink)
        del c["name"]
        w = work(c)
        # a drawn case costs no more than the largest listed one of its operator, its plain form and its pool included
        if w["bytes"] > most[op][0] or w["flops"] > 0.5 * most[op][1] and op == "prefill" and dtype == "f32":
            continue
        lens, new = _lengths(c)
        if w["flops"] > most[op][1] or sum(lens) * hk * d > 600_000_000 or max(lens) * max(new) * len(lens) * hq > 2_400_000_000:
            continue
        return c


# ---------------------------------------------------------------- sizes

def _spread(n, lo, hi):
    """n whole numbers in [lo, hi], the first of them hi: the ragged lengths of a batch, the same for every seed."""
    return [hi if i == 0 else lo + int((hi - lo) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _lengths(case):
    """Entries in the cache of every sequence after the call's tokens have joined it, and the number of those tokens."""
    n = case["batch"] - (min(case.get("pad", 0), case["batch"] - 1) if case["op"] == "decode" else 0)
    lens = _spread(n, case["lo"], case["hi"])
    if case["op"] == "decode":
        empty = case["batch"] - n
        return lens + [0] * empty, [1] * n + [0] * empty
    if case["op"] == "prefill":
        new = _spread(n, case["new_lo"], case["new_hi"])
        return [c + t for c, t in zip(lens, new)], new
    return lens, [0] * n


def _visible(pos, window, sink):
    """Entries that the token at `pos` attends to."""
    if not window or pos < window:
        return pos + 1
    return window + min(sink, pos + 1 - window)


def work(case):
    lens, new = _lengths(case)
    e, hq, hk, d = (2 if case["dtype"] == "bf16" else 4), case["hq"], case["hk"], case["d"]
    row = hk * d * e                                   # one token's keys, or its values, over the kv heads
    table = sum(-(-n // case["page"]) for n in lens) * 4
    if case["op"] == "evict":
        kept = sum(min(n, case["budget"]) for n in lens)
        # weights read and the kept ones written, kept rows read and written, their indexes written
        return {"bytes": sum(lens) * hk * 4 + kept * (4 * row + 8 * hk) + table, "flops": 0}
    tokens, pairs, seen = sum(new), 0, 0
    for n, t in zip(lens, new):
        w, s = case["window"], case["sink"]
        if not w:
            pairs += t * (n - t) + t * (t + 1) // 2
            seen += n - t
        else:
            pairs += sum(_visible(p, w, s) for p in range(n - t, n))
            if t:                                      # cached entries that any of the new tokens sees
                first = max(0, n - t + 1 - w)
                seen += max(0, n - t - first) + min(s, first)
    scores = (seen + tokens) * hk * 8 if case["scores"] else 0
    # cached keys and values once; the new ones in and out; queries in, outputs and their log-sums out
    return {"bytes": 2 * row * seen + 4 * row * tokens + tokens * hq * (2 * d * e + 4) + scores + table, "flops": 4 * d * hq * pairs}


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    lens, new = _lengths(case)
    B, hq, hk, d, page = case["batch"], case["hq"], case["hk"], case["d"], case["page"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    used = [-(-n // page) for n in lens]
    width = max(used)
    extra = [-(-min(n, case["budget"]) // page) for n in lens] if case["op"] == "evict" else []
    n_pages = sum(used) + sum(extra) + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    # keys with a few loud channels, so that attention is skewed
    loud = torch.ones(d, device=dev)
    loud[torch.randperm(d, generator=g, device=dev)[:4]] = 3.0
    k_pool = torch.randn(1, n_pages, hk, page, d, generator=g, device=dev, dtype=dt).mul_(loud.to(dt))
    v_pool = torch.randn(1, n_pages, hk, page, d, generator=g, device=dev, dtype=dt)
    s = dict(case=dict(case), width=width, k_pool=k_pool, v_pool=v_pool,
             table=_table(order, 0, used, width, dev), seq_lens=torch.tensor(lens, dtype=torch.int32, device=dev))
    if case["op"] == "evict":
        # weights added up over the tokens since: an entry's falls with its index, scattered over decades; some were never seen
        stride = width * page
        x = torch.randn(B, hk, stride, generator=g, device=dev).mul_(1.5).exp_()
        x /= torch.arange(1, stride + 1, device=dev).sqrt()
        s["scores"] = x.masked_fill_(torch.rand(B, hk, stride, generator=g, device=dev) < 0.05, 0.0)
        s["dst_table"] = _table(order, sum(used), extra, max(extra), dev)
        s["new_lens"] = torch.zeros(B, dtype=torch.int32, device=dev)
        s["scores_out"] = torch.zeros(B, hk, case["budget"], device=dev)
        s["kept"] = torch.full((B, hk, case["budget"]), -1, dtype=torch.int32, device=dev)
    else:
        # a projection's output, q | k | v side by side: the operators take its columns as they lie
        T = (sum(new) + case["pad"]) if case["op"] == "prefill" else B
        qkv = torch.randn(T, (hq + 2 * hk), d, generator=g, device=dev, dtype=dt)
        qkv[:, hq:hq + hk].mul_(loud.to(dt))
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        s["out"] = torch.zeros(T, hq, d, device=dev, dtype=dt)
        s["lse"] = torch.zeros(T, hq, device=dev)
        if case["op"] == "prefill":
            starts = [0]
            for t in new:
                starts.append(starts[-1] + t)
            s["q_start"] = torch.tensor(starts, dtype=torch.int32, device=dev)
            s["max_new"] = max(new)
        # sums of the steps since the last eviction
        s["scores"] = torch.rand(B, hk, width * page, generator=g, device=dev).mul_(0.05) if case["scores"] else None
    if own:
        from paper_2503_01330_b200 import binding
        s["cache"] = binding.PagedCache(1, n_pages, page, hq, hk, d, max_batch=B, max_pages=width,
                                        dtype=binding.WKV_BF16 if case["dtype"] == "bf16" else binding.WKV_F32,
                                        scores=s["scores"] is not None, device=dev, k_pool=k_pool, v_pool=v_pool)
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
    op = s["case"]["op"]
    if own:
        return _RUN_OWN[op](s, s["case"])
    return _RUN_PLAIN[op](s, s["case"])


def _own_decode(s, c):
    s["cache"].wkv_paged_decode(0, s["q"], s["k"], s["v"], s["table"], s["seq_lens"], s["out"], window=c["window"],
                                sink=c["sink"], scores=s["scores"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"], "scores": s["scores"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _own_prefill(s, c):
    s["cache"].wkv_paged_prefill(0, s["q"], s["k"], s["v"], s["q_start"], s["table"], s["seq_lens"], s["out"],
                                 window=c["window"], sink=c["sink"], scores=s["scores"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"], "scores": s["scores"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _own_evict(s, c):
    s["cache"].wkv_paged_evict(0, s["table"], s["dst_table"], s["seq_lens"], s["new_lens"], c["budget"], c["recent"],
                               c["sink"], scores=s["scores"], scores_out=s["scores_out"], kept=s["kept"])
    return {"new_lens": s["new_lens"], "kept": s["kept"], "scores_out": s["scores_out"], "k_pool": s["k_pool"],
            "v_pool": s["v_pool"]}


_RUN_OWN = {"decode": _own_decode, "prefill": _own_prefill, "evict": _own_evict}


def _rows(pool, table):
    """[B, hk, width * page, d] in fp32: every sequence's entries in order."""
    x = pool[0][table.long()]                          # [B, width, hk, page, d]
    B, w, hk, page, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(B, hk, w * page, d).float()


def _store(pool, table, seq, idx, rows):
    """Entry idx[n] of sequence seq[n] becomes rows[n] [hk, d]."""
    page = pool.shape[3]
    pool[0][table[seq, idx // page].long(), :, idx % page] = rows


def _attend(s, c, q, pos, valid):
    """q [B, Tq, hq, d] at positions pos [B, Tq] against all entries: out [B, Tq, hq, d], lse [B, Tq, hq], weights summed over
    the tokens and averaged over a kv head's query heads [B, hk, L]."""
    B, Tq, hq, d = q.shape
    hk = c["hk"]
    G = hq // hk
    K, V = _rows(s["k_pool"], s["table"]), _rows(s["v_pool"], s["table"])
    L = K.shape[2]
    j = torch.arange(L, device=q.device)
    see = (j <= pos[..., None]) & valid[..., None]
    if c["window"]:
        see &= (j > pos[..., None] - c["window"]) | (j < c["sink"])
    V = V.masked_fill((j >= s["seq_lens"][:, None])[:, None, :, None], 0.0)
    qf = q.float().reshape(B, Tq, hk, G, d).permute(0, 2, 3, 1, 4).reshape(B, hk, G * Tq, d)
    x = (qf @ K.transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).view(B, hk, G, Tq, L)
    x.masked_fill_(~see[:, None, None], NEG)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == NEG, 0.0, m)
    x.sub_(m).exp_()
    z = x.sum(-1, keepdim=True)
    inv = torch.where(z > 0, 1.0 / z, 0.0)
    x.mul_(inv)
    out = (x.view(B, hk, G * Tq, L) @ V).view(B, hk, G, Tq, d).permute(0, 3, 1, 2, 4).reshape(B, Tq, hq, d)
    lse = (m + z.log())[..., 0].permute(0, 3, 1, 2).reshape(B, Tq, hq)
    return out, lse, (x.sum((2, 3)) / G if c["scores"] else None)


def _add_scores(s, lens, new, w):
    """Weights join the sums; entries that came with this call start from zero."""
    j = torch.arange(w.shape[-1], device=w.device)
    fresh = (j >= (lens - new)[:, None]) & (j < lens[:, None])
    s["scores"].masked_fill_(fresh[:, None], 0.0).add_(w)


def _plain_decode(s, c):
    lens = s["seq_lens"].long()
    on = lens > 0
    seq = on.nonzero()[:, 0]
    _store(s["k_pool"], s["table"], seq, lens[seq] - 1, s["k"][seq])
    _store(s["v_pool"], s["table"], seq, lens[seq] - 1, s["v"][seq])
    out, lse, w = _attend(s, c, s["q"][:, None], (lens - 1)[:, None], on[:, None])
    s["out"].copy_(out[:, 0])
    s["lse"].copy_(lse[:, 0])
    if c["scores"]:
        _add_scores(s, lens, on.long(), w)
    return {"out": s["out"], "lse": s["lse"], "scores": s["scores"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _plain_prefill(s, c):
    lens, start = s["seq_lens"].long(), s["q_start"].long()
    new = start[1:] - start[:-1]
    t = torch.arange(s["max_new"], device=lens.device)
    valid = t < new[:, None]
    row = (start[:-1, None] + t).clamp(max=s["q"].shape[0] - 1)
    pos = (lens - new)[:, None] + t
    seq, tok = valid.nonzero(as_tuple=True)
    at = row[seq, tok]
    _store(s["k_pool"], s["table"], seq, pos[seq, tok], s["k"][at])
    _store(s["v_pool"], s["table"], seq, pos[seq, tok], s["v"][at])
    out, lse, w = _attend(s, c, s["q"][row], pos, valid)
    s["out"][at] = out[seq, tok].to(s["out"].dtype)
    s["lse"][at] = lse[seq, tok]
    if c["scores"]:
        _add_scores(s, lens, new, w)
    return {"out": s["out"], "lse": s["lse"], "scores": s["scores"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _plain_evict(s, c):
    lens, x = s["seq_lens"].long(), s["scores"]
    B, hk, L = x.shape
    j = torch.arange(L, device=x.device)
    n = lens[:, None, None]
    # leave first the smallest weights, of equal ones the lowest index; the first and the newest entries stay
    safe = (j < c["sink"]) | (j >= n - c["recent"])
    order = torch.sort(x.masked_fill(safe.expand_as(x), math.inf), dim=-1, stable=True).indices
    place = torch.empty_like(order).scatter_(-1, order, j.expand_as(order))
    keep = (place >= n - c["budget"]) & (j < n)
    new = lens.clamp(max=c["budget"])
    # kept entries in their order
    idx = torch.sort((~keep).to(torch.uint8), dim=-1, stable=True).indices[..., :c["budget"]]
    if idx.shape[-1] < c["budget"]:
        idx = torch.nn.functional.pad(idx, (0, c["budget"] - idx.shape[-1]))
    live = (torch.arange(c["budget"], device=x.device) < new[:, None])[:, None].expand_as(idx)
    s["new_lens"].copy_(new)
    s["kept"].copy_(torch.where(live, idx.int(), s["kept"]))
    s["scores_out"].copy_(torch.where(live, x.gather(-1, idx), s["scores_out"]))
    b, h, i = live.nonzero(as_tuple=True)
    src, page = idx[b, h, i], c["page"]
    sp, dp = s["table"][b, src // page].long(), s["dst_table"][b, i // page].long()
    s["k_pool"][0][dp, h, i % page] = s["k_pool"][0][sp, h, src % page]
    s["v_pool"][0][dp, h, i % page] = s["v_pool"][0][sp, h, src % page]
    return {"new_lens": s["new_lens"], "kept": s["kept"], "scores_out": s["scores_out"], "k_pool": s["k_pool"],
            "v_pool": s["v_pool"]}


_RUN_PLAIN = {"decode": _plain_decode, "prefill": _plain_prefill, "evict": _plain_evict}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    """One sequence and one kv head at a time, in 64 bits.  Pools, indexes and moved weights are copies, not computed: None."""
    if case["op"] == "evict":
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    lens, new = _lengths(case)
    hk, G, page, d = case["hk"], case["hq"] // case["hk"], case["page"], case["d"]
    f8 = torch.float64
    out, lse = s["out"].to(f8), s["lse"].to(f8)
    scores = s["scores"].to(f8) if case["scores"] else None
    at = 0
    for b, (n, t) in enumerate(zip(lens, new)):
        first = b if case["op"] == "decode" else at    # the sequence's first row of q
        at += t
        if t == 0:
            if case["op"] == "decode":
                out[first], lse[first] = 0.0, NEG
            continue
        pages = s["table"][b, :-(-n // page)].long()
        rows = torch.arange(n - t, n, device="cuda")[:, None]
        col = torch.arange(n, device="cuda")[None]
        hidden = col > rows
        if case["window"]:
            hidden |= (rows - col >= case["window"]) & (col >= case["sink"])
        for h in range(hk):
            keys = s["k_pool"][0, pages, h].reshape(-1, d)[:n - t]
            vals = s["v_pool"][0, pages, h].reshape(-1, d)[:n - t]
            keys = torch.cat([keys, s["k"][first:first + t, h]]).to(f8)
            vals = torch.cat([vals, s["v"][first:first + t, h]]).to(f8)
            total = torch.zeros(n, dtype=f8, device="cuda")
            for r in range(h * G, h * G + G):
                logit = torch.einsum("td,nd->tn", s["q"][first:first + t, r].to(f8), keys) / d ** 0.5
                logit[hidden] = NEG
                norm = torch.logsumexp(logit, -1)
                weight = torch.exp(logit - norm[:, None])
                out[first:first + t, r] = weight @ vals
                lse[first:first + t, r] = norm
                total += weight.sum(0)
            if case["scores"]:
                scores[b, h, n - t:n] = 0.0
                scores[b, h, :n] += total / G
    return {"out": out, "lse": lse, "scores": scores, "k_pool": None, "v_pool": None}
