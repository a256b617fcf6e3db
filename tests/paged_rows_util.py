"""Appending with rotation, rows in 4 bits and page selection for the tests: definitions and derived bounds.

What is specified operation by operation (codes, scales, zero points, bounds of pages, scores and choice of pages) is restated here in
numpy binary32 and compared bit for bit.  The rest is compared with 64-bit arithmetic within (u = 2^-24, half a step of fp32):
  - a turned channel: two products and a sum, each rounded: 2u (|a cos| + |b sin|), then half a step of the storage type;
  - a logit over 4-bit keys: products of whole numbers, exact but for the query's: its channels become whole numbers with the head's largest
    in [2^21, 2^22), so a channel is off by half of 1, 2^-22 of the largest: scale 2^-22 max|q| sum_c |k_c|.  Then fp32: |ds| <=
    2 (d + 16) u T with T = scale sum_c |q_c| s (n_c + z) is more than the few operations per group need;
  - bf16 rows: weights go as bf16 high and low parts, 2^-9 of 2^-9: 2^-17 A with room for one more rounding;
  - a weight: E = 2 |ds| + 2^-20 + (n + 8 + 2 T) u relative, as for bf16 rows;
  - an output: (E + 2 * 2^-11) A for the weights and the rounding of p and of p s to fp16, half a step each (A = sum p s |n - z|: the same
    rounded weights multiply codes and zero points), 2 (n + 16) u B for the sums (B = sum p s (n + z)), half a step of bf16; and for
    what is below fp16's normal range: p is held times 2^14 and s times a power of two that brings the largest, s_max, to [1, 2), so p s is
    off by 2^-25 2^-14 s_max more per entry, and p s_max 2^-25 where s is below 2^-21 s_max (above that its four bits are exact): times
    |n - z| <= 15, under (n + 128) 2^-28 s_max in all;
  - a prompt on bf16 rows rounds its weights to bf16: half a step, 2^-8, of each, so 2^-8 A more (round_p);
  - a log-sum: |ds| + (n + 8) u + 2^-20 + 2u |lse|."""
import math

import numpy as np
import torch

from paper_2503_01330_b200 import binding

U = 2.0 ** -24
F = np.float32


# ---------------------------------------------------------------- rows in 4 bits, from the header's text

def quantise(x):
    """x [..., d] float32 -> codes [..., d] uint8, scales [..., d/32] float32 as stored, scale bytes, zero points."""
    x = np.asarray(x, F)
    g = x.reshape(*x.shape[:-1], -1, 32)
    lo, hi = np.minimum(g.min(-1), F(0)), np.maximum(g.max(-1), F(0))
    r = (hi - lo).astype(F) * F(1.0 / 15.0)
    mant, exp = np.frexp(r.astype(np.float64))
    step = np.exp2(np.maximum(exp, -13) - 4.0)
    s = np.clip(np.ceil(r.astype(np.float64) / step) * step, 2.0 ** -17, 4096.0).astype(F)
    inv = F(1) / s
    z = np.clip(np.rint(-lo * inv), 0, 15).astype(F)
    n = np.clip(np.rint(g * inv[..., None]) + z[..., None], 0, 15)
    byte = (s.astype(np.float16).view(np.uint16) >> 7).astype(np.uint8)
    return n.reshape(x.shape).astype(np.uint8), s, byte, z.astype(np.uint8)


def places(kind, d, page):
    """Byte and shift of every code of a chunk: [page, d] each."""
    S = d // 32
    byte, shift = np.zeros((page, d), np.int64), np.zeros((page, d), np.int64)
    for i in range(page):
        for c in range(d):
            g, r = divmod(c, 32)
            if kind == "k":
                w, e = divmod(r, 8)
                x = (i // 2) % 4 if d == 128 else (i // 4) % 2
                bit = 4 * (e // 2) + 16 * (e % 2)
                at = 16 * (g ^ x) + 4 * w
            else:
                u, e = divmod(r, 4)
                x = 32 * ((i // 2) % 2) if d == 128 else 0
                bit = 4 * e
                at = (2 * S * u + 2 * g) ^ x
            byte[i, c], shift[i, c] = i * (d // 2) + at + bit // 8, bit % 8
    return byte, shift


def pack_chunks(kind, x):
    """x [..., page, d] float32 -> chunks [..., bytes] uint8, and the values that the codes stand for."""
    page, d = x.shape[-2:]
    n, s, sb, z = quantise(x)
    byte, shift = places(kind, d, page)
    out = np.zeros((*x.shape[:-2], page * (d // 2 + d // 16)), np.uint8)
    flat, codes = out.reshape(-1, out.shape[-1]), n.reshape(-1, page * d)
    for lowhigh in (0, 4):
        sel = shift.reshape(-1) == lowhigh
        flat[:, byte.reshape(-1)[sel]] |= codes[:, sel] << lowhigh
    flat[:, page * d // 2:] = np.stack([sb, z], -1).reshape(flat.shape[0], -1)
    return out, dequantise(n, s, z)


def dequantise(n, s, z):
    g = n.reshape(*n.shape[:-1], -1, 32).astype(np.float64)
    return ((g - z[..., None].astype(np.float64)) * s[..., None].astype(np.float64)).reshape(n.shape)


def unpack_chunks(kind, chunks, page, d):
    """chunks [..., bytes] -> codes [..., page, d], scales and zero points [..., page, d/32] in 64 bits."""
    byte, shift = places(kind, d, page)
    n = (chunks[..., byte] >> shift) & 15
    pairs = chunks[..., page * d // 2:].reshape(*chunks.shape[:-1], page, d // 32, 2)
    s = (pairs[..., 0].astype(np.uint16) << 7).view(np.float16).astype(np.float64)
    return n, s, pairs[..., 1].astype(np.float64)


# ---------------------------------------------------------------- rotation

def angle_table(rows, dim, seed=0):
    """Not of any frequency: random angles show a wrong row or channel at once."""
    a = np.random.default_rng(seed).uniform(-np.pi, np.pi, (rows, dim // 2))
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], -1).astype(F))


def rotate32(x, row, paired):
    """x [heads, d] float32 turned by one row of the table, every operation in binary32."""
    x = np.asarray(x, F)
    dim = row.shape[0]
    c, w = row[:dim // 2].astype(F), row[dim // 2:].astype(F)
    ia, ib = (np.arange(0, dim, 2), np.arange(1, dim, 2)) if paired else (np.arange(dim // 2), np.arange(dim // 2, dim))
    y = x.copy()
    y[:, ia] = (x[:, ia] * c).astype(F) - (x[:, ib] * w).astype(F)
    y[:, ib] = (x[:, ib] * c).astype(F) + (x[:, ia] * w).astype(F)
    return y


def rotate64(x, row, paired):
    """... in 64 bits, and the bound's |a cos| + |b sin|."""
    x, row = np.asarray(x, np.float64), np.asarray(row, np.float64)
    dim = row.shape[0]
    c, w = row[:dim // 2], row[dim // 2:]
    ia, ib = (np.arange(0, dim, 2), np.arange(1, dim, 2)) if paired else (np.arange(dim // 2), np.arange(dim // 2, dim))
    y, m = x.copy(), np.zeros_like(x)
    y[:, ia], m[:, ia] = x[:, ia] * c - x[:, ib] * w, np.abs(x[:, ia] * c) + np.abs(x[:, ib] * w)
    y[:, ib], m[:, ib] = x[:, ib] * c + x[:, ia] * w, np.abs(x[:, ib] * c) + np.abs(x[:, ia] * w)
    return y, m


# ---------------------------------------------------------------- bounds of pages, scores, choice

def page_bounds(keys):
    """keys [n, d] as stored -> codes int8 [2, d], scale."""
    keys = np.asarray(keys, F)
    hi, lo = keys.max(0), keys.min(0)
    scale = F(max(abs(float(hi.max())), abs(float(hi.min())), abs(float(lo.max())), abs(float(lo.min())))) * F(1.0 / 127.0)
    inv = F(1) / scale if scale >= 2.0 ** -100 else F(0)
    up, down = np.minimum(np.ceil(hi * inv), 127), np.maximum(np.floor(lo * inv), -127)
    return np.stack([up, down]).astype(np.int8), F(scale)


def query_codes(q):
    """q [G, d] of one kv head -> int64 [2, d]."""
    q = np.asarray(q, F)
    u, w = np.maximum(q[0], F(0)), np.minimum(q[0], F(0))
    for g in range(1, q.shape[0]):
        u, w = (u + np.maximum(q[g], F(0))).astype(F), (w + np.minimum(q[g], F(0))).astype(F)
    step = F(max(u.max(), (-w).max())) * F(1.0 / 127.0)
    inv = F(1) / step if step >= 2.0 ** -100 else F(0)
    return np.stack([np.clip(np.rint(u * inv), 0, 127), np.clip(np.rint(w * inv), -127, 0)]).astype(np.int64)


def choose_pages(scores, n_select, recent, sink):
    """scores [n] float32 -> the chosen indexes, rising."""
    n = len(scores)
    taken = [p for p in range(n) if p < sink or p >= n - recent]
    rest = sorted((p for p in range(n) if p not in set(taken)), key=lambda p: (-float(scores[p]), p))
    return sorted(taken + rest[:max(0, min(n_select, n) - len(taken))])


# ---------------------------------------------------------------- attention in 64 bits

def attend(q, K, V, see, scale, half, Kabs=None, Vabs=None, s_max=0.0, round_p=0.0):
    """One head: q [d], K, V [n, d] in 64 bits, see [n].  Output, log-sum and their bounds; Kabs, Vabs: s (n + z) of 4-bit rows."""
    n, d = K.shape
    four = Kabs is not None
    if not see.any():
        return np.zeros(d), -math.inf, np.zeros(d), 0.0
    x = np.where(see, K @ q * scale, -np.inf)
    z = float(np.logaddexp.reduce(x[see]))
    p = np.exp(x - z)
    T = float((np.abs(q) @ (Kabs if four else np.abs(K)).T)[see].max()) * scale
    ds = 2 * (d + 16) * U * T
    if four:
        ds += scale * 2.0 ** -22 * float(np.abs(q).max()) * float(np.abs(K).sum(-1)[see].max())
    E = 2 * ds + 2.0 ** -20 + (n + 8 + 2 * T) * U
    out = p @ V
    A = p @ np.abs(V)
    B = p @ Vabs if four else A
    bound = (E + round_p + (2.0 ** -10 if four else 2.0 ** -17 if half > 2.0 ** -20 else 0.0)) * A + 2 * (n + 16) * U * B + ((n + 128) * 2.0 ** -28 * s_max if four else 0.0)
    bound = bound * (1 + half) + half * np.abs(out) + 1e-37
    return out, z, bound, ds + (n + 8) * U + 2.0 ** -20 + 2 * U * abs(z)


# ---------------------------------------------------------------- a cache with its contents

class Pool:
    """Ragged sequences in pages of a cache of any row type; contents known in 64 bits."""

    def __init__(self, lens, hq=4, hk=2, d=128, kind="kv4", page=16, layers=1, seed=0, spare=2, extra_cols=0, spread=1.0, width=None):
        self.lens, self.hq, self.hk, self.d, self.kind, self.page, self.layers = list(lens), hq, hk, d, kind, page, layers
        self.G, self.layer, self.scale = hq // hk, layers - 1, 1.0 / math.sqrt(d)
        self.tdt = torch.float32 if kind == "f32" else torch.bfloat16
        self.half = torch.finfo(self.tdt).eps / 2
        g = torch.Generator().manual_seed(seed * 7919 + 17)
        B = len(self.lens)
        used = [-(-n // page) for n in self.lens]
        self.width = (max(used + [1]) + extra_cols) if width is None else width
        self.n_pages = sum(used) + spare
        order = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((B, self.width), 0x7ffffff0, dtype=torch.int32)
        at = 0
        for b, n in enumerate(used):
            self.table[b, :n] = order[at:at + n].int()
            at += n
        self.free_pages = order[at:].int()
        shape = (layers, self.n_pages, hk, page, d)
        K, V = torch.randn(shape, generator=g), torch.randn(shape, generator=g)
        K[..., :3] *= 3.0
        K, V = K * spread, V * spread
        if kind == "kv4":
            kc, _ = pack_chunks("k", K.bfloat16().float().numpy())
            vc, _ = pack_chunks("v", V.bfloat16().float().numpy())
            self.k_pool, self.v_pool = torch.from_numpy(kc), torch.from_numpy(vc)
        else:
            self.k_pool, self.v_pool = K.to(self.tdt), V.to(self.tdt)
        self.q = torch.randn(B, hq, d, generator=g).to(self.tdt)
        self.g = g

    def garbage(self, value=0xff):
        """Rows behind every sequence's length and pages of nobody get any bits."""
        for name, pool in (("k", self.k_pool), ("v", self.v_pool)):
            raw = pool if self.kind == "kv4" else None
            live = {}
            for b, n in enumerate(self.lens):
                for c in range(-(-n // self.page)):
                    live[int(self.table[b, c])] = min(self.page, n - c * self.page)
            for pg in range(self.n_pages):
                n = live.get(pg, 0)
                if raw is None:
                    pool[:, pg, :, n:] = float("nan")
                else:
                    nc, d, page = self.d // 2, self.d, self.page
                    pool[:, pg, :, n * nc:page * nc] = value
                    pool[:, pg, :, page * nc + n * (d // 16):] = value

    def cache(self, **kw):
        self.gk, self.gv = self.k_pool.cuda(), self.v_pool.cuda()
        dtype = {"kv4": binding.WKV_KV4, "f32": binding.WKV_F32, "bf16": binding.WKV_BF16}[self.kind]
        args = dict(max_batch=max(1, len(self.lens)), max_pages=self.width, dtype=dtype, k_pool=self.gk, v_pool=self.gv)
        return binding.PagedCache(self.layers, self.n_pages, self.page, self.hq, self.hk, self.d, **{**args, **kw})

    def dev(self):
        return self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32, device="cuda")

    def rows(self, b, h, n=None, k_pool=None, v_pool=None):
        """Entries of sequence b, kv head h in 64 bits: K, V and for 4-bit rows s (n + z) of both, the largest value scale."""
        n = self.lens[b] if n is None else n
        pages = self.table[b, :-(-n // self.page)].long()
        kp, vp = (self.k_pool if k_pool is None else k_pool), (self.v_pool if v_pool is None else v_pool)
        kc, vc = kp[self.layer, pages, h].cpu(), vp[self.layer, pages, h].cpu()
        if self.kind != "kv4":
            return [x.double().reshape(-1, self.d).numpy()[:n] for x in (kc, vc)] + [None, None, 0.0]
        out = []
        for kind, x in (("k", kc), ("v", vc)):
            c, s, z = unpack_chunks(kind, x.numpy(), self.page, self.d)
            c, s, z = c.reshape(-1, self.d), s.reshape(-1, self.d // 32), z.reshape(-1, self.d // 32)
            rep = lambda y: np.repeat(y, 32, axis=-1)
            out.append(((c - rep(z)) * rep(s))[:n])
            out.append(((c + rep(z)) * rep(s))[:n])
        return [out[0], out[2], out[1], out[3], float(s[:n].max()) if n else 0.0]

    def check(self, out, lse, see_of, what="", q=None, lens=None, round_p=0.0):
        """out [B, hq, d], lse [B, hq] against 64 bits; see_of(b, h): which of the entries are seen."""
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        q = (self.q if q is None else q).double().cpu().numpy()
        lens = self.lens if lens is None else lens
        for b, n in enumerate(lens):
            for h in range(self.hk):
                if n:
                    K, V, Ka, Va, sm = self.rows(b, h, n, getattr(self, "gk", None), getattr(self, "gv", None))
                    see = see_of(b, h)
                for r in range(h * self.G, h * self.G + self.G):
                    if n == 0 or not see.any():
                        assert (out[b, r] == 0).all() and lse[b, r] == -math.inf, f"{what}: empty row {b}"
                        continue
                    w, z, bo, bz = attend(q[b, r], K, V, see, self.scale, self.half, Ka, Va, sm, round_p)
                    e = np.abs(out[b, r] - w) / bo
                    assert (e <= 1).all(), f"{what}: output of sequence {b}, head {r}: {e.max():.3g} of the bound at {int(e.argmax())}"
                    assert abs(lse[b, r] - z) <= bz, f"{what}: log-sum of sequence {b}, head {r}: {abs(lse[b, r] - z) / bz:.3g} of the bound"


def window_sees(n, window, sink):
    i = np.arange(n)
    return np.ones(n, bool) if not window else (i >= n - window) | (i < sink)
