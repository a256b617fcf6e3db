"""A paged cache in 64 bits for the tests, and the bounds that the library's results have to keep.

Bounds.  With u = 2^-24 (half a step of fp32) and A = sum_i p_i |v_i|:
  - a logit is a sum of d products accumulated in fp32 (tensor cores may truncate: 2u a step), scaled by a rounded factor:
    |ds| <= 2 (d + 4) u S, S = scale * max_i sum_c |q_c k_ic|;
  - a weight p_i = 2^(s_i log2e - m) / l then has the relative error 2 |ds| + 2^-21 (ex2.approx: 2 ulp, and the argument's
    rounding, |argument| * u, which the factor S + 4 below covers) + n u for the sum l of n terms:
    E = 4 (d + 4) u S + 2^-20 + (n + 8 + 2 S) u;
  - an output is off by E A (weights) + (n + 8) u A (accumulation) + its own rounding, half a step of its type;
    where the kernel rounds the weights to bf16 for the tensor cores (prompts on bf16 rows), by 2^-8 A more;
  - a log-sum is off by |ds| + (n + 8) u + 2^-20, and its own rounding 2u |lse|;
  - a sum of weights over T tokens: E + (T + 8) u, relative, plus rounding of the old sum it joins."""
import math

import torch

from paper_2503_01330_b200 import binding

U = 2.0 ** -24


class Case:
    def __init__(self, lens, new, hq=4, hk=2, d=64, dtype="bf16", page=16, window=0, sink=0, scores=False, layers=1, seed=0,
                 strided=False, extra_cols=0, extra_rows=0, append=True, prefill=None, spare=3, garbage=float("nan"), width=None,
                 spikes=0.0):
        self.lens, self.new = list(lens), list(new)
        self.hq, self.hk, self.d, self.page, self.G = hq, hk, d, page, hq // hk
        self.window, self.sink, self.append, self.layers = window, sink, append, layers
        self.prefill = (max(new) > 1 if new else False) if prefill is None else prefill
        self.bf16 = dtype == "bf16"
        self.tdt = torch.bfloat16 if self.bf16 else torch.float32
        g = torch.Generator().manual_seed(seed * 7919 + 13)
        B = len(self.lens)
        used = [-(-n // page) for n in self.lens]
        self.width = (max(used + [1]) + extra_cols) if width is None else width
        self.n_pages = sum(used) + spare
        order = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((B, self.width), 0x7ffffff0, dtype=torch.int32)     # columns behind the last page: never read
        at = 0
        for b, n in enumerate(used):
            self.table[b, :n] = order[at:at + n].int()
            at += n
        self.free_pages = order[at:].int()
        shape = (layers, self.n_pages, hk, page, d)
        self.k_pool = torch.full(shape, garbage, dtype=self.tdt)
        self.v_pool = torch.full(shape, garbage, dtype=self.tdt)
        self.layer = layers - 1
        self.K, self.V = [], []                      # [len, hk, d] in the storage type
        for b, n in enumerate(self.lens):
            k, v = torch.randn(n, hk, d, generator=g), torch.randn(n, hk, d, generator=g)
            k[..., :2] *= 3.0
            if spikes:                               # a few keys whose logits tower over all before them
                k[torch.rand(n, generator=g) < spikes] *= 25.0
            self.K.append(k.to(self.tdt))
            self.V.append(v.to(self.tdt))
            there = n - (self.new[b] if append else 0)
            for i in range(n):
                if i < there:
                    pg = int(self.table[b, i // page])
                    self.k_pool[self.layer, pg, :, i % page] = self.K[b][i]
                    self.v_pool[self.layer, pg, :, i % page] = self.V[b][i]
        self.starts = [0]
        if self.prefill:
            for t in self.new:
                self.starts.append(self.starts[-1] + t)
            T = self.starts[-1] + extra_rows
        else:
            T = B
            self.starts = list(range(B + 1))
        self.T = T
        pad = 8 if strided else 0
        buf = torch.randn(T, hq + 2 * hk + pad, d, generator=g).to(self.tdt)
        for b in range(B):
            t, n = self.new[b], self.lens[b]
            s = self.starts[b]
            buf[s:s + t, hq:hq + hk] = self.K[b][n - t:n]
            buf[s:s + t, hq + hk:hq + 2 * hk] = self.V[b][n - t:n]
        self.buf = buf
        self.strided = strided
        self.scores = torch.rand(B, hk, self.width * page, generator=g) if scores else None

    # ---- the library ----
    def cache(self, **kw):
        self.gk, self.gv = self.k_pool.cuda(), self.v_pool.cuda()
        return binding.PagedCache(self.layers, self.n_pages, self.page, self.hq, self.hk, self.d, max_batch=max(1, len(self.lens)),
                                  max_pages=self.width, dtype=binding.WKV_BF16 if self.bf16 else binding.WKV_F32,
                                  scores=self.scores is not None, k_pool=self.gk, v_pool=self.gv, **kw)

    def rows(self):
        buf = self.buf.cuda()
        q, k, v = buf[:, :self.hq], buf[:, self.hq:self.hq + self.hk], buf[:, self.hq + self.hk:self.hq + 2 * self.hk]
        return (q, k, v) if self.strided else (q.contiguous(), k.contiguous(), v.contiguous())

    def run(self, cache=None):
        c = cache or self.cache()
        q, k, v = self.rows()
        if not self.append:
            k = v = None
        out = torch.full((self.T, self.hq, self.d), 7.0, dtype=self.tdt, device="cuda")
        lse = torch.full((self.T, self.hq), 7.0, device="cuda")
        scores = None if self.scores is None else self.scores.cuda()
        table, lens = self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        if self.prefill:
            start = torch.tensor(self.starts, dtype=torch.int32, device="cuda")
            c.wkv_paged_prefill(self.layer, q, k, v, start, table, lens, out, self.window, self.sink, scores, lse)
        else:
            c.wkv_paged_decode(self.layer, q, k, v, table, lens, out, self.window, self.sink, scores, lse)
        status = c.wkv_status()
        if cache is None:
            c.close()
        assert status == 0
        return out, lse, scores

    # ---- the definition ----
    def check(self, out, lse, scores=None, what=""):
        out, lse = out.double().cpu(), lse.double().cpu()
        scale = 1.0 / math.sqrt(self.d)
        round_p = 2.0 ** -8 if self.bf16 and self.prefill else 0.0
        half = torch.finfo(self.tdt).eps / 2
        touched = torch.zeros(self.T, dtype=torch.bool)
        for b, (n, t) in enumerate(zip(self.lens, self.new)):
            first = self.starts[b]
            if t == 0:
                if not self.prefill:
                    assert (out[first] == 0).all() and torch.isneginf(lse[first]).all(), f"{what}: padded row {b}"
                    touched[first] = True
                if scores is not None:
                    assert torch.equal(scores[b].cpu(), self.scores[b])
                continue
            touched[first:first + t] = True
            pos = torch.arange(n - t, n)[:, None]
            j = torch.arange(n)[None]
            see = j <= pos
            if self.window:
                see &= (j > pos - self.window) | (j < self.sink)
            for h in range(self.hk):
                K, V = self.K[b][:, h].double(), self.V[b][:, h].double()
                w = torch.zeros(n, dtype=torch.float64)
                worst_e = 0.0
                for g in range(self.G):
                    r = h * self.G + g
                    q = self.buf[first:first + t, r].double()
                    x = (q @ K.T * scale).masked_fill(~see, -math.inf)
                    z = torch.logsumexp(x, -1, keepdim=True)
                    p = (x - z).exp()
                    S = scale * (q.abs() @ K.abs().T).masked_fill(~see, 0).amax(-1, keepdim=True)
                    ds = 2 * (self.d + 4) * U * S
                    E = 2 * ds + 2.0 ** -20 + (n + 8 + 2 * S) * U
                    want, A = p @ V, p @ V.abs()
                    err = (out[first:first + t, r] - want).abs()
                    bound = (E + (n + 8) * U + round_p) * A * (1 + half) + half * want.abs() + 1e-37
                    assert (err <= bound).all(), (f"{what}: output of sequence {b}, head {r}: {float((err / bound).max()):.3g} "
                                                  f"of the bound at {(err / bound).flatten().argmax()}")
                    e_lse = (lse[first:first + t, r] - z[:, 0]).abs()
                    b_lse = (ds + (n + 8) * U + 2.0 ** -20 + 2 * U * z.abs())[:, 0]
                    assert (e_lse <= b_lse).all(), f"{what}: log-sum of sequence {b}, head {r}: {float((e_lse / b_lse).max()):.3g}"
                    w += p.sum(0)
                    worst_e = max(worst_e, float(E.max()))
                if scores is not None:
                    base = self.scores[b, h, :n].double().clone()
                    if self.append:
                        base[n - t:] = 0
                    want = base + w / self.G
                    got = scores[b, h].double().cpu()
                    bound = worst_e * w / self.G + (t * self.G + 8) * U * w / self.G + 2 * U * want.abs() + 1e-37
                    bad = (got[:n] - want).abs() / bound
                    assert (bad <= 1).all(), f"{what}: weights of sequence {b}, kv head {h}: {float(bad.max()):.3g} at {int(bad.argmax())}"
                    assert torch.equal(got[n:].float(), self.scores[b, h, n:]), f"{what}: weights behind sequence {b}"
        assert (out[~touched] == 7).all() and (lse[~touched] == 7).all(), f"{what}: rows of no sequence were written"
        self.check_pool(what)

    def check_pool(self, what=""):
        """Every row of the pool: the entries where they belong, all other rows bit for bit as they were."""
        for name, pool, was, rows in (("K", self.gk, self.k_pool, self.K), ("V", self.gv, self.v_pool, self.V)):
            want = was.clone()
            for b, n in enumerate(self.lens):
                for i in range(n):
                    want[self.layer, int(self.table[b, i // self.page]), :, i % self.page] = rows[b][i]
            i16 = torch.int16 if self.bf16 else torch.int32
            assert torch.equal(pool.cpu().view(i16), want.view(i16)), f"{what}: pool of {name}"


def run_and_check(what="", **kw):
    c = Case(**kw)
    out, lse, scores = c.run()
    c.check(out, lse, scores, what)
    return c
