"""Appending with rotation (bf16, fp32 and 4-bit rows, bounds of pages) and spreading 4-bit rows out."""
import numpy as np
import pytest
import torch

from paged_rows_util import U, Pool, angle_table, pack_chunks, page_bounds, rotate32, rotate64, unpack_chunks
from paper_2503_01330_b200 import binding

pytestmark = pytest.mark.gpu


class Append:
    """One call and its definition."""

    def __init__(self, lens, new, kind="bf16", hq=4, hk=2, d=128, page=16, rot=None, paired=False, bounds=False, shift=None, step=False,
                 extra_rows=0, strided=False, inplace=False, layers=1, seed=0, no_q=False, no_kv=False):
        self.P = P = Pool(lens, hq=hq, hk=hk, d=d, kind=kind, page=page, layers=layers, seed=seed)
        self.new, self.step, self.paired, self.bounds, self.inplace, self.no_q, self.no_kv = list(new), step, paired, bounds, inplace, no_q, no_kv
        B = len(lens)
        self.starts = list(range(B + 1)) if step else list(np.concatenate([[0], np.cumsum(new)]))
        self.T = B if step else self.starts[-1] + extra_rows
        buf = torch.randn(self.T, hq + 2 * hk + (1 if strided else 0), d, generator=P.g).to(P.tdt)
        self.buf, self.strided = buf, strided
        self.tok = [(b, self.starts[b] + t, P.lens[b] - new[b] + t) for b in range(B) for t in range(new[b])]     # sequence, row, entry
        self.pos = None
        rows = max(list(lens) + [1])
        if shift is not None:
            rows += shift
            self.pos = torch.zeros(self.T, dtype=torch.int32)
            for b, r, i in self.tok:
                self.pos[r] = rows - 1 - i if shift == 0 else i + shift
        self.rope = None if rot == 0 else angle_table(rows, rot or d, seed)

    def turned(self, x, r, i, exact):
        x = x.float().numpy()
        if self.rope is None:
            return (x.astype(np.float64), np.zeros_like(x)) if exact else x
        row = self.rope[int(self.pos[r]) if self.pos is not None else i].numpy()
        return rotate64(x, row, self.paired) if exact else rotate32(x, row, self.paired)

    def run(self, cache=None):
        P, hq, hk = self.P, self.P.hq, self.P.hk
        c = cache or P.cache()
        buf = self.buf.cuda()
        q, k, v = buf[:, :hq], buf[:, hq:hq + hk], buf[:, hq + hk:hq + 2 * hk]
        if not self.strided:
            q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        q_out = q if self.inplace else torch.full((self.T, hq, P.d), 7.0, dtype=P.tdt, device="cuda")
        if self.no_q:
            q = q_out = None
        if self.no_kv:
            k = v = None
        table, lens = P.dev()
        kw = {}
        if self.bounds:
            self.gb = torch.full((P.layers, P.n_pages, hk, 2, P.d), 77, dtype=torch.int8, device="cuda")
            self.gs = torch.full((P.layers, P.n_pages, hk), 7.0, device="cuda")
            kw = dict(page_bounds=self.gb, page_scale=self.gs)
        c.wkv_paged_append(P.layer, q, k, v, table, lens, None if self.step else torch.tensor(self.starts, dtype=torch.int32, device="cuda"),
                           None if self.rope is None else self.rope.cuda(), self.paired, None if self.pos is None else self.pos.cuda(), q_out, **kw)
        self.status = c.wkv_status()
        if cache is None:
            c.close()
        return q_out

    def check(self, q_out, what=""):
        P, hq, hk = self.P, self.P.hq, self.P.hk
        assert self.status == 0
        if not self.no_q:
            got = q_out.double().cpu().numpy()
            touched = np.zeros(self.T, bool)
            for b, r, i in self.tok:
                touched[r] = True
                w, m = self.turned(self.buf[r, :hq], r, i, True)
                e = np.abs(got[r] - w) - (2 * U * m * (1 + P.half) + P.half * np.abs(w) + 1e-38)
                assert (e <= 0).all(), f"{what}: queries of row {r}"
                exact = self.turned(self.buf[r, :hq], r, i, False)
                assert torch.equal(q_out[r].cpu(), torch.from_numpy(exact).to(P.tdt)), f"{what}: queries of row {r}, bit for bit"
            left = self.buf[:, :hq].cpu() if self.inplace else torch.full((self.T, hq, P.d), 7.0, dtype=P.tdt)
            assert torch.equal(q_out.cpu()[~touched], left[~touched]), f"{what}: rows of no sequence"
        # the pool: new rows where they belong, everything else as it was
        want_k, want_v = P.k_pool.clone(), P.v_pool.clone()
        pages = {}
        if not self.no_kv:
            for b, r, i in self.tok:
                pages.setdefault((b, i // P.page), []).append((r, i))
        for (b, p), toks in pages.items():
            pg = int(P.table[b, p])
            ks = np.stack([self.turned(self.buf[r, hq:hq + hk], r, i, False) for r, i in toks], 1)           # [hk, n, d]
            vs = np.stack([self.buf[r, hq + hk:hq + 2 * hk].float().numpy() for r, i in toks], 1)
            at = [i % P.page for r, i in toks]
            if P.kind != "kv4":
                want_k[P.layer, pg, :, at] = torch.from_numpy(ks).to(P.tdt)
                want_v[P.layer, pg, :, at] = torch.from_numpy(vs).to(P.tdt)
                continue
            nc, npair = P.d // 2, P.d // 16
            for kind, rows, want in (("k", ks, want_k), ("v", vs, want_v)):
                full = np.zeros((hk, P.page, P.d), np.float32)
                full[:, at] = rows
                chunk = torch.from_numpy(pack_chunks(kind, full)[0])
                lo, hi = min(at), max(at) + 1
                want[P.layer, pg, :, lo * nc:hi * nc] = chunk[:, lo * nc:hi * nc]
                o = P.page * nc
                want[P.layer, pg, :, o + lo * npair:o + hi * npair] = chunk[:, o + lo * npair:o + hi * npair]
        bits = {"kv4": torch.uint8, "bf16": torch.int16, "f32": torch.int32}[P.kind]
        assert torch.equal(P.gk.cpu().view(bits), want_k.view(bits)), f"{what}: keys"
        assert torch.equal(P.gv.cpu().view(bits), want_v.view(bits)), f"{what}: values"
        if self.bounds:
            gb, gs = self.gb.cpu().numpy(), self.gs.cpu().numpy()
            seen = set()
            for (b, p), toks in pages.items():
                pg = int(P.table[b, p])
                seen.add(pg)
                n = min(P.page, P.lens[b] - p * P.page)
                for h in range(hk):
                    if P.kind == "kv4":
                        c, s, z = unpack_chunks("k", want_k[P.layer, pg, h].numpy(), P.page, P.d)
                        keys = ((c - np.repeat(z, 32, -1)) * np.repeat(s, 32, -1))[:n]
                    else:
                        keys = want_k[P.layer, pg, h, :n].float().numpy()
                    wb, ws = page_bounds(keys)
                    assert (gb[P.layer, pg, h] == wb).all() and gs[P.layer, pg, h] == ws, f"{what}: bounds of page {pg}"
            others = [pg for pg in range(P.n_pages) if pg not in seen]
            assert (gb[:, others] == 77).all() and (gs[:, others] == 7).all()


def go(*a, what="", **kw):
    x = Append(*a, **kw)
    x.check(x.run(), what)
    return x


KINDS = ["bf16", "f32", "kv4"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("bounds", [False, True])
def test_chunks(kind, d, page, bounds):
    go([40, 1, 64, 65, 150, 7], [40, 1, 1, 33, 20, 0], kind=kind, d=d, page=page, bounds=bounds, extra_rows=3, seed=page + d)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("paired", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 32, 48, 64, 80, 112, 128])
def test_rotations(kind, paired, rot):
    go([20, 37], [5, 37], kind=kind, rot=rot, paired=paired, bounds=True, seed=rot)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hk", [(1, 1), (8, 1), (32, 8), (16, 16), (3, 3)])
def test_steps(kind, hq, hk):
    go([1, 16, 17, 0, 48, 100], [1, 1, 1, 0, 1, 1], kind=kind, hq=hq, hk=hk, bounds=True, step=True, strided=True, seed=hq)


@pytest.mark.parametrize("kind", KINDS)
def test_positions_and_layers(kind):
    go([30, 16], [30, 2], kind=kind, shift=1000, layers=3, bounds=True, seed=1)
    go([30, 16], [7, 2], kind=kind, shift=0, layers=2, strided=True, seed=2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("strided", [False, True])
def test_queries_in_place_alone_and_not_at_all(kind, strided):
    go([50, 8], [50, 3], kind=kind, inplace=True, strided=strided, extra_rows=2, seed=3)
    go([50, 8], [50, 3], kind=kind, no_kv=True, strided=strided, seed=4)
    go([50, 8], [50, 3], kind=kind, no_q=True, strided=strided, seed=5)


def test_long_chunks_and_many_sequences():
    go([1000, 333], [1000, 300], kind="bf16", hq=8, hk=4, page=64, bounds=True, seed=6)
    go([900], [850], kind="kv4", hq=4, hk=4, page=32, seed=7)
    go([(i * 7) % 23 for i in range(300)], [((i * 7) % 23) // 2 for i in range(300)], kind="f32", hq=2, hk=1, d=64, seed=8)


def test_4_bit_rows_of_any_size():
    """Zeros, one sign only, the border of the scales, values that saturate: codes bit for bit, and the error that the format promises."""
    x = Append([48], [48], kind="kv4", hq=2, hk=2, rot=0, bounds=True, seed=9)
    k = x.buf[:, 2:4]
    for r in range(48):
        k[r] = (k[r].float() * 2.0 ** (r - 24)).bfloat16()
    k[3] = 0
    k[5] = k[5].abs()
    k[7] = -k[7].abs()
    k[20] = 1.0
    x.buf[:, 4:6] = k.flip(0)
    x.check(x.run())
    vals = []
    for p in range(3):
        c, s, z = unpack_chunks("k", x.P.gk[0, int(x.P.table[0, p]), 0].cpu().numpy(), 16, 128)
        vals.append(((c - np.repeat(z, 32, -1)) * np.repeat(s, 32, -1), np.repeat(s, 32, -1)))
    got, s = np.concatenate([v[0] for v in vals]), np.concatenate([v[1] for v in vals])
    want = k[:, 0].double().numpy()
    g = want.reshape(48, 4, 32)
    fits = np.repeat(np.maximum(g.max(-1), 0) - np.minimum(g.min(-1), 0) <= 15 * 4096, 32, -1)
    # half a step for the code, half a step where rounded ends meet
    assert (np.abs(got - want)[fits] <= s[fits] * (1 + 2.0 ** -20)).all()
    assert (got[3] == 0).all()


@pytest.mark.parametrize("kind", KINDS)
def test_bad_pages_and_positions(kind):
    x = Append([40, 20], [40, 4], kind=kind, bounds=True, seed=10)
    x.P.table[0, 1] = x.P.n_pages
    q = x.run()
    assert x.status == binding.WKV_ERR_STATE
    # the other pages got theirs
    ok = Append([40, 20], [40, 4], kind=kind, bounds=True, seed=10)
    q2 = ok.run()
    assert torch.equal(q, q2)
    bad = int(ok.P.table[0, 1])
    keep = [p for p in range(ok.P.n_pages) if p != bad]
    assert torch.equal(x.P.gk[:, keep].view(torch.uint8), ok.P.gk[:, keep].view(torch.uint8))
    assert torch.equal(x.P.gk[:, bad].cpu().view(torch.uint8), x.P.k_pool[:, bad].view(torch.uint8))
    # positions outside of the table leave their rows unturned
    y = Append([10], [10], kind=kind, shift=5, seed=11)
    y.pos[3], y.pos[6] = y.rope.shape[0], -1
    q = y.run()
    assert y.status == binding.WKV_ERR_STATE
    for r in (3, 6):
        assert torch.equal(q[r].cpu(), y.buf[r, :4])


def test_offsets_that_do_not_rise_or_run_over():
    x = Append([20, 20, 20], [5, 5, 5], kind="bf16", seed=12)
    for starts in ([0, 9, 3, 15], [0, 5, 10, 99], [-3, 5, 10, 15]):
        x.starts = starts
        x.run()
        assert x.status == binding.WKV_ERR_STATE


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,to_page", [(16, 16), (16, 64), (64, 16), (32, 32)])
def test_spreading_out(d, page, to_page):
    lens = [1, 0, 64, 65, 200, 17]
    P = Pool(lens, hq=4, hk=2, d=d, page=page, layers=2, extra_cols=1, seed=20)
    P.garbage()
    Q = Pool(lens, hq=4, hk=2, d=d, kind="bf16", page=to_page, layers=3, seed=21, extra_cols=6)
    a, b = P.cache(), Q.cache()
    table, n = P.dev()
    Q.layer = 1
    a.wkv_paged_expand(1, table, n, b, 1, Q.table.cuda())
    assert a.wkv_status() == 0 and b.wkv_status() == 0
    want_k, want_v = Q.k_pool.clone(), Q.v_pool.clone()
    for s, m in enumerate(lens):
        for h in range(2):
            K, V = P.rows(s, h)[:2] if m else ([], [])
            for i in range(m):
                pg = int(Q.table[s, i // to_page])
                want_k[1, pg, h, i % to_page] = torch.from_numpy(K[i]).bfloat16()
                want_v[1, pg, h, i % to_page] = torch.from_numpy(V[i]).bfloat16()
                assert torch.equal(want_k[1, pg, h, i % to_page].double(), torch.from_numpy(K[i]))      # a value is a bf16 number
    assert torch.equal(Q.gk.cpu(), want_k) and torch.equal(Q.gv.cpu(), want_v)


def test_spreading_out_bad_pages():
    P, Q = Pool([40, 40], seed=22), Pool([40, 40], kind="bf16", seed=23)
    P.table[0, 1] = -7
    Q.table[1, 2] = Q.n_pages + 5
    a, b = P.cache(), Q.cache()
    table, n = P.dev()
    a.wkv_paged_expand(0, table, n, b, 0, Q.table.cuda())
    assert a.wkv_status() == binding.WKV_ERR_STATE
    assert (Q.gk[0, int(Q.table[0, 1])] == 0).all() and (Q.gv[0, int(Q.table[0, 1])] == 0).all()
    a.wkv_paged_expand(0, table, n, b, 0, Q.table[:, :1].contiguous().cuda())     # too few columns
    assert a.wkv_status() == binding.WKV_ERR_STATE
    K = P.rows(1, 0)[0]
    assert torch.equal(Q.gk[0, int(Q.table[1, 0]), 0].double().cpu(), torch.from_numpy(K[:16]))


def test_captured_append_follows_lengths():
    P = Pool([40, 40], kind="bf16", seed=24)
    c = P.cache()
    table, _ = P.dev()
    n = torch.ones(2, dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros(2, h, 128, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2))
    q_out, rope = torch.zeros_like(q), angle_table(40, 128, 3)
    rg = rope.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.wkv_set_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.wkv_paged_append(0, q, k, v, table, n, rope=rg, q_out=q_out)
        for lens in ([7, 33], [40, 1]):
            n.copy_(torch.tensor(lens, dtype=torch.int32))
            for x in (q, k, v):
                x.copy_(torch.randn(x.shape))
            graph.replay()
            s.synchronize()
            for b, m in enumerate(lens):
                want = rotate32(k[b].float().cpu().numpy(), rope[m - 1].numpy(), False)
                assert torch.equal(P.gk[0, int(P.table[b, (m - 1) // 16]), :, (m - 1) % 16].cpu(), torch.from_numpy(want).bfloat16())
                want = rotate32(q[b].float().cpu().numpy(), rope[m - 1].numpy(), False)
                assert torch.equal(q_out[b].cpu(), torch.from_numpy(want).bfloat16())
    assert c.wkv_status() == 0


def test_calls_of_no_tokens():
    P = Pool([0, 0], kind="bf16", seed=25)
    c = P.cache()
    table, n = P.dev()
    q, k = (torch.zeros(0, h, 128, dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    gb, gs = torch.zeros(1, P.n_pages, 2, 2, 128, dtype=torch.int8, device="cuda"), torch.zeros(1, P.n_pages, 2, device="cuda")
    before = c.wkv_launch_count()
    c.wkv_paged_append(0, q, k, k, table, n, torch.zeros(3, dtype=torch.int32, device="cuda"), angle_table(4, 128).cuda(), q_out=q,
                       page_bounds=gb, page_scale=gs)
    assert c.wkv_status() == 0 and c.wkv_launch_count() == before


def test_calls_on_another_stream_than_their_pools():
    """A handle moved to another stream, and a destination that lives on the first one."""
    P, Q = Pool([300, 77], seed=26), Pool([300, 77], kind="bf16", seed=27)
    a, b = P.cache(), Q.cache()
    table, n = P.dev()
    to = Q.table.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a.wkv_set_stream(s)
    a.wkv_paged_expand(0, table, n, b, 0, to)
    torch.cuda.current_stream().wait_stream(s)
    assert a.wkv_status() == 0
    for q, m in enumerate(P.lens):
        for h in range(2):
            K, V = P.rows(q, h)[:2]
            for i in (0, 15, 16, m - 1):
                pg = int(Q.table[q, i // 16])
                assert torch.equal(Q.gk[0, pg, h, i % 16].double().cpu(), torch.from_numpy(K[i]))
                assert torch.equal(Q.gv[0, pg, h, i % 16].double().cpu(), torch.from_numpy(V[i]))
