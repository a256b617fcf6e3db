"""Choosing pages by their bounds and attending to chosen pages; a run of all calls together, as a serving loop makes them."""
import numpy as np
import pytest
import torch

from paged_rows_util import Pool, angle_table, choose_pages, page_bounds, query_codes, rotate32, window_sees
from paper_2503_01330_b200 import binding

pytestmark = pytest.mark.gpu
KINDS = ["bf16", "f32", "kv4"]


def bounds_of(P):
    b = np.zeros((P.layers, P.n_pages, P.hk, 2, P.d), np.int8)
    s = np.zeros((P.layers, P.n_pages, P.hk), np.float32)
    for q, n in enumerate(P.lens):
        for h in range(P.hk):
            if n == 0:
                continue
            K = P.rows(q, h)[0]
            for p in range(-(-n // P.page)):
                pg = int(P.table[q, p])
                b[P.layer, pg, h], s[P.layer, pg, h] = page_bounds(K[p * P.page:(p + 1) * P.page])
    return torch.from_numpy(b), torch.from_numpy(s)


def select(P, c, n_select, recent, sink, q, bounds=None, scale=None, stride=None):
    if bounds is None:
        bounds, scale = bounds_of(P)
    table, n = P.dev()
    B = len(P.lens)
    ps = torch.full((B, P.hk, stride or P.width), 7.0, device="cuda")
    pages = torch.full((B, P.hk, n_select), -9, dtype=torch.int32, device="cuda")
    c.wkv_paged_select(P.layer, q.cuda(), table, n, bounds.cuda(), scale.cuda(), ps, pages, recent, sink)
    return ps.cpu().numpy(), pages, bounds.numpy(), scale.numpy()


def check_select(P, ps, pages, bounds, scale, n_select, recent, sink, q):
    pages = pages.cpu().numpy()
    q = q.float().numpy()
    for b, n in enumerate(P.lens):
        m = -(-n // P.page)
        for h in range(P.hk):
            code = query_codes(q[b, h * P.G:(h + 1) * P.G])
            pg = P.table[b, :m].long().numpy()
            whole = (bounds[P.layer, pg, h].astype(np.int64) * code).sum((-1, -2))
            want = whole.astype(np.float32) * scale[P.layer, pg, h]
            assert (ps[b, h, :m] == want).all() and (ps[b, h, m:] == 7).all()
            chosen = choose_pages(want, n_select, recent, sink)
            assert pages[b, h].tolist() == chosen + [-1] * (n_select - len(chosen)), f"sequence {b}, kv head {h}"


def go(lens, n_select, recent=1, sink=0, **kw):
    P = Pool(lens, **kw)
    c = P.cache()
    q = P.q
    ps, pages, bounds, scale = select(P, c, n_select, recent, sink, q)
    check_select(P, ps, pages, bounds, scale, n_select, recent, sink, q)
    table, n = P.dev()
    out = torch.full((len(lens), P.hq, P.d), 7.0, dtype=P.tdt, device="cuda")
    lse = torch.full((len(lens), P.hq), 7.0, device="cuda")
    c.wkv_paged_decode_pages(P.layer, q.cuda(), table, n, pages, out, lse)
    assert c.wkv_status() == 0
    host = pages.cpu().numpy()

    def sees(b, h):
        see = np.zeros(P.lens[b], bool)
        for p in host[b, h]:
            if p >= 0:
                see[p * P.page:(p + 1) * P.page] = True
        return see
    P.check(out, lse, sees)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64])
def test_layouts(kind, d, page):
    go([1, 0, 16, 17, 300, 64, 65, 700], 4, 2, 1, kind=kind, d=d, page=page, hq=4, hk=2, seed=page + d)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 4), (8, 4), (8, 2), (8, 1)])
def test_heads(kind, hq, hk):
    go([500, 33, 257], 7, kind=kind, hq=hq, hk=hk, seed=hq + hk, extra_cols=2, layers=2)


@pytest.mark.parametrize("n_select,recent,sink", [(1, 1, 0), (2, 1, 1), (3, 3, 0), (8, 2, 6), (31, 1, 0), (32, 1, 1), (33, 4, 2), (200, 1, 0), (2000, 9, 90)])
def test_counts(n_select, recent, sink):
    go([512, 500, 16, 0, 48], n_select, recent, sink, kind="bf16", hq=4, hk=2, seed=n_select)


@pytest.mark.parametrize("kind", ["bf16", "kv4"])
def test_long_sequences(kind):
    go([9000, 4097], 64, 2, 1, kind=kind, hq=2, hk=1, d=64, page=16, seed=31)
    go([5000], 40, 2, 1, kind=kind, hq=8, hk=2, page=64, seed=32)


@pytest.mark.parametrize("kind", KINDS)
def test_lanes_that_share_the_sms_evenly(kind):
    """A hundred lanes of the same number of chosen pages, and some of less: a few CTAs for each, more than a tile each."""
    go([1900, 1500, 1000, 1100, 0, 16, 1200, 300, 1300, 1000, 1001, 1002, 1400], 60, 2, 1, kind=kind, hq=8, hk=8, d=64, page=16, seed=9)


def test_many_pages_and_ties():
    """Scores held in registers and looked up; whole bits of equal scores, negative and signed zeros among them."""
    for n, n_select in ((2048, 64), (2049, 64), (9999, 5), (9999, 4321)):
        P = Pool([n * 16], hq=2, hk=1, d=64, kind="bf16", spare=0, seed=n)
        rng = np.random.default_rng(n)
        b = rng.integers(-127, 128, (1, P.n_pages, 1, 2, 64)).astype(np.int8)
        s = rng.choice(np.array([0.0, 1e-3, 0.5, 0.5, 2.0], np.float32), (1, P.n_pages, 1))
        b[0, ::3] = b[0, 0]                              # a third of the pages alike
        c = P.cache()
        ps, pages, bounds, scale = select(P, c, n_select, 2, 1, P.q, torch.from_numpy(b), torch.from_numpy(s))
        check_select(P, ps, pages, bounds, scale, n_select, 2, 1, P.q)
        # all scores equal: the lowest pages
        z = torch.zeros_like(torch.from_numpy(s))
        ps, pages, bounds, scale = select(P, c, n_select, 2, 1, P.q, torch.from_numpy(b), z)
        assert pages[0, 0].tolist() == list(range(n_select - 2)) + [n - 2, n - 1]
        assert c.wkv_status() == 0


def test_queries_that_are_zero_tiny_or_not_finite():
    P = Pool([300, 300, 300, 300], hq=4, hk=2, kind="bf16", seed=40)
    q = P.q.clone()
    q[0] = 0
    q[1] = (q[1].float() * 2.0 ** -110).bfloat16()
    c = P.cache()
    ps, pages, b, s = select(P, c, 5, 1, 1, q)
    check_select(P, ps, pages, b, s, 5, 1, 1, q)
    q[2, 0, 0] = float("inf")
    q[3, 0, 0] = float("nan")
    ps, pages, b, s = select(P, c, 5, 1, 1, q)               # any choice, but a choice
    pages = pages.cpu().numpy()
    assert ((pages[2:] >= 0) & (pages[2:] < 19)).all() and (np.diff(pages[2:], axis=-1) > 0).all() and c.wkv_status() == 0


@pytest.mark.parametrize("kind", KINDS)
def test_lists_of_the_callers_own(kind):
    """Any order, gaps, numbers outside of the sequence; places behind the sequence's number of pages are not read."""
    P = Pool([150, 40, 0], hq=4, hk=2, kind=kind, seed=41)
    P.garbage()
    lists = torch.tensor([[[9, -1, 3, 0, 5, 77], [2, 2 ** 30, -5, 1, 8, 4]], [[2, 0, 9, 1, 1, 1], [1, -1, -1, 0, 0, 0]],
                          [[0, 1, 2, 3, 4, 5], [0, 0, 0, 0, 0, 0]]], dtype=torch.int32)
    c = P.cache()
    table, n = P.dev()
    out, lse = torch.zeros(3, 4, 128, dtype=P.tdt, device="cuda"), torch.zeros(3, 4, device="cuda")
    c.wkv_paged_decode_pages(0, P.q.cuda(), table, n, lists.cuda(), out, lse)
    assert c.wkv_status() == 0

    def sees(b, h):
        see = np.zeros(P.lens[b], bool)
        m = -(-P.lens[b] // 16)
        for p in lists[b, h, :min(6, m)].tolist():
            if 0 <= p < m:
                see[p * 16:(p + 1) * 16] = True
        return see
    P.check(out, lse, sees)


@pytest.mark.parametrize("kind", KINDS)
def test_all_pages_chosen_is_decode(kind):
    P = Pool([333, 1, 700], hq=8, hk=2, kind=kind, page=32, seed=42)
    c = P.cache()
    table, n = P.dev()
    lists = torch.arange(P.width, dtype=torch.int32).expand(3, 2, -1).contiguous().cuda()
    out, lse = torch.zeros(3, 8, 128, dtype=P.tdt, device="cuda"), torch.zeros(3, 8, device="cuda")
    c.wkv_paged_decode_pages(0, P.q.cuda(), table, n, lists, out, lse)
    P.check(out, lse, lambda b, h: window_sees(P.lens[b], 0, 0))
    out2, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    c.wkv_paged_decode(0, P.q.cuda(), None, None, table, n, out2, lse=lse2)
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and c.wkv_status() == 0


@pytest.mark.parametrize("kind", KINDS)
def test_bad_page_numbers_are_reported(kind):
    P = Pool([100, 100], hq=4, hk=2, kind=kind, seed=43)
    bounds, scale = bounds_of(P)
    P.table[1, 2] = P.n_pages
    c = P.cache()
    ps, pages, b, s = select(P, c, 7, 1, 0, P.q, bounds, scale)
    assert (ps[1, :, 2] == 0).all() and c.wkv_status() == binding.WKV_ERR_STATE
    table, n = P.dev()
    out, lse = torch.zeros(2, 4, 128, dtype=P.tdt, device="cuda"), torch.zeros(2, 4, device="cuda")
    c.wkv_paged_decode_pages(0, P.q.cuda(), table, n, pages, out, lse)
    assert c.wkv_status() == binding.WKV_ERR_STATE and torch.isfinite(out.float()).all()


def test_captured_choice_follows_lengths_and_repeats():
    P = Pool([900, 300], hq=4, hk=2, kind="bf16", seed=44)
    bounds, scale = (x.cuda() for x in bounds_of(P))
    c = P.cache()
    table, n = P.dev()
    q = P.q.cuda()
    ps = torch.zeros(2, 2, P.width, device="cuda")
    pages = torch.zeros(2, 2, 6, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 4, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.wkv_set_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.wkv_paged_select(0, q, table, n, bounds, scale, ps, pages, 1, 1)
            c.wkv_paged_decode_pages(0, q, table, n, pages, out, lse)
        for lens in ([900, 300], [16, 0], [480, 64], [900, 300]):
            n.copy_(torch.tensor(lens, dtype=torch.int32))
            graph.replay()
            s.synchronize()
            for b, m in enumerate(lens):
                for h in range(2):
                    k = -(-m // 16)
                    want = choose_pages(ps[b, h, :k].cpu().numpy(), 6, 1, 1)
                    assert pages[b, h].tolist() == want + [-1] * (6 - len(want))
    assert c.wkv_status() == 0


@pytest.mark.parametrize("kind", KINDS)
def test_serving_loop(kind):
    """Prompts, then steps: append with rotation and bounds, choose, attend to the choice; against a loop in plain arithmetic.  On 4-bit rows
    the prompts' later chunk attends to the earlier one through spread-out pages."""
    hq, hk, d, page, B, steps = 8, 2, 128, 16, 2, 5
    first, second = [70, 33], [20, 50]
    total = [a + b + steps for a, b in zip(first, second)]
    P = Pool(total, hq=hq, hk=hk, d=d, page=page, kind=kind, seed=50)
    table = P.table.cuda()
    c = P.cache()
    wide = None
    if kind == "kv4":
        W = Pool(total, hq=hq, hk=hk, d=d, page=page, kind="bf16", seed=51)
        wide = W.cache()
        wide_table = W.table.cuda()
    rope = angle_table(max(total), d, 9)
    gr = rope.cuda()
    g = torch.Generator().manual_seed(60)
    gb = torch.zeros(1, P.n_pages, hk, 2, d, dtype=torch.int8, device="cuda")
    gs = torch.zeros(1, P.n_pages, hk, device="cuda")
    kept_q, lens = None, [0, 0]
    for new in (first, second):
        lens = [a + b for a, b in zip(lens, new)]
        start = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        qkv = torch.randn(sum(new), hq + 2 * hk, d, generator=g).to(P.tdt).cuda()
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        qr = torch.empty(sum(new), hq, d, dtype=P.tdt, device="cuda")
        c.wkv_paged_append(0, q, k, v, table, n, start, gr, q_out=qr, page_bounds=gb, page_scale=gs)
        out, lse = torch.empty_like(qr), torch.empty(sum(new), hq, device="cuda")
        if kind == "kv4":
            c.wkv_paged_expand(0, table, n, wide, 0, wide_table)
            wide.wkv_paged_prefill(0, qr, None, None, start, wide_table, n, out, lse=lse)
            assert wide.wkv_status() == 0
        else:
            c.wkv_paged_prefill(0, qr, None, None, start, table, n, out, lse=lse)
        assert c.wkv_status() == 0
        # the last token of each sequence sees all entries: checked as a decode step's row
        rows = [new[0] - 1, sum(new) - 1]
        P.check(out[rows], lse[rows], lambda b, h: np.ones(lens[b], bool), q=qr[rows].cpu(), lens=lens,
                round_p=2.0 ** -8 if kind != "f32" else 0.0)       # prompts on bf16 rows round their weights to bf16
    ps = torch.zeros(B, hk, P.width, device="cuda")
    pages = torch.zeros(B, hk, 4, dtype=torch.int32, device="cuda")
    for t in range(steps):
        lens = [m + 1 for m in lens]
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        qkv = torch.randn(B, hq + 2 * hk, d, generator=g).to(P.tdt).cuda()
        before = qkv.cpu()
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        c.wkv_paged_append(0, q, k, v, table, n, rope=gr, q_out=q, page_bounds=gb, page_scale=gs)      # in place
        c.wkv_paged_select(0, q, table, n, gb, gs, ps, pages, recent=1, sink=1)
        out, lse = torch.empty(B, hq, d, dtype=P.tdt, device="cuda"), torch.empty(B, hq, device="cuda")
        c.wkv_paged_decode_pages(0, q, table, n, pages, out, lse)
        assert c.wkv_status() == 0
        for b in range(B):
            want = rotate32(before[b, :hq].float().numpy(), rope[lens[b] - 1].numpy(), False)
            assert torch.equal(q[b].cpu(), torch.from_numpy(want).to(P.tdt))
        saved, P.lens = P.lens, lens
        host_b, host_s = gb.cpu().numpy(), gs.cpu().numpy()
        P.k_pool, P.v_pool = P.gk.cpu(), P.gv.cpu()
        wb, ws = bounds_of(P)
        used = sorted({int(P.table[b, p]) for b in range(B) for p in range(-(-lens[b] // page))})
        assert (host_b[:, used] == wb.numpy()[:, used]).all() and (host_s[:, used] == ws.numpy()[:, used]).all()
        full = np.full((B, hk, P.width), 7.0, np.float32)
        for b in range(B):
            m = -(-lens[b] // page)
            full[b, :, :m] = ps[b, :, :m].cpu().numpy()
        check_select(P, full, pages, host_b, host_s, 4, 1, 1, q.cpu())
        host = pages.cpu().numpy()

        def sees(b, h):
            see = np.zeros(lens[b], bool)
            for p in host[b, h]:
                if p >= 0:
                    see[p * page:(p + 1) * page] = True
            return see
        P.check(out, lse, sees, q=q.cpu(), lens=lens)
        P.lens = saved
