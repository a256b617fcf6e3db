"""Decode attention on rows in 4 bits against 64-bit arithmetic, at the sizes and masks where it can go wrong."""
import numpy as np
import pytest
import torch

from paged_rows_util import Pool, window_sees
from paper_2503_01330_b200 import binding

pytestmark = pytest.mark.gpu


def run(P, cache=None, window=0, sink=0, k=None, v=None, lens=None, q=None):
    c = cache or P.cache()
    table, n = P.dev()
    if lens is not None:
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q = (P.q if q is None else q).cuda()
    out = torch.full((len(P.lens), P.hq, P.d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((len(P.lens), P.hq), 7.0, device="cuda")
    c.wkv_paged_decode(P.layer, q, k, v, table, n, out, window, sink, None, lse)
    status = c.wkv_status()
    if cache is None:
        c.close()
    return out, lse, status


def go(lens, window=0, sink=0, what="", **kw):
    P = Pool(lens, **kw)
    P.garbage()
    out, lse, status = run(P, window=window, sink=sink)
    assert status == 0
    P.check(out, lse, lambda b, h: window_sees(P.lens[b], window, sink), what)
    assert torch.equal(P.gk.cpu(), P.k_pool) and torch.equal(P.gv.cpu(), P.v_pool)


@pytest.mark.parametrize("hq,hk", [(2, 2), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64])
def test_layouts(hq, hk, d, page):
    go([1, 15, 16, 17, 127, 128, 129, 0, 300], hq=hq, hk=hk, d=d, page=page, seed=page + d)


@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (5, 3), (16, 16), (100, 4), (128, 33), (1000, 4)])
@pytest.mark.parametrize("page", [16, 64])
def test_windows_and_sinks(window, sink, page):
    go([1, 5, 16, 100, 129, 260, 513, 0], window=window, sink=sink, page=page, seed=window + page)


def test_long_lanes_in_pieces():
    go([5000, 1, 777], hq=8, hk=2, page=32, seed=3)
    go([4100], hq=2, hk=2, d=64, page=16, seed=4)
    go([3333, 4444, 1234, 0, 2222], hq=4, hk=4, page=64, seed=5)


@pytest.mark.parametrize("lens", [[2368] * 16, [2400, 2304, 1, 0, 130, 2399, 2305, 257, 2300, 2300, 2300, 2300, 2300, 2300, 2300, 2300], [1500] * 9])
def test_lanes_of_nearly_equal_length(lens):
    """A few CTAs for each lane, of which short lanes use some; more than one tile each."""
    go(lens, hq=16, hk=8, d=64, page=32, seed=7)


def test_many_short_lanes_and_layers():
    go([(i * 37) % 90 for i in range(70)], hq=8, hk=4, layers=2, extra_cols=3, seed=6)


@pytest.mark.parametrize("spread", [2.0 ** -12, 1e-3, 300.0])
def test_magnitudes(spread):
    """Scales at the border of the format and fp16-subnormal weights."""
    go([200, 31], hq=4, hk=2, spread=spread, seed=7)


def test_queries_of_any_size():
    P = Pool([150, 64], hq=4, hk=2, seed=8)
    for f in (2.0 ** -60, 2.0 ** -8, 2.0 ** 4):
        q = (P.q.float() * f).bfloat16()
        out, lse, status = run(P, q=q)
        assert status == 0
        P.check(out, lse, lambda b, h: window_sees(P.lens[b], 0, 0), f"q * {f}", q=q)
    # one loud channel, the others 2^-20 of it
    q = P.q.clone()
    q[..., 5] = 2.0 ** 10
    q[..., 6:] = (q[..., 6:].float() * 2.0 ** -10).bfloat16()
    out, lse, status = run(P, q=q)
    P.check(out, lse, lambda b, h: window_sees(P.lens[b], 0, 0), "loud channel", q=q)


def test_value_scales_that_grow_along_the_cache():
    """The weights' power of two follows the largest scale seen: values grow by 2^24 over the entries, and shrink again."""
    P = Pool([400], hq=2, hk=1, seed=9)
    from paged_rows_util import pack_chunks
    g = torch.Generator().manual_seed(5)
    x = torch.randn(1, P.n_pages, 1, P.page, P.d, generator=g)
    order = {int(p): i for i, p in enumerate(P.table[0, :25])}
    for pg in range(P.n_pages):
        i = order.get(pg, 0)
        x[0, pg] *= 2.0 ** (min(i, 24 - i) * 2 - 12)
    P.v_pool = torch.from_numpy(pack_chunks("v", x.bfloat16().float().numpy())[0])
    out, lse, status = run(P)
    assert status == 0
    P.check(out, lse, lambda b, h: window_sees(400, 0, 0))


def test_logits_that_tower():
    P = Pool([300], hq=4, hk=2, seed=10)
    q = (P.q.float() * 30).bfloat16()
    out, lse, status = run(P, q=q)
    P.check(out, lse, lambda b, h: window_sees(300, 0, 0), q=q)


def test_new_entries_are_stored_in_4_bits_first():
    """k and v given: the same pool and the same outputs, bit for bit, as an append followed by a decode without them."""
    lens = [1, 16, 17, 40, 0, 64]
    P = Pool(lens, hq=8, hk=2, seed=11)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(len(lens), 2, 128, generator=g).bfloat16().cuda() for _ in range(2))
    a, la, st = run(P, k=k, v=v)
    assert st == 0
    gk, gv = P.gk.clone(), P.gv.clone()
    P.check(a, la, lambda b, h: window_sees(P.lens[b], 0, 0))
    c = P.cache()
    table, n = P.dev()
    c.wkv_paged_append(0, None, k, v, table, n)
    b, lb, st = run(P, cache=c)
    assert st == 0 and torch.equal(a, b) and torch.equal(la, lb) and torch.equal(P.gk, gk) and torch.equal(P.gv, gv)
    assert not torch.equal(gk.cpu(), P.k_pool)


def test_bad_pages_count_as_zeros():
    lens = [100, 40]
    P = Pool(lens, hq=4, hk=2, seed=12)
    P.table[0, 2] = P.n_pages
    P.table[1, 1] = -1
    out, lse, status = run(P)
    assert status == binding.WKV_ERR_STATE
    out, lse = out.double().cpu(), lse.double().cpu()
    for b, lo in ((0, 32), (1, 16)):
        hole = np.zeros(lens[b], bool)
        hole[lo:lo + 16] = True
        table, P.table = P.table, P.table.clone()
        P.table[b, lo // 16] = int(P.free_pages[0])
        for h in range(2):
            K, V, Ka, Va, sm = P.rows(b, h)
            for x in (K, V, Ka, Va):
                x[hole] = 0
            from paged_rows_util import attend
            for r in (2 * h, 2 * h + 1):
                w, z, bo, bz = attend(P.q[b, r].double().numpy(), K, V, np.ones(lens[b], bool), P.scale, P.half, Ka, Va, sm)
                assert (np.abs(out[b, r].numpy() - w) <= bo).all() and abs(float(lse[b, r]) - z) <= bz
        P.table = table


def test_lengths_out_of_range_are_clamped():
    P = Pool([32, 32], hq=2, hk=2, seed=13)
    out, lse, status = run(P, lens=[100, -5])
    assert status == binding.WKV_ERR_STATE
    P.check(out, lse, lambda b, h: np.ones(32, bool), lens=[32, 0])


def test_released_pages_behind_the_window():
    P = Pool([200], hq=4, hk=2, seed=14)
    P.table[0, 1:8] = -1
    out, lse, status = run(P, window=60, sink=7)
    assert status == 0
    P.table[0, 1:8] = int(P.free_pages[0])
    P.check(out, lse, lambda b, h: window_sees(200, 60, 7))


def test_repeats_bit_for_bit_and_strided_queries():
    P = Pool([3000, 517, 90], hq=8, hk=2, seed=15)
    c = P.cache()
    a = run(P, cache=c)
    for _ in range(3):
        b = run(P, cache=c)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    wide = torch.randn(3, 20, 128).bfloat16().cuda()
    wide[:, 5:13] = P.q.cuda()
    table, n = P.dev()
    out, lse = torch.empty_like(a[0]), torch.empty_like(a[1])
    c.wkv_paged_decode(0, wide[:, 5:13], None, None, table, n, out, lse=lse)
    assert c.wkv_status() == 0 and torch.equal(out, a[0]) and torch.equal(lse, a[1])


def test_captured_step_follows_lengths_and_tables():
    P = Pool([700, 300], hq=4, hk=2, seed=16)
    c = P.cache()
    table, n = P.dev()
    n.fill_(1)
    q = P.q.cuda()
    out, lse = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 4, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.wkv_set_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.wkv_paged_decode(0, q, None, None, table, n, out, lse=lse)
        for lens in ([700, 300], [1, 0], [129, 128]):
            n.copy_(torch.tensor(lens, dtype=torch.int32))
            graph.replay()
            s.synchronize()
            P.check(out, lse, lambda b, h: np.ones(lens[b], bool), lens=lens)
    assert c.wkv_status() == 0
