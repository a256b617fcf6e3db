"""4-bit rows, page bounds and chosen pages where values, page numbers or sizes are at an edge."""
import numpy as np
import pytest
import torch

from paged_rows_util import Pool, attend, window_sees
from paper_2503_01330_b200 import binding

pytestmark = pytest.mark.gpu


def decode(P, c, q=None, window=0, sink=0, lists=None):
    """Output, log-sum and status of a decode step, over all pages or over `lists` [B, hk, n]."""
    table, n = P.dev()
    q = (P.q if q is None else q).cuda()
    out = torch.full((len(P.lens), P.hq, P.d), 7.0, dtype=P.tdt, device="cuda")
    lse = torch.full((len(P.lens), P.hq), 7.0, device="cuda")
    if lists is None:
        c.wkv_paged_decode(P.layer, q, None, None, table, n, out, window, sink, None, lse)
    else:
        c.wkv_paged_decode_pages(P.layer, q, table, n, lists.cuda(), out, lse)
    return out, lse, c.wkv_status()


def shuffled_lists(P, seed, every=True):
    """Lists of all pages (or of every other one) of each sequence in an order of their own per kv head."""
    rng = np.random.default_rng(seed)
    n = P.width if every else max(1, P.width // 2)
    lists = torch.full((len(P.lens), P.hk, n), -1, dtype=torch.int32)
    for b, m in enumerate(P.lens):
        pages = -(-m // P.page)
        for h in range(P.hk):
            pick = rng.permutation(pages)[:n]
            lists[b, h, :len(pick)] = torch.from_numpy(pick.astype(np.int32))
    return lists


def list_sees(P, lists):
    def sees(b, h):
        see = np.zeros(P.lens[b], bool)
        for p in lists[b, h].tolist():
            if p >= 0:
                see[p * P.page:(p + 1) * P.page] = True
        return see
    return sees


# ---- page numbers that are none

@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("hq,hk,d", [(2, 2, 128), (8, 2, 64)])
@pytest.mark.parametrize("column", [0, 1])
def test_bad_page_counts_as_zeros_wherever_it_lies(page, hq, hk, d, column):
    """The sequences' first page has entry 0; halves of tiles, windows that reach into it, lists that have it anywhere.  What the
    block's memory holds from before (large values) must not show."""
    lens = [100, 64 + 47, 700, 63]
    loud = Pool([2000] * 4, hq=hq, hk=hk, d=d, page=page, spread=1000.0, seed=3)
    P = Pool(lens, hq=hq, hk=hk, d=d, page=page, seed=page + d)
    good = P.table.clone()
    P.table[0, column], P.table[2, column] = P.n_pages + 1, -1
    if column * page + page < 63:
        P.table[3, column] = -5
    bad = P.table.clone()
    lc, c = loud.cache(), P.cache()
    lists = shuffled_lists(P, page)
    for window, sink, over in ((0, 0, None), (690, 3, None), (95, 0, None), (0, 0, lists)):
        decode(loud, lc)
        P.table = bad
        out, lse, status = decode(P, c, None, window, sink, over)
        assert status == binding.WKV_ERR_STATE
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        P.table = good
        for b, n in enumerate(lens):
            hole = np.zeros(n, bool)
            if not torch.equal(bad[b], good[b]):
                hole[column * page:column * page + page] = True
            for h in range(hk):
                K, V, Ka, Va, sm = P.rows(b, h)
                for x in (K, V, Ka, Va):
                    x[hole] = 0
                for r in range(h * P.G, (h + 1) * P.G):
                    w, z, bo, bz = attend(P.q[b, r].double().numpy(), K, V, window_sees(n, window, sink), P.scale, P.half, Ka, Va, sm)
                    assert (np.abs(out[b, r] - w) <= bo).all() and abs(lse[b, r] - z) <= bz, (b, r, window, sink)


# ---- queries of any finite size

@pytest.mark.parametrize("hq,hk", [(2, 2), (4, 2), (8, 2), (8, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_and_softmax_scale_by_inverse_powers_of_two(hq, hk, d):
    """Queries times 2^n and the softmax scale times 2^-n are the same attention, bit for bit: the codes' products take a power of two of the
    query into the scale."""
    scale = float(np.float32(1 / np.sqrt(d)))
    P = Pool([300, 17, 2000], hq=hq, hk=hk, d=d, page=32, seed=d + hq)
    P.q = (P.q.float().sign() * (P.q.float().abs() + 2.0 ** -6)).bfloat16()        # no channel so small that 2^-96 of it has fewer bits
    want = decode(P, P.cache(scale=scale))
    assert want[2] == 0
    P.check(want[0], want[1], lambda b, h: window_sees(P.lens[b], 0, 0))
    for n in (60, 114, 119, 121, 123, -60, -96):
        q = (P.q.float() * 2.0 ** n).bfloat16()
        assert torch.isfinite(q.float()).all() and torch.equal(q.double() * 2.0 ** -n, P.q.double())
        got = decode(P, P.cache(scale=scale * 2.0 ** -n), q)
        assert got[2] == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), n


# ---- queries that are no numbers

def check_nan_queries(kind, hq, hk, page=16):
    """The heads that have a NaN, or logits without a largest number, get NaN for output and log-sum, whole or cut into pieces; the
    others and padded rows what they got without it."""
    P = Pool([5000, 40, 0, 300], hq=hq, hk=hk, kind=kind, page=page, seed=5)
    c = P.cache()
    lists = shuffled_lists(P, 1, False)
    q = P.q.clone()
    q[0, 0, 3] = q[1, hq - 1, 70] = q[2, 0, 0] = float("nan")
    q[3, 1 % hq] = float("inf")
    hit = torch.zeros(4, hq, dtype=torch.bool)
    hit[0, 0] = hit[1, hq - 1] = hit[3, 1 % hq] = True
    for over in (None, lists):
        out, lse, status = decode(P, c, None, lists=over)
        nan_out, nan_lse, nan_status = decode(P, c, q, lists=over)
        assert status == 0 and nan_status == 0
        assert torch.isnan(nan_out.float().cpu()[hit]).all() and torch.isnan(nan_lse.cpu()[hit]).all()
        assert torch.equal(nan_out.cpu()[~hit], out.cpu()[~hit]) and torch.equal(nan_lse.cpu()[~hit], lse.cpu()[~hit])
        assert (out[2] == 0).all() and (lse[2] == -float("inf")).all()


@pytest.mark.parametrize("hq,hk", [(2, 2), (4, 2), (8, 2), (8, 1)])
def test_queries_with_a_nan_show_in_log_sums_of_4_bit_rows(hq, hk):
    check_nan_queries("kv4", hq, hk)
    check_nan_queries("kv4", hq, hk, 64)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk", [(2, 2), (4, 2), (8, 2), (8, 1)])
def test_queries_with_a_nan_show_in_log_sums(kind, hq, hk):
    check_nan_queries(kind, hq, hk)


# ---- keys that are not finite

@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_pages_with_an_infinite_key_are_chosen_first(kind, d):
    """Their scale is infinite and their bounds lie outwards, so that their score is +infinity or no number, which both rank above all."""
    P = Pool([600, 77], hq=4, hk=2, d=d, kind=kind, seed=d)
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(677, 2, d, generator=g).to(P.tdt) for _ in range(2))
    up, down, both = [(0, 33, 1, 5)], [(0, 100, 0, d - 1), (1, 20, 1, 0)], [(0, 330, 1, 17), (0, 331, 1, 17)]      # sequence, entry, head, channel
    for (b, i, h, ch), x in [*((e, np.inf) for e in up), *((e, -np.inf) for e in down), (both[0], np.inf), (both[1], -np.inf)]:
        k[600 * b + i, h, ch] = x
    c = P.cache()
    table, n = P.dev()
    gb = torch.zeros(1, P.n_pages, 2, 2, d, dtype=torch.int8, device="cuda")
    gs = torch.zeros(1, P.n_pages, 2, device="cuda")
    start = torch.tensor([0, 600, 677], dtype=torch.int32, device="cuda")
    c.wkv_paged_append(0, None, k.cuda(), v.cuda(), table, n, start, page_bounds=gb, page_scale=gs)
    bounds, scale = gb.cpu()[0], gs.cpu()[0]
    loud = {(b, i // 16, h) for b, i, h, _ in up + down + both}
    for b in range(2):
        for p in range(-(-P.lens[b] // 16)):
            for h in range(2):
                assert torch.isinf(scale[int(P.table[b, p]), h]) == ((b, p, h) in loud)
    for b, i, h, ch in up + both[:1]:
        assert bounds[int(P.table[b, i // 16]), h, 0, ch] == 127
    for b, i, h, ch in down + both[:1]:
        assert bounds[int(P.table[b, i // 16]), h, 1, ch] == -127
    for seed in range(3):
        q = torch.randn(2, 4, d, generator=g).to(P.tdt)
        if seed == 2:
            q[:] = 0
        ps, pages = torch.zeros(2, 2, P.width, device="cuda"), torch.zeros(2, 2, 4, dtype=torch.int32, device="cuda")
        c.wkv_paged_select(0, q.cuda(), table, n, gb, gs, ps, pages, recent=1)
        for b, p, h in loud:
            assert not ps[b, h, p] < float("inf") and p in pages[b, h].tolist()
    assert c.wkv_status() == 0


# ---- value scales far apart

@pytest.mark.parametrize("hq,hk,d,page", [(2, 2, 128, 16), (4, 2, 64, 64), (8, 2, 128, 32), (8, 1, 128, 64)])
@pytest.mark.parametrize("n", [40, 600])
@pytest.mark.parametrize("small", [2.0 ** -11, 2.0 ** -13, 2.0 ** -15])
def test_large_values_without_weight_leave_small_ones_their_bits(hq, hk, d, page, n, small):
    """Entry 0 has value scales at the format's upper end and next to no weight.  A weight times a scale, fp16 times powers of two that bring
    the largest scale S to [2^5, 2^6) and weights of 1 to 2^9, is off by 2^-25 at most where it is below fp16's normal range: 2^-39 S, or by
    all of it; the weight itself by 2^-25 2^-9 of the largest at most.  The other roundings are relative."""
    from paged_rows_util import pack_chunks
    P = Pool([n], hq=hq, hk=hk, d=d, page=page, seed=n + hq)
    g = torch.Generator().manual_seed(n)
    shape = (1, P.n_pages, hk, page, d)
    K, V = torch.randn(shape, generator=g), torch.randn(shape, generator=g) * small
    q = torch.randn(1, hq, d, generator=g) * 2
    K[..., 0], q[..., 0] = 0.0, 16.0
    first = int(P.table[0, 0])
    K[0, first, :, 0, 0] = -120.0
    V[0, first, :, 0] = 6e4 * torch.randn(hk, d, generator=g).sign()
    P.k_pool, P.v_pool = (torch.from_numpy(pack_chunks(w, x.bfloat16().float().numpy())[0]) for w, x in (("k", K), ("v", V)))
    q = q.bfloat16()
    out, lse, status = decode(P, P.cache(), q)
    assert status == 0
    out = out.double().cpu().numpy()
    for h in range(hk):
        K64, V64, Ka, Va, _ = P.rows(0, h)
        for r in range(h * P.G, (h + 1) * P.G):
            x = q[0, r].double().numpy()
            w, z, bo, _ = attend(x, K64, V64, np.ones(n, bool), P.scale, P.half, Ka, Va, 0.0)
            p = np.exp(K64 @ x * P.scale - z)
            top = p.max()
            assert p[0] < 1e-30
            step = np.abs(Va)                                                  # s (n + z), 0 .. 30 s
            lost = np.minimum(p[:, None] * step, 15 * 2.0 ** -39 * 4096.0 * 2 * top)[1:].sum(0) + 2.0 ** -34 * top * step[1:].sum(0)
            e = np.abs(out[0, r] - w) / (bo + lost)
            assert (e <= 1).all(), f"head {r}: {e.max():.3g} of the bound"


# ---- choosing pages

@pytest.mark.parametrize("kind", ["bf16", "f32", "kv4"])
@pytest.mark.parametrize("hq,hk", [(8, 1), (4, 2)])
def test_choice_does_not_depend_on_a_factor_of_the_query(kind, hq, hk):
    """Scores are in steps of the query's largest channel sum: whatever its size, the sum over the heads beyond fp32 included."""
    P = Pool([1000, 90], hq=hq, hk=hk, kind=kind, seed=8)
    g = torch.Generator().manual_seed(1)
    bounds = torch.randint(-127, 128, (1, P.n_pages, hk, 2, P.d), generator=g, dtype=torch.int8).cuda()
    scale = torch.rand(1, P.n_pages, hk, generator=g).cuda()
    base = (P.q.float().abs().clamp(2.0 ** -3, 1.75) * P.q.float().sign()).to(P.tdt)
    base[0, :, 5] = 1.75                                     # the sum over the heads: 1.75 * 8
    c = P.cache()
    table, n = P.dev()
    got = []
    for f in (1.0, 2.0 ** 100, 2.0 ** 124, 2.0 ** 127, 2.0 ** -80):
        q = (base.double() * f).to(P.tdt)
        assert torch.equal(q.double(), base.double() * f)
        ps, pages = torch.zeros(2, hk, P.width, device="cuda"), torch.zeros(2, hk, 9, dtype=torch.int32, device="cuda")
        c.wkv_paged_select(0, q.cuda(), table, n, bounds, scale, ps, pages, recent=1)
        assert c.wkv_status() == 0
        got.append((ps, pages))
    for ps, pages in got[1:]:
        assert torch.equal(ps, got[0][0]) and torch.equal(pages, got[0][1])


# ---- sizes

def test_spreading_out_refuses_what_a_launch_cannot_hold():
    """batch * n_kv_heads * (table_width * page_size / 64) CTAs: at most 2^31 - 1."""
    heads, width, batch = 32, 1 << 18, 1024
    args = dict(n_layers=1, n_pages=1, page_size=64, n_q_heads=heads, n_kv_heads=heads, head_dim=64, max_batch=batch, max_pages=width)
    a, b = binding.PagedCache(dtype=binding.WKV_KV4, **args), binding.PagedCache(dtype=binding.WKV_BF16, **{**args, "max_batch": 1})
    one = torch.zeros(batch, dtype=torch.int32, device="cuda")
    for n in (256, batch):                                   # 2^31 CTAs, 2^33 (nothing is read: the call ends on the host)
        before = a.wkv_launch_count()
        rc = binding.lib().wkv_paged_expand(a._h, 0, n, one.data_ptr(), width, one.data_ptr(), b._h, 0, one.data_ptr(), 1)
        assert rc == binding.WKV_ERR_INVALID and "too large" in binding.lib().wkv_paged_last_error(a._h).decode()
        assert a.wkv_launch_count() == before and a.wkv_status() == 0


# ---- one entry with nearly all weight

@pytest.mark.parametrize("hq,hk,d,page", [(2, 2, 128, 16), (2, 2, 64, 32), (4, 2, 128, 64), (4, 2, 64, 16), (8, 2, 128, 32), (8, 2, 64, 64), (8, 1, 128, 16)])
def test_small_weights_beside_one_large_one(hq, hk, d, page):
    """The entry with nearly all weight holds zeros (codes equal to the zero point, not 0), so that the others' weights, 2^-8 to 2^-24 of it,
    are all there is: sums of codes and of zero points must hold both to fp32's bits."""
    from paged_rows_util import pack_chunks
    gaps = list(range(8, 25, 2))
    lens = [16, 40, 300] * 3
    P = Pool(lens, hq=hq, hk=hk, d=d, page=page, seed=d + hq)
    g = torch.Generator().manual_seed(hq)
    shape = (1, P.n_pages, hk, page, d)
    K, V = torch.zeros(shape), torch.randn(shape, generator=g)
    q = torch.zeros(len(lens), hq, d)
    for b, (n, gap) in enumerate(zip(lens, gaps)):
        at = (5 * b + 3) % n
        pg, row = int(P.table[b, at // page]), at % page
        K[0, pg, :, row, 0] = 64.0
        V[0, pg, :, row] = 0.0
        V[0, pg, :, row, 3::32], V[0, pg, :, row, 20::32] = 2.0, -2.0
        q[b, :, 0] = gap * np.log(2.0) / (64.0 * P.scale)
    P.k_pool, P.v_pool = (torch.from_numpy(pack_chunks(w, x.bfloat16().float().numpy())[0]) for w, x in (("k", K), ("v", V)))
    P.q = q.bfloat16()
    c = P.cache()
    for lists in (None, shuffled_lists(P, 3)):
        out, lse, status = decode(P, c, lists=lists)
        assert status == 0
        P.check(out, lse, lambda b, h: np.ones(P.lens[b], bool))
