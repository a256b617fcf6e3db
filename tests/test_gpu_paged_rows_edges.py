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
