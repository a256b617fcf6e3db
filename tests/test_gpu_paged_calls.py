"""Paged calls as programs make them: streams, status, shared and released pages, bad pages, scales, many items a CTA.  Results
are held against the definition of tests/paged_util.py."""
import pytest
import torch

from paged_util import Case
from paper_2503_01330_b200 import binding

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- arguments

@pytest.mark.parametrize("prefill", [False, True])
@pytest.mark.parametrize("which", ["q", "k", "v", "kv"])
def test_rows_broadcast_over_the_batch_are_refused(prefill, which):
    c = Case(lens=[40, 20, 33], new=[1, 1, 1], page=16, prefill=prefill)
    cache = c.cache()
    rows = dict(zip("qkv", c.rows()))
    for x in which:
        rows[x] = rows[x][:1].expand_as(rows[x])
    i32 = dict(dtype=torch.int32, device="cuda")
    table, lens, out = c.table.cuda(), torch.tensor(c.lens, **i32), torch.empty(3, 4, 64, dtype=c.tdt, device="cuda")
    with pytest.raises(binding.WkvError) as e:
        if prefill:
            cache.wkv_paged_prefill(0, **rows, q_start=torch.tensor([0, 1, 2, 3], **i32), block_table=table, seq_lens=lens, out=out)
        else:
            cache.wkv_paged_decode(0, **rows, block_table=table, seq_lens=lens, out=out)
    assert e.value.code == binding.WKV_ERR_INVALID and cache.wkv_launch_count() == 0
    cache.close()


# ---------------------------------------------------------------- streams, status

@pytest.mark.parametrize("raw", [False, True])
def test_pools_of_a_dropped_cache_wait_for_its_stream(raw):
    """Pools that the cache made itself go back to torch's allocator with it, but not to a new tensor while the stream that the
    cache ran on still has work."""
    cache = binding.PagedCache(1, 1000, 16, 4, 2, 64, 2, 4)
    nbytes, addresses = cache.k_pool.nbytes, {cache.k_pool.data_ptr(), cache.v_pool.data_ptr()}
    q, k = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    table, lens, out = (torch.zeros(*s, dtype=t, device="cuda") for s, t in (((2, 4), torch.int32), ((2,), torch.int32), ((2, 4, 64), torch.bfloat16)))
    table[1] += 1
    lens += 1
    side = torch.cuda.Stream()
    cache.wkv_set_stream(side.cuda_stream if raw else side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)
    cache.wkv_paged_decode(0, q, k, k, table, lens, out)
    cache.close()
    del cache
    later = [torch.empty(nbytes, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert not side.query()
    assert not addresses & {x.data_ptr() for x in later}
    torch.cuda.synchronize()


def test_status_on_a_side_stream_keeps_the_next_report():
    """wkv_paged_status clears what it reports in the order of the handle's stream, so a bad call right behind it is reported too,
    also on a stream that does not wait for the default one."""
    c = Case(lens=[40, 20], new=[1, 1], page=16)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache = c.cache()
        q, k, v = c.rows()
        table, lens, out = c.table.cuda(), torch.tensor(c.lens, dtype=torch.int32, device="cuda"), torch.empty(2, 4, 64, dtype=c.tdt, device="cuda")
        bad = table.clone()
        bad[0, 1] = -1
        for i in range(200):
            cache.wkv_paged_decode(0, q, k, v, bad, lens, out)
            assert cache.wkv_status() == binding.WKV_ERR_STATE, i
        cache.wkv_paged_decode(0, q, k, v, table, lens, out)
        assert cache.wkv_status() == 0
        side.synchronize()
    cache.close()


def test_a_wait_that_gives_up_is_reported_and_the_handle_goes_on():
    """The self-test's waits, of 400 polls, are for barriers that nothing arrives at."""
    for prefill in (False, True):
        c = Case(lens=[300, 20], new=[200, 9] if prefill else [1, 1], page=16, prefill=prefill, scores=True)
        cache = c.cache()
        cache.wkv_selftest_wait_timeout()                  # loads the kernel
        assert cache.wkv_status() == binding.WKV_ERR_TIMEOUT and cache.wkv_status() == 0
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        cache.wkv_selftest_wait_timeout()
        end.record()
        assert cache.wkv_status() == binding.WKV_ERR_TIMEOUT and cache.wkv_status() == 0
        ms = start.elapsed_time(end)
        assert ms < 500, f"{ms:.3f} ms"
        c.check(*c.run(cache), "afterwards")
        cache.close()


# ---------------------------------------------------------------- released and bad pages

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefill,scores", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("page,window,sink", [(16, 100, 4), (16, 1, 0), (32, 200, 33), (64, 64, 0)])
def test_pages_that_nobody_sees_may_be_released(dtype, prefill, scores, page, window, sink):
    """A window's cache gives back the pages behind it: any number may stand in the table there, with and without weights."""
    new = [300, 140, 3, 33] if prefill else [1] * 4
    c = Case(lens=[300, 1513, 600, 33], new=new, hq=8, hk=2, d=64, dtype=dtype, page=page, window=window, sink=sink, scores=scores,
             seed=window, prefill=prefill)
    table, released = c.table, c.table.clone()
    for b, (n, t) in enumerate(zip(c.lens, c.new)):
        for p in range(-(-n // page)):
            if p * page >= sink and (p + 1) * page <= n - t - window + 1:
                released[b, p] = (-1, c.n_pages, 2 ** 31 - 1)[p % 3]
    assert (released != table).sum() > 10
    c.table = released
    result = c.run()                                       # asserts the status
    c.table = table
    c.check(*result, "released")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_evict_from_and_to_bad_pages(dtype):
    """An entry of a bad source page counts as zeros: its place in the destination holds zeros, and not what was there.  What goes
    to a bad destination page goes nowhere."""
    page, hk, d, budget = 16, 2, 64, 40
    c = Case(lens=[100, 70], new=[1, 1], hq=hk, hk=hk, d=d, dtype=dtype, page=page, append=False, scores=True, spare=8, seed=21)
    cache = c.cache()
    dst = c.free_pages[:6].reshape(2, 3).clone()
    good_dst = dst.clone()
    table = c.table.clone()
    table[0, 0], table[0, 5] = -1, c.n_pages               # sequence 0: two bad source pages
    dst[1, 1] = 2 ** 31 - 1                                # sequence 1: a bad destination page
    new_lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    kept = torch.full((2, hk, budget), -1, dtype=torch.int32, device="cuda")
    lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    cache.wkv_paged_evict(0, table.cuda(), dst.cuda(), lens, new_lens, budget, 6, 3, scores=c.scores.cuda(), kept=kept)
    assert cache.wkv_status() == binding.WKV_ERR_STATE and cache.wkv_status() == 0
    assert new_lens.tolist() == [budget, budget]
    kept = kept.cpu()
    want_k, want_v = c.k_pool.clone(), c.v_pool.clone()
    zeroed = 0
    for b in range(2):
        for h in range(hk):
            for at, i in enumerate(kept[b, h].tolist()):
                if b == 1 and at // page == 1:
                    continue
                bad = b == 0 and i // page in (0, 5)
                zeroed += bad
                pg = int(good_dst[b, at // page])
                want_k[0, pg, h, at % page] = torch.zeros(d) if bad else c.K[b][i, h]
                want_v[0, pg, h, at % page] = torch.zeros(d) if bad else c.V[b][i, h]
    assert zeroed >= 4
    as_int = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(c.gk.cpu().view(as_int), want_k.view(as_int)) and torch.equal(c.gv.cpu().view(as_int), want_v.view(as_int))
    cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefill", [False, True])
@pytest.mark.parametrize("window,sink", [(0, 0), (30, 4)])
def test_entries_of_bad_pages_count_as_zeros(dtype, prefill, window, sink):
    """Outputs, log-sums and weights of a sequence with bad pages are those of a cache that holds zeros there, the call's own new
    entries among them; nothing else is touched."""
    new = [60, 30, 20] if prefill else [1, 1, 1]
    c = Case(lens=[100, 90, 80], new=new, hq=4, hk=2, d=64, dtype=dtype, page=16, scores=True, seed=22, prefill=prefill, window=window,
             sink=sink)
    cache = c.cache()
    q, k, v = c.rows()
    table = c.table.clone()
    bad = {0: [4, 6], 1: [1, 5], 2: [0, 3]} if prefill else {0: [6], 1: [1, 5], 2: [0, 3]}
    for b, pages in bad.items():
        for p in pages:
            table[b, p] = (-1, c.n_pages, 2 ** 31 - 1, -2 ** 31)[(b + p) % 4]
            c.K[b][p * 16:(p + 1) * 16] = 0
            c.V[b][p * 16:(p + 1) * 16] = 0
    out, lse = torch.full((c.T, 4, 64), 7.0, dtype=c.tdt, device="cuda"), torch.full((c.T, 4), 7.0, device="cuda")
    scores, lens = c.scores.cuda(), torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    if prefill:
        cache.wkv_paged_prefill(0, q, k, v, torch.tensor(c.starts, dtype=torch.int32, device="cuda"), table.cuda(), lens, out, window, sink, scores, lse)
    else:
        cache.wkv_paged_decode(0, q, k, v, table.cuda(), lens, out, window, sink, scores, lse)
    assert cache.wkv_status() == binding.WKV_ERR_STATE
    rows_k, rows_v = c.K, c.V
    was_k, was_v = c.k_pool, c.v_pool
    # the bad pages' rows stay as they were, whatever the definition counts there
    want_k, want_v = was_k.clone(), was_v.clone()
    for b, n in enumerate(c.lens):
        for i in range(n - c.new[b], n):
            if i // 16 not in bad[b]:
                pg = int(c.table[b, i // 16])
                want_k[0, pg, :, i % 16], want_v[0, pg, :, i % 16] = rows_k[b][i], rows_v[b][i]
    as_int = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(c.gk.cpu().view(as_int), want_k.view(as_int)) and torch.equal(c.gv.cpu().view(as_int), want_v.view(as_int))
    c.check_pool = lambda what="": None
    c.check(out, lse, scores, "bad pages")
    cache.close()


# ---------------------------------------------------------------- sizes

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("total_q", [5, 40000])
def test_prompt_call_without_tokens(dtype, total_q):
    """A captured call's batch may be all padding: rows of no sequence are left alone, whether the call is one that is cut or not,
    and the next call on the handle is right."""
    c = Case(lens=[300, 40], new=[200, 40], hq=4, hk=2, d=64, dtype=dtype, page=16, scores=True, seed=51)
    cache = c.cache()
    q, k, v = (torch.zeros(total_q, h, 64, dtype=c.tdt, device="cuda") for h in (4, 2, 2))
    out, lse, scores = torch.full_like(q, 7.0), torch.full((total_q, 4), 7.0, device="cuda"), c.scores.cuda()
    none, lens = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    for n in (lens, torch.zeros_like(lens)):
        cache.wkv_paged_prefill(0, q, k, v, none, c.table.cuda(), n, out, scores=scores, lse=lse)
        assert cache.wkv_status() == 0
        assert (out == 7).all() and (lse == 7).all() and torch.equal(scores.cpu(), c.scores)
    c.check(*c.run(cache), "afterwards")
    cache.close()
