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


MANY = [
    # one kv head per query head; the last block of a sequence has one row tile (1 and 76 rows), or is full
    dict(hq=32, hk=32, d=64, page=16, lens=[1537, 2300, 128, 1740, 40], new=[1537, 1100, 128, 1024, 0]),
    # grouped heads under a window with sinks: row tiles that see nothing of a block's first or last tiles
    dict(hq=32, hk=4, d=128, page=64, lens=[2100, 1001, 3000], new=[2100, 1001, 1290], window=300, sink=70),
    # entries that are in the pool already, behind contexts, rows of q apart
    dict(hq=40, hk=10, d=128, page=32, lens=[2500, 1500, 700], new=[1210, 1500, 333], append=False, strided=True),
]


@pytest.mark.parametrize("case", range(len(MANY)))
@pytest.mark.parametrize("scores", [False, True])
def test_prompts_of_many_items_a_cta(case, scores):
    """The prompt kernel's CTAs, one per SM, take several row blocks each: what one leaves behind (barrier phases, ring positions,
    item slots, counters) carries over to the next, and to the next call, whose results are the same bit for bit."""
    c = Case(**MANY[case], scores=scores, seed=60 + case, prefill=True, extra_rows=2)
    items = sum(-(-t * c.G // 256) for t in c.new) * c.hk
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert items > 3 * sms
    cache = c.cache()
    first = c.run(cache)
    c.check(*first, f"{items} items")
    small = Case(lens=[90], new=[90], hq=c.hq, hk=c.hk, d=c.d, page=c.page)
    for _ in range(3):
        again = c.run(cache)
        for x, y in zip(first, again):
            assert x is None or torch.equal(x, y)
    cache.close()
    small.check(*small.run(), "a handle of its own")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefill", [False, True])
@pytest.mark.parametrize("scale", [0.5, 0.01, 0.73])
def test_scales(dtype, prefill, scale):
    """A softmax scale of the caller's: the definition, whose scale is 1 / sqrt(d), on queries that are scale * sqrt(d) times as large."""
    c = Case(lens=[300, 70], new=[200, 9] if prefill else [1, 1], hq=8, hk=2, d=64, dtype=dtype, page=16, scores=True, seed=71, prefill=prefill)
    cache = c.cache(scale=scale)
    result = c.run(cache)
    c.buf = c.buf.double()
    c.buf[:, :c.hq] *= scale * c.d ** 0.5
    c.check(*result, f"scale {scale}")
    cache.close()


# ---------------------------------------------------------------- shared pages

def _shared(page, entries, **kw):
    """Two sequences whose first `entries` entries (whole pages) are the same ones."""
    c = Case(page=page, scores=True, **kw)
    c.K[1][:entries], c.V[1][:entries] = c.K[0][:entries], c.V[0][:entries]
    c.table[1, :entries // page] = c.table[0, :entries // page]
    return c


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefill", [False, True])
@pytest.mark.parametrize("window,sink", [(0, 0), (100, 20)])
def test_sequences_share_context_pages(dtype, prefill, window, sink):
    """Each sequence's weights are its own, and the shared pages stay as they were."""
    c = _shared(16, 128, lens=[300, 200, 20], new=[150, 60, 20] if prefill else [1, 1, 1], hq=8, hk=2, d=64, dtype=dtype, window=window,
                sink=sink, seed=81, prefill=prefill)
    c.check(*c.run(), "shared")                            # the whole pool among it


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sequences_that_share_pages_are_evicted_by_their_own_weights(dtype):
    page, hk, d, budget, recent, sink = 32, 2, 64, 70, 20, 3
    c = _shared(page, 96, lens=[200, 150], new=[1, 1], hq=hk, hk=hk, d=d, dtype=dtype, append=False, spare=8, seed=82)
    cache = c.cache()
    dst = c.free_pages[:6].reshape(2, 3)
    new_lens, kept = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, hk, budget, dtype=torch.int32, device="cuda")
    cache.wkv_paged_evict(0, c.table.cuda(), dst.cuda(), torch.tensor(c.lens, dtype=torch.int32, device="cuda"), new_lens, budget, recent, sink,
                          scores=c.scores.cuda(), kept=kept)
    assert cache.wkv_status() == 0 and new_lens.tolist() == [budget, budget]
    want_k, want_v = c.k_pool.clone(), c.v_pool.clone()
    for b, n in enumerate(c.lens):
        for h in range(hk):
            order = sorted(range(sink, n - recent), key=lambda i: (float(c.scores[b, h, i]), i))
            stay = sorted(set(range(n)) - set(order[:n - budget]))
            assert kept[b, h].tolist() == stay
            for at, i in enumerate(stay):
                pg = int(dst[b, at // page])
                want_k[0, pg, h, at % page], want_v[0, pg, h, at % page] = c.K[b][i, h], c.V[b][i, h]
    as_int = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(c.gk.cpu().view(as_int), want_k.view(as_int)) and torch.equal(c.gv.cpu().view(as_int), want_v.view(as_int))
    cache.close()


# ---------------------------------------------------------------- eviction around its shared memory

@pytest.mark.parametrize("n", [32767, 32768, 32769, 33792, 33793])
def test_evict_around_the_staged_length(n):
    """Lanes of up to 32768 entries are selected from shared memory, longer ones from the scores themselves."""
    from test_gpu_paged import _evict
    _evict([n, 5], 900, 50, 4, hk=1, d=64, page=64, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [0, 300])
def test_decode_repeats_bit_for_bit(dtype, window):
    """Lanes cut over many CTAs: whichever piece comes last joins them, in the order of the pieces."""
    c = Case(lens=[5000, 1200, 3, 2500], new=[1] * 4, hq=16, hk=4, d=128, dtype=dtype, page=32, scores=True, seed=91, window=window, sink=9 if window else 0)
    cache = c.cache()
    first = c.run(cache)
    c.check(*first, "first")
    for _ in range(20):
        for x, y in zip(first, c.run(cache)):
            assert torch.equal(x, y)
    cache.close()
