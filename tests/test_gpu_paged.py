"""Paged caches on the GPU against the definition in 64 bits (tests/paged_util.py has the bounds and their derivation)."""
import pytest
import torch

from paged_util import Case, run_and_check
from paper_2503_01330_b200 import binding

pytestmark = pytest.mark.gpu

LAYOUTS = [(4, 4, 64), (8, 2, 128), (16, 2, 64), (4, 2, 128), (4, 4, 128), (8, 1, 64), (8, 1, 128)]


# ---------------------------------------------------------------- decode

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,d", LAYOUTS)
@pytest.mark.parametrize("page", [16, 32, 64])
def test_decode_layouts(dtype, hq, hk, d, page):
    lens = [1, 15, 16, 17, 0, 63, 64, 65, 127, 130, 300]
    run_and_check("decode", lens=lens, new=[1 if n else 0 for n in lens], hq=hq, hk=hk, d=d, dtype=dtype, page=page,
                  scores=page == 16, layers=2, seed=page, extra_cols=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (7, 0), (64, 4), (100, 64), (100, 65), (33, 300), (508, 4), (5000, 9), (0, 5)])
def test_decode_windows(dtype, window, sink):
    lens = [1, 2, 8, 64, 65, 101, 164, 165, 166, 259, 700]
    run_and_check("decode window", lens=lens, new=[1] * len(lens), hq=8, hk=4, d=64, dtype=dtype, page=16, window=window,
                  sink=sink, scores=True, seed=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("append", [True, False])
def test_decode_strided_rows_and_no_append(dtype, append):
    run_and_check("decode", lens=[5, 700, 90], new=[1, 1, 1], hq=8, hk=2, d=128, dtype=dtype, page=32, strided=True, scores=True,
                  append=append, seed=3)


@pytest.mark.parametrize("dtype,hq,hk,d", [("bf16", 8, 1, 128), ("bf16", 8, 8, 128), ("f32", 4, 4, 64), ("bf16", 32, 8, 64)])
def test_decode_long(dtype, hq, hk, d):
    """One long sequence, cut over many CTAs, and a ragged batch whose pieces cross sequences."""
    run_and_check("one long", lens=[9001], new=[1], hq=hq, hk=hk, d=d, dtype=dtype, page=64, scores=True, seed=4)
    run_and_check("ragged", lens=[4000, 1, 777, 2049], new=[1] * 4, hq=hq, hk=hk, d=d, dtype=dtype, page=16, seed=5)


def test_decode_many_sequences():
    lens = [1 + (i * 37) % 150 for i in range(200)] + [0] * 7
    run_and_check("many", lens=lens, new=[1 if n else 0 for n in lens], hq=4, hk=2, d=64, dtype="bf16", page=16, scores=True, seed=6)


# ---------------------------------------------------------------- prompts

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,d", LAYOUTS)
@pytest.mark.parametrize("page", [16, 32, 64])
def test_prefill_layouts(dtype, hq, hk, d, page):
    # whole prompts, a chunk behind a context, one token, no token, a length at a tile's edge
    run_and_check("prefill", lens=[1, 130, 300, 77, 40, 128, 257], new=[1, 130, 50, 1, 0, 128, 129], hq=hq, hk=hk, d=d, dtype=dtype,
                  page=page, layers=2, seed=page, extra_rows=3, scores=page == 32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 2), (16, 4), (100, 64), (129, 1), (128, 130), (1000, 5)])
def test_prefill_windows(dtype, window, sink):
    run_and_check("prefill window", lens=[300, 513, 600, 33], new=[300, 140, 3, 33], hq=8, hk=2, d=64, dtype=dtype, page=16,
                  window=window, sink=sink, scores=True, seed=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_strided_and_no_append(dtype):
    for append in (True, False):
        run_and_check("prefill", lens=[90, 400], new=[90, 61], hq=8, hk=2, d=128, dtype=dtype, page=64, strided=True, scores=True,
                      append=append, seed=8)


@pytest.mark.parametrize("hq,hk,d", [(4, 4, 128), (8, 1, 128), (4, 2, 64)])
def test_prefill_long(hq, hk, d):
    run_and_check("long prompt", lens=[1500], new=[1500], hq=hq, hk=hk, d=d, page=32, scores=True, seed=9)
    run_and_check("few tokens, long context", lens=[5003, 2600], new=[5, 17], hq=hq, hk=hk, d=d, page=64, scores=True, seed=10)


# ---------------------------------------------------------------- eviction

def _evict(lens, budget, recent, sink, hk=2, d=64, dtype="bf16", page=16, seed=0, scores=None, kept_given=True, spare=None):
    need = sum(-(-min(n, budget) // page) for n in lens)
    c = Case(lens=lens, new=[min(n, 1) for n in lens], hq=hk, hk=hk, d=d, dtype=dtype, page=page, append=False, scores=True, seed=seed,
             layers=2, spare=need + 2, extra_cols=1)
    if scores is not None:
        scores(c.scores)
    B = len(lens)
    dst_w = max(max(-(-min(n, budget) // page) for n in lens), -(-min(budget, c.width * page) // page))
    dst = torch.full((B, dst_w), -5, dtype=torch.int32)
    at = 0
    for b, n in enumerate(lens):
        m = -(-min(n, budget) // page)
        dst[b, :m] = c.free_pages[at:at + m]
        at += m
    cache = c.cache()
    new_lens = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    kept = torch.full((B, hk, budget), -1, dtype=torch.int32, device="cuda") if kept_given else None
    scores_out = torch.full((B, hk, budget + 3), 9.0, device="cuda")
    cache.wkv_paged_evict(c.layer, c.table.cuda(), dst.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), new_lens,
                          budget, recent, sink, scores=c.scores.cuda(), scores_out=scores_out, kept=kept)
    assert cache.wkv_status() == 0
    want_k, want_v = c.k_pool.clone(), c.v_pool.clone()
    for b, n in enumerate(lens):
        m = min(n, budget)
        assert int(new_lens[b]) == m
        for h in range(hk):
            x = c.scores[b, h, :n].tolist()
            safe = [i < sink or i >= n - recent for i in range(n)]
            key = lambda i: (float("inf") if x[i] != x[i] else x[i], x[i] != x[i], i)
            gone = set(sorted((i for i in range(n) if not safe[i]), key=key)[:n - m])
            stay = [i for i in range(n) if i not in gone]
            if kept is not None:
                assert kept[b, h, :m].tolist() == stay, f"sequence {b}, head {h}"
                assert (kept[b, h, m:] == -1).all()
            got = scores_out[b, h].cpu()
            assert torch.equal(got[:m].view(torch.int32), c.scores[b, h, stay].view(torch.int32)) and (got[m:] == 9).all()
            for at, i in enumerate(stay):
                pg = int(dst[b, at // page])
                want_k[c.layer, pg, h, at % page] = c.K[b][i, h]
                want_v[c.layer, pg, h, at % page] = c.V[b][i, h]
    i16 = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(c.gk.cpu().view(i16), want_k.view(i16)) and torch.equal(c.gv.cpu().view(i16), want_v.view(i16))
    cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("budget,recent,sink", [(1, 1, 0), (1, 0, 0), (16, 4, 2), (100, 33, 4), (100, 96, 4), (300, 0, 0)])
def test_evict(dtype, page, budget, recent, sink):
    _evict([1, 17, 100, 101, 0, 299, 300, 301], budget, recent, sink, dtype=dtype, page=page, seed=budget)


@pytest.mark.parametrize("d,hk", [(128, 3), (64, 8)])
def test_evict_long(d, hk):
    _evict([3000, 1500, 1025, 2048], 1024, 508, 4, hk=hk, d=d, seed=1, kept_given=False)
    _evict([9000], 700, 64, 4, hk=1, d=d, page=64, seed=2)


def test_evict_past_the_register_form():
    """Lanes around 32768 entries, where keys no longer fit registers, and beyond."""
    _evict([32768, 32769, 40001], 33, 5, 2, hk=1, d=64, page=64, seed=6)

    def few(x):
        x.copy_((x * 5).floor())
    _evict([40000, 32767], 20000, 50, 4, hk=1, d=64, page=64, seed=7, scores=few)


def test_evict_ties_and_special_scores():
    def few(x):
        x.copy_((x * 3).floor())                    # many equal scores
    _evict([200, 90], 50, 10, 2, scores=few, seed=3)

    def same(x):
        x.fill_(0.25)
    _evict([200, 1300], 50, 10, 2, scores=same, seed=4)

    def special(x):
        x[..., 5::7] = float("inf")
        x[..., 3::11] = float("nan")
        x[..., 2::5] = -0.0
        x[..., 4::9] = 0.0
        x[..., 6::13] = -1.5
        x[..., 1::17] = 1e-42
        x[..., 8::19] = float("-inf")
    _evict([200, 1300], 50, 10, 2, scores=special, seed=5)


def test_evict_overlapping_tables_move_nothing():
    c = Case(lens=[100, 60], new=[1, 1], hq=2, hk=2, d=64, page=16, append=False, scores=True, spare=8)
    cache = c.cache()
    dst = torch.zeros(2, 2, dtype=torch.int32)
    dst[0] = torch.tensor([int(c.free_pages[0]), int(c.table[0, 3])])       # the second page is one of the sequence's own
    dst[1] = c.free_pages[1:3]
    new_lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    kept = torch.full((2, 2, 32), -1, dtype=torch.int32, device="cuda")
    cache.wkv_paged_evict(0, c.table.cuda(), dst.cuda(), torch.tensor(c.lens, dtype=torch.int32, device="cuda"), new_lens, 32, 4, 0,
                          scores=c.scores.cuda(), kept=kept)
    assert cache.wkv_status() == binding.WKV_ERR_STATE and cache.wkv_status() == 0
    assert new_lens.tolist() == [100, 32] and (kept[0] == -1).all() and (kept[1] >= 0).all()
    used = torch.zeros(c.n_pages, dtype=torch.bool)
    used[c.free_pages[1:3].long()] = True
    same = c.gk.cpu().view(torch.int16) == c.k_pool.view(torch.int16)
    assert same[:, ~used].all()
    cache.close()


# ---------------------------------------------------------------- as they are used together

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_evict_decode(dtype):
    """A heavy-hitter cache: prompts in two chunks with weights, eviction, decode steps with weights, eviction, a step."""
    hq, hk, d, page, budget, recent, sink = 8, 2, 64, 16, 96, 24, 4
    lens, chunk = [210, 150], 64
    first = Case(lens=[chunk, chunk], new=[chunk, chunk], hq=hq, hk=hk, d=d, dtype=dtype, page=page, scores=True, seed=1, width=16, spare=80)
    # page lists of both sequences: the first chunk's, then free ones
    cache = first.cache()
    free = first.free_pages.tolist()
    take = lambda n: [free.pop() for _ in range(n)]
    table = first.table.clone()
    for b in range(2):
        table[b, chunk // page:] = torch.tensor(take(16 - chunk // page))
    scores = first.scores.clone().cuda()

    def step(case_lens, new, tab, K, V, base, prefill):
        """One library call on explicit contents; K, V: per sequence [len, hk, d]; returns the case for its check."""
        c = Case(lens=case_lens, new=new, hq=hq, hk=hk, d=d, dtype=dtype, page=page, scores=True, seed=sum(case_lens), width=16, prefill=prefill)
        for b in range(2):
            n, t = case_lens[b], new[b]
            K[b] = torch.cat([K[b], c.K[b][n - t:]])
            V[b] = torch.cat([V[b], c.V[b][n - t:]])
        c.K, c.V, c.scores = K, V, base.cpu()
        for b in range(2):
            s, n, t = c.starts[b], case_lens[b], new[b]
            c.buf[s:s + t, hq:hq + hk], c.buf[s:s + t, hq + hk:hq + 2 * hk] = K[b][n - t:], V[b][n - t:]
        q, k, v = c.rows()
        out, lse = torch.full((c.T, hq, d), 7.0, dtype=c.tdt, device="cuda"), torch.full((c.T, hq), 7.0, device="cuda")
        L = torch.tensor(case_lens, dtype=torch.int32, device="cuda")
        if prefill:
            cache.wkv_paged_prefill(0, q, k, v, torch.tensor(c.starts, dtype=torch.int32, device="cuda"), tab.cuda(), L, out, scores=base, lse=lse)
        else:
            cache.wkv_paged_decode(0, q, k, v, tab.cuda(), L, out, scores=base, lse=lse)
        assert cache.wkv_status() == 0
        c.check_pool = lambda what="": None
        c.check(out, lse, base, "run")

    E = torch.empty(0, hk, d, dtype=first.tdt)
    K, V = [E, E], [E, E]
    step([chunk, chunk], [chunk, chunk], table, K, V, scores, True)
    step(lens, [n - chunk for n in lens], table, K, V, scores, True)

    def evict(cur, tab):
        dst = torch.tensor([take(budget // page) for _ in range(2)], dtype=torch.int32)
        new_lens = torch.zeros(2, dtype=torch.int32, device="cuda")
        out = torch.zeros(2, hk, 16 * page, device="cuda")
        kept = torch.zeros(2, hk, budget, dtype=torch.int32, device="cuda")
        cache.wkv_paged_evict(0, tab.cuda(), dst.cuda(), torch.tensor(cur, dtype=torch.int32, device="cuda"), new_lens, budget, recent,
                              sink, scores=scores, scores_out=out, kept=kept)
        assert cache.wkv_status() == 0 and new_lens.tolist() == [budget, budget]
        kept = kept.long().cpu()
        for b in range(2):
            K[b] = torch.stack([K[b][kept[b, h], h] for h in range(hk)], 1)
            V[b] = torch.stack([V[b][kept[b, h], h] for h in range(hk)], 1)
        wide = torch.zeros(2, 16, dtype=torch.int32)
        wide[:, :budget // page] = dst
        for b in range(2):
            wide[b, budget // page:budget // page + 2] = torch.tensor(take(2))
        return out, wide

    scores, table = evict(lens, table)
    cur = budget
    for _ in range(20):
        cur += 1
        step([cur, cur], [1, 1], table, K, V, scores, False)
    scores, table = evict([cur, cur], table)
    step([budget + 1, budget + 1], [1, 1], table, K, V, scores, False)
    cache.close()


# ---------------------------------------------------------------- streams, graphs, tables, refusals

def test_captured_steps_follow_new_lengths_and_tables():
    """One captured decode step replayed while the sequences grow, beside a second handle's eager calls."""
    c = Case(lens=[70, 33, 0], new=[1, 1, 0], hq=8, hk=2, d=128, page=16, scores=True, seed=11, spare=40, width=12)
    for b in range(3):
        n = -(-c.lens[b] // 16)
        c.table[b, n:] = c.free_pages[b * 12:b * 12 + 12 - n]
    cache = c.cache()
    q, k, v = c.rows()
    table, lens = c.table.cuda(), torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    out, lse = torch.empty(3, 8, 128, dtype=c.tdt, device="cuda"), torch.empty(3, 8, device="cuda")
    scores = c.scores.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache.wkv_set_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cache.wkv_paged_decode(0, q, k, v, table, lens, out, scores=scores, lse=lse)
    for n in ([70, 33, 0], [71, 0, 1], [192, 34, 17]):
        new = [1 if x else 0 for x in n]
        d = Case(lens=n, new=new, hq=8, hk=2, d=128, page=16, scores=True, seed=sum(n), width=12, spare=40, append=False)
        c.gk.copy_(torch.full_like(c.gk, float("nan")))
        c.gv.copy_(c.gk)
        for b in range(3):
            for i in range(n[b]):
                pg = int(c.table[b, i // 16])
                c.gk[0, pg, :, i % 16], c.gv[0, pg, :, i % 16] = d.K[b][i].cuda(), d.V[b][i].cuda()
        d.append = True                                  # the last entry comes with the call
        dq, dk, dv = d.rows()
        q.copy_(dq); k.copy_(dk); v.copy_(dv); lens.copy_(torch.tensor(n, dtype=torch.int32)); scores.copy_(d.scores)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        d.check_pool = lambda what="": None
        d.check(out, lse, scores, f"replay {n}")
    assert cache.wkv_status() == 0
    del graph
    cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_prompt_and_eviction(dtype):
    """A prompt call and an eviction captured once, replayed for batches of other lengths, interleaved with a second handle's
    calls on another stream."""
    B, hq, hk, d, page, T, width = 3, 8, 2, 64, 16, 300, 24
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    base = Case(lens=[1] * B, new=[1] * B, hq=hq, hk=hk, d=d, dtype=dtype, page=page, scores=True, seed=31, spare=2 * B * width, width=width)
    pages = torch.randperm(base.n_pages, generator=torch.Generator().manual_seed(5)).int()
    table, dst = pages[:B * width].reshape(B, width).cuda(), pages[B * width:2 * B * width].reshape(B, width).cuda()
    cache = base.cache()
    side, other_stream = torch.cuda.Stream(), torch.cuda.Stream()
    other = Case(lens=[200, 3], new=[150, 3], hq=hq, hk=hk, d=d, dtype=dtype, page=page, scores=True, seed=32)
    with torch.cuda.stream(other_stream):
        other_cache = other.cache()
    q, k, v = (torch.zeros(T, h, d, dtype=tdt, device="cuda") for h in (hq, hk, hk))
    out, lse = torch.zeros(T, hq, d, dtype=tdt, device="cuda"), torch.zeros(T, hq, device="cuda")
    scores, kept = torch.zeros(B, hk, width * page, device="cuda"), torch.zeros(B, hk, 40, dtype=torch.int32, device="cuda")
    scores_out = torch.zeros(B, hk, 40, device="cuda")
    starts, lens, new_lens = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B + 1, B, B))
    cache.wkv_set_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cache.wkv_paged_prefill(0, q, k, v, starts, table, lens, out, window=70, sink=3, scores=scores, lse=lse)
        cache.wkv_paged_evict(0, table, dst, lens, new_lens, 40, 10, 3, scores=scores, scores_out=scores_out, kept=kept)
    for new in ([100, 1, 30], [0, 299, 1], [64, 65, 128]):
        c = Case(lens=new, new=new, hq=hq, hk=hk, d=d, dtype=dtype, page=page, scores=True, seed=sum(new), width=width, window=70, sink=3,
                 prefill=True, extra_rows=T - sum(new))
        cq, ck, cv = c.rows()
        q.copy_(cq); k.copy_(ck); v.copy_(cv)
        out.fill_(7); lse.fill_(7); scores.copy_(c.scores); kept.fill_(-1)
        starts.copy_(torch.tensor(c.starts, dtype=torch.int32)); lens.copy_(torch.tensor(new, dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(other_stream):
            result = other.run(other_cache)
        torch.cuda.synchronize()
        c.check_pool = lambda what="": None
        c.check(out, lse, scores, f"replay {new}")
        other.check(*result, "beside it")
        assert new_lens.tolist() == [min(n, 40) for n in new]
        for b in range(B):
            for h in range(hk):
                i = kept[b, h, :min(new[b], 40)].long().cpu()
                assert torch.equal(scores_out[b, h, :len(i)].cpu(), scores[b, h].cpu()[i]) and (i[1:] > i[:-1]).all()
                for at in range(0, len(i), 7):
                    got = base.gk[0, int(dst[b, at // page]), h, at % page].cpu()
                    assert torch.equal(got, c.K[b][int(i[at]), h])
    assert cache.wkv_status() == 0 and other_cache.wkv_status() == 0
    del graph
    cache.close()
    other_cache.close()


@pytest.mark.parametrize("prefill", [False, True])
def test_logits_that_tower_over_all_before(prefill):
    """The softmax's running reference has to follow: keys 25 times as long as the others turn up late."""
    for dtype in ("bf16", "f32"):
        run_and_check("spikes", lens=[700, 300], new=[700, 130] if prefill else [1, 1], hq=8, hk=2, d=128, dtype=dtype, page=16, scores=True,
                      seed=41, spikes=0.02, prefill=prefill)


@pytest.mark.parametrize("prefill", [False, True])
def test_bad_tables_and_lengths_are_reported_and_touch_nothing_else(prefill):
    new = [40, 30, 20] if prefill else [1, 1, 1]
    c = Case(lens=[100, 90, 80], new=new, hq=4, hk=2, d=64, page=16, scores=True, seed=12, prefill=prefill, garbage=0.0)
    cache = c.cache()
    q, k, v = c.rows()
    out, lse, scores = torch.zeros(c.T, 4, 64, dtype=c.tdt, device="cuda"), torch.zeros(c.T, 4, device="cuda"), c.scores.cuda()
    start = torch.tensor(c.starts, dtype=torch.int32, device="cuda")

    def call(table, lens, start=start):
        t, n = table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
        if prefill:
            cache.wkv_paged_prefill(0, q, k, v, start, t, n, out, scores=scores, lse=lse)
        else:
            cache.wkv_paged_decode(0, q, k, v, t, n, out, scores=scores, lse=lse)
        return cache.wkv_status()

    assert call(c.table, c.lens) == 0
    good = out.clone()
    for bad in (-1, c.n_pages, 2 ** 31 - 1, -2 ** 31):
        t = c.table.clone()
        t[1, 2] = bad
        t[1, 5] = bad                                   # the page that the new rows go to
        scores.copy_(c.scores)
        assert call(t, c.lens) == binding.WKV_ERR_STATE
        first, last = c.starts[1], c.starts[2]
        assert torch.equal(out[:first], good[:first]) and torch.equal(out[last:], good[last:]), bad
    for lens in ([100, -3, 80], [100, 2 ** 31 - 1, 80], [100, c.width * 16 + 1, 80]):
        t = c.table.clone()
        t[1] = t[0]                                     # any valid pages; appends of both land in one sequence's rows
        t[1, -1] = c.free_pages[0]
        assert call(t, lens) == binding.WKV_ERR_STATE
    if prefill:
        for s in ([0, 40, 30, 90], [0, 40, 70, 1000], [-5, 40, 70, 90], [0, 2 ** 31 - 1, 70, 90]):
            assert call(c.table, c.lens, torch.tensor(s, dtype=torch.int32, device="cuda")) == binding.WKV_ERR_STATE
    c2 = Case(lens=[100, 90, 80], new=new, hq=4, hk=2, d=64, page=16, scores=True, seed=12, prefill=prefill)
    run = c2.run()
    c2.check(*run, "afterwards")
    cache.close()


def test_large_pool_offsets():
    """Pages whose first element lies past 2^31: pools of 4.4 GB."""
    hk, page, d = 8, 64, 128
    n_pages = (2 ** 31 + 2 ** 26) // (hk * page * d)
    k_pool = torch.empty(1, n_pages, hk, page, d, dtype=torch.bfloat16, device="cuda")
    v_pool = torch.empty_like(k_pool)
    c = Case(lens=[200, 77], new=[1, 1], hq=16, hk=hk, d=d, page=page, seed=13, scores=True)
    table = c.table.clone()
    used = (table < c.n_pages)
    far = torch.where(used, n_pages - 1 - table, table)
    for p in table[used].tolist():
        k_pool[0, n_pages - 1 - p], v_pool[0, n_pages - 1 - p] = c.k_pool[0, p].cuda(), c.v_pool[0, p].cuda()
    cache = binding.PagedCache(1, n_pages, page, 16, hk, d, 2, c.width, scores=True, k_pool=k_pool, v_pool=v_pool)
    c.check_pool = lambda what="": None
    for prefill in (False, True):
        q, k, v = c.rows()
        out, lse, scores = torch.empty(2, 16, d, dtype=c.tdt, device="cuda"), torch.empty(2, 16, device="cuda"), c.scores.cuda()
        lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
        c.prefill = prefill
        if prefill:
            cache.wkv_paged_prefill(0, q, k, v, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), far.cuda(), lens, out, scores=scores, lse=lse)
        else:
            cache.wkv_paged_decode(0, q, k, v, far.cuda(), lens, out, scores=scores, lse=lse)
        assert cache.wkv_status() == 0
        c.check(out, lse, scores, "far pages")
    dst = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    new_lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    kept = torch.zeros(2, hk, 100, dtype=torch.int32, device="cuda")
    cache.wkv_paged_evict(0, far.cuda(), dst, lens, new_lens, 100, 9, 3, scores=scores, kept=kept)
    assert cache.wkv_status() == 0 and new_lens.tolist() == [100, 77]
    for h in (0, hk - 1):
        got = k_pool[0, :2, h].reshape(-1, d)[:100].cpu()
        assert torch.equal(got, c.K[0][kept[0, h].long().cpu(), h])
    cache.close()


def test_memory_provider_failing_at_every_request():
    """wkv_paged_create asks for one block after the other; whichever is refused, it returns WKV_ERR_ALLOC and hands all back."""
    import ctypes as C
    L = binding.lib()
    for pools in (False, True):
        kp, vp = (torch.zeros(2, 4, 2, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        fail_at, n = 0, 1
        while fail_at < n:
            live, count = {}, [0]

            def alloc(nbytes, _user):
                count[0] += 1
                if count[0] - 1 == fail_at:
                    return None
                buf = torch.empty(int(nbytes), dtype=torch.uint8, device="cuda")
                live[buf.data_ptr()] = buf
                return buf.data_ptr()

            a, r = binding.ALLOC_FN(alloc), binding.RELEASE_FN(lambda p, _user: live.__delitem__(p))
            cfg = binding.make_paged_config(2, 4, 16, 4, 2, 64, 2, 4, scores=1, k_pool=kp.data_ptr() if pools else None,
                                            v_pool=vp.data_ptr() if pools else None)
            cfg.alloc, cfg.release = a, r
            h = C.c_void_p()
            rc = L.wkv_paged_create(C.byref(cfg), C.byref(h))
            if fail_at == 0 and n == 1:                       # how many requests a creation makes
                assert rc == binding.WKV_ERR_ALLOC and not h.value and not live
                fail_at = 1 << 30
                count[0] = 0
                rc = L.wkv_paged_create(C.byref(cfg), C.byref(h))
                assert rc == binding.WKV_OK and L.wkv_paged_device_bytes(h) > 0
                n, fail_at = count[0], 1
                torch.cuda.synchronize()
                L.wkv_paged_destroy(h)
                assert not live
                continue
            assert rc == binding.WKV_ERR_ALLOC and not h.value and not live, f"request {fail_at}"
            fail_at += 1
        assert n >= (8 if pools else 10)


def test_refusals():
    c = Case(lens=[40, 20], new=[1, 1], hq=4, hk=2, d=64, page=16, scores=True, seed=14)
    cache = c.cache()
    q, k, v = c.rows()
    t, n = c.table.cuda(), torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    out, lse, scores = torch.empty_like(q), torch.empty(2, 4, device="cuda"), c.scores.cuda()
    start = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    launches = cache.wkv_launch_count()

    def refused(call, fragment):
        with pytest.raises(binding.WkvError) as e:
            call()
        assert e.value.code == binding.WKV_ERR_INVALID and fragment in str(e.value), str(e.value)

    dec = lambda **kw: cache.wkv_paged_decode(**{**dict(layer=0, q=q, k=k, v=v, block_table=t, seq_lens=n, out=out), **kw})
    pre = lambda **kw: cache.wkv_paged_prefill(**{**dict(layer=0, q=q, k=k, v=v, q_start=start, block_table=t, seq_lens=n, out=out), **kw})
    for call in (dec, pre):
        refused(lambda: call(layer=1), "layer")
        refused(lambda: call(layer=-1), "layer")
        refused(lambda: call(window=-1), "window")
        refused(lambda: call(sink=-1), "window")
        refused(lambda: call(k=None), "k and v")
        refused(lambda: call(q=q.float()), "q must be")
        refused(lambda: call(q=q[:, :, :32]), "q must be")
        refused(lambda: call(q=q.cpu()), "q must be")
        refused(lambda: call(q=q.transpose(1, 2).contiguous().transpose(1, 2)), "q must be")
        refused(lambda: call(k=k.expand(2, 2, 64)[:, :1]), "k must be")
        refused(lambda: call(seq_lens=n.long()), "seq_lens")
        refused(lambda: call(block_table=t.long()), "block_table")
        refused(lambda: call(out=out[:1]), "out")
        refused(lambda: call(scores=scores[:, :, :16].contiguous(), lse=lse), "score_stride")
        refused(lambda: call(scores=scores.double(), lse=lse), "scores")
        odd = torch.zeros(2, 4 * 64 + 4, dtype=c.tdt, device="cuda")[:, :256].view(2, 4, 64)
        refused(lambda: call(q=odd), "aligned")
    refused(lambda: pre(scores=scores), "lse")
    refused(lambda: pre(q_start=start[:2]), "q_start")
    wide = torch.zeros(2, c.width + 1, dtype=torch.int32, device="cuda")
    refused(lambda: dec(block_table=wide), "table_width")
    big = torch.zeros(3, 4, 64, dtype=c.tdt, device="cuda")
    refused(lambda: dec(q=big, k=big[:, :2], v=big[:, :2], block_table=torch.zeros(3, 1, dtype=torch.int32, device="cuda"),
                        seq_lens=torch.zeros(3, dtype=torch.int32, device="cuda"), out=torch.empty_like(big)), "batch")
    new = torch.zeros(2, dtype=torch.int32, device="cuda")
    dst = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    ev = lambda **kw: cache.wkv_paged_evict(**{**dict(layer=0, src_table=t, dst_table=dst, seq_lens=n, new_lens=new, budget=20, recent=4,
                                                      sink=2, scores=scores), **kw})
    refused(lambda: ev(budget=0), "budget")
    refused(lambda: ev(budget=5), "budget")
    refused(lambda: ev(recent=-1), "budget")
    refused(lambda: ev(budget=40), "dst_table")
    refused(lambda: ev(new_lens=n), "must not be")
    refused(lambda: ev(scores_out=scores), "must not be")
    refused(lambda: ev(scores_out=torch.empty(2, 2, 19, device="cuda")), "out_stride")
    refused(lambda: ev(kept=torch.empty(2, 2, 19, dtype=torch.int32, device="cuda")), "kept")
    assert cache.wkv_launch_count() == launches
    plain = binding.PagedCache(1, 8, 16, 4, 2, 64, 2, 4)
    with pytest.raises(binding.WkvError, match="scores = 1"):
        plain.wkv_paged_decode(0, q, k, v, t, n, out, scores=scores)
    plain.close()
    # nothing to do is no error
    e = torch.empty(0, 4, 64, dtype=c.tdt, device="cuda")
    cache.wkv_paged_prefill(0, e, e[:, :2], e[:, :2], torch.zeros(3, dtype=torch.int32, device="cuda"), t, n, e)
    assert cache.wkv_launch_count() == launches and cache.wkv_status() == 0
    cache.close()
