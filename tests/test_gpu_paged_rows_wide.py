"""Calls of the largest batch, and seeded random ones over wider ranges: every draw has work to do."""
import random

import pytest
import torch

import test_gpu_paged_choose as choose
import test_gpu_paged_kv4 as kv4
import test_gpu_paged_rows as rows
from paged_rows_util import Pool, window_sees

pytestmark = pytest.mark.gpu
MOST = 1024                                    # sequences of a call: tables of offsets and lengths in shared memory are that long


def _log_int(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))


@pytest.mark.parametrize("kind", rows.KINDS)
@pytest.mark.parametrize("step", [False, True])
def test_append_to_the_most_sequences(kind, step):
    lens = [(i * 37) % 41 for i in range(MOST)]
    new = [min(n, 1) if step else min(n, i % 5) for i, n in enumerate(lens)]
    rows.go(lens, new, kind=kind, hq=2, hk=1, d=64, bounds=True, step=step, extra_rows=0 if step else 3, seed=1, what=kind)


@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 1)])
def test_4_bit_decode_of_the_most_sequences(hq, hk):
    kv4.go([(i * 37) % 150 for i in range(MOST)], hq=hq, hk=hk, d=64, seed=2)
    kv4.go([0] * (MOST - 1) + [700], hq=hq, hk=hk, d=64, seed=3)


@pytest.mark.parametrize("kind", rows.KINDS)
def test_chosen_pages_of_the_most_sequences(kind):
    choose.go([(i * 37) % 150 for i in range(MOST)], 4, 2, 1, kind=kind, hq=2, hk=1, d=64, seed=4)


def draw_decode4(rng):
    hq, hk = rng.choice([(1, 1), (4, 4), (4, 2), (8, 2), (8, 1), (16, 2), (6, 3)])
    n = _log_int(rng, 1, 24)
    even = rng.random() < 0.3                  # lanes of nearly equal length have a deal of their own
    top = _log_int(rng, 1, 12000)
    lens = [0 if rng.random() < 0.1 else top - rng.randint(0, top // 20) if even else _log_int(rng, 1, top) for _ in range(n)]
    if not any(lens):
        lens[0] = top
    window = rng.choice([0, 0, _log_int(rng, 1, 3000)])
    return lens, window, rng.choice([0, rng.randint(1, 200)]) if window else 0, dict(
        hq=hq, hk=hk, d=rng.choice([64, 128]), page=rng.choice([16, 32, 64]), layers=rng.choice([1, 2]), spread=2.0 ** rng.randint(-8, 8))


@pytest.mark.parametrize("seed", range(24))
def test_random_4_bit_decode(seed):
    """Half of the calls store their own rows first: the new token sees its entry as stored."""
    rng = random.Random(1000 + seed)
    lens, window, sink, kind = draw_decode4(rng)
    P = Pool(lens, seed=seed, **kind)
    P.garbage()
    k = v = None
    if seed % 2:
        k, v = ((torch.randn(len(lens), P.hk, P.d, generator=P.g) * kind["spread"]).bfloat16().cuda() for _ in range(2))
    out, lse, status = kv4.run(P, window=window, sink=sink, k=k, v=v)
    assert status == 0
    P.check(out, lse, lambda b, h: window_sees(P.lens[b], window, sink), f"{lens} {window} {sink} {kind}")
    for b, n in enumerate(lens):               # the rest of the pool is as it was
        keep = [int(P.table[b, p]) for p in range((n - 1) // P.page)] if n else []
        assert torch.equal(P.gk[:, keep].cpu(), P.k_pool[:, keep]) and torch.equal(P.gv[:, keep].cpu(), P.v_pool[:, keep])


@pytest.mark.parametrize("seed", range(16))
def test_random_appends(seed):
    rng = random.Random(2000 + seed)
    hq, hk = rng.choice([(1, 1), (4, 4), (8, 2), (16, 2), (6, 3), (5, 5)])
    lens = [0 if rng.random() < 0.15 else _log_int(rng, 1, 3000) for _ in range(_log_int(rng, 1, 30))]
    lens[rng.randrange(len(lens))] = _log_int(rng, 1, 3000)
    step = rng.random() < 0.3
    new = [min(m, 1) if step else min(m, rng.choice([1, 0, _log_int(rng, 1, 400)])) for m in lens]
    if sum(new) == 0:
        new[max(range(len(lens)), key=lambda b: lens[b])] = 1
    d = rng.choice([64, 128])
    rows.go(lens, new, what=f"seed {seed}", kind=rows.KINDS[seed % 3], hq=hq, hk=hk, d=d, page=rng.choice([16, 32, 64]), layers=rng.choice([1, 2]),
            rot=rng.choice([0, 16, 48, d]), paired=rng.random() < 0.5, bounds=rng.random() < 0.7, shift=rng.choice([None, 0, 5]), step=step,
            strided=rng.random() < 0.5, inplace=rng.random() < 0.5, extra_rows=0 if step else rng.choice([0, 3]), seed=seed)


@pytest.mark.parametrize("seed", range(16))
def test_random_choices(seed):
    rng = random.Random(3000 + seed)
    hq, hk = rng.choice([(1, 1), (4, 4), (8, 2), (8, 1), (16, 2), (6, 3)])
    page = rng.choice([16, 32, 64])
    top = _log_int(rng, page, 9000)
    lens = [0 if rng.random() < 0.1 else _log_int(rng, 1, top) for _ in range(_log_int(rng, 1, 12))]
    lens[rng.randrange(len(lens))] = top
    n_select = _log_int(rng, 1, 150)
    recent = rng.randint(1, min(n_select, 4))
    choose.go(lens, n_select, recent, rng.randint(0, min(3, n_select - recent)), kind=rows.KINDS[seed % 3], hq=hq, hk=hk, d=rng.choice([64, 128]),
              page=page, layers=rng.choice([1, 2]), seed=seed)
