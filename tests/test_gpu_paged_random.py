"""Seeded random paged calls against the definition: every operator, head layout, type, page size, ragged lengths, window and sink."""
import random

import pytest

from paged_util import run_and_check
from test_gpu_paged import LAYOUTS, _evict

pytestmark = pytest.mark.gpu


def _log_int(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))


def draw(seed):
    rng = random.Random(seed)
    op = rng.choice(["decode", "prefill", "prefill", "evict"])
    hq, hk, d = rng.choice(LAYOUTS)
    c = dict(hq=hq, hk=hk, d=d, dtype=rng.choice(["bf16", "bf16", "f32"]), page=rng.choice([16, 32, 64]), seed=seed)
    if op == "evict":
        lens = [rng.choice([0, 1, _log_int(rng, 1, 3000)]) if rng.random() < 0.3 else _log_int(rng, 1, 3000) for _ in range(rng.randint(1, 5))]
        lens[0] = max(1, lens[0])
        budget = _log_int(rng, 1, max(lens))
        sink = rng.randint(0, min(budget, 9))
        return op, dict(lens=lens, budget=budget, recent=rng.randint(0, budget - sink), sink=sink, hk=hk, d=d, dtype=c["dtype"], page=c["page"],
                        seed=seed, kept_given=rng.random() < 0.5)
    c["window"] = rng.choice([0, 0, _log_int(rng, 1, 700)])
    c["sink"] = rng.choice([0, rng.randint(1, 5), rng.randint(1, 200)]) if c["window"] else rng.choice([0, 7])
    c["scores"] = rng.random() < 0.5
    c["strided"] = rng.random() < 0.4
    c["append"] = rng.random() < 0.7
    c["layers"] = rng.choice([1, 1, 2])
    c["extra_cols"] = rng.choice([0, 0, 3, 40])
    c["spikes"] = rng.choice([0.0, 0.0, 0.01])
    n = rng.randint(1, 6)
    if op == "decode":
        lens = [0 if rng.random() < 0.1 else _log_int(rng, 1, 2500) for _ in range(n)]
        return op, dict(c, lens=lens, new=[1 if x else 0 for x in lens], prefill=False)
    new = [0 if rng.random() < 0.1 else _log_int(rng, 1, 600) for _ in range(n)]
    ctx = [rng.choice([0, _log_int(rng, 1, 1500)]) for _ in range(n)]
    return op, dict(c, lens=[a + b for a, b in zip(new, ctx)], new=new, prefill=True, extra_rows=rng.choice([0, 0, 5]))


def check(seed):
    op, kw = draw(seed)
    if op == "evict":
        _evict(**kw)
    else:
        run_and_check(f"seed {seed}: {op} {kw}", **kw)


@pytest.mark.parametrize("block", range(8))
def test_random_calls(block):
    for seed in range(block * 8, block * 8 + 8):
        check(seed)
