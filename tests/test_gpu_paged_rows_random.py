"""Seeded random calls of appending, 4-bit decode and page selection against their definitions."""
import random

import pytest

import test_gpu_paged_choose as choose
import test_gpu_paged_kv4 as kv4
import test_gpu_paged_rows as rows

pytestmark = pytest.mark.gpu
LAYOUTS = [(1, 1), (4, 4), (4, 2), (8, 2), (8, 1), (16, 2), (6, 3)]


def _log_int(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))


def draw(seed):
    rng = random.Random(seed)
    op = rng.choice(["append", "append", "decode4", "choose"])
    hq, hk = rng.choice(LAYOUTS)
    c = dict(hq=hq, hk=hk, d=rng.choice([64, 128]), page=rng.choice([16, 32, 64]), layers=rng.choice([1, 2]), seed=seed)
    n = rng.randint(1, 6)
    lens = [0 if rng.random() < 0.15 else _log_int(rng, 1, 2500) for _ in range(n)]
    if op == "append":
        step = rng.random() < 0.3
        new = [min(m, 1 if step else rng.choice([0, 1, _log_int(rng, 1, 300)])) for m in lens]
        c.update(kind=rng.choice(rows.KINDS), step=step, rot=rng.choice([0, 16, 32, c["d"]]), paired=rng.random() < 0.5,
                 bounds=rng.random() < 0.6, shift=rng.choice([None, 0, 5]), strided=rng.random() < 0.5, inplace=rng.random() < 0.5)
        if not step:
            c["extra_rows"] = rng.choice([0, 3])
        if sum(new) == 0:
            new = [min(m, 1) for m in lens] if any(lens) else new
        return op, (lens, new), c
    if op == "decode4":
        window = rng.choice([0, 0, _log_int(rng, 1, 700)])
        return op, (lens, window, rng.choice([0, rng.randint(1, 70)]) if window else 0), c
    n_select = _log_int(rng, 1, 60)
    recent = rng.randint(1, min(n_select, 4))
    return op, (lens, n_select, recent, rng.randint(0, min(3, n_select - recent))), dict(c, kind=rng.choice(choose.KINDS))


def check(seed):
    op, a, c = draw(seed)
    if op == "append":
        if a[1] and sum(a[1]) + c.get("extra_rows", 0) > 0:
            rows.go(*a, what=f"seed {seed}", **c)
    elif op == "decode4":
        kv4.go(*a, **c)
    else:
        choose.go(*a, **c)


@pytest.mark.parametrize("seed", range(40))
def test_random(seed):
    check(seed)
