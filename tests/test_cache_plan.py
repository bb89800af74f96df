"""Which form vs_cache_attend takes, as its workspace shows it: none for a workgroup a head, then (heads + workers) parts; with longer sequences it never
goes back, so that the longest's workspace serves all.  Host only."""
import random

import pytest

import paper_2603_04460_amd as vs

BLOCKS = sorted(set(range(1, 400)) | {int(1.01 ** i) for i in range(600, 976)} | {16384})


def sizes(batch, hq, hk, n_q):
    return [vs.cache_attend_workspace(batch, hq, hk, n_q, 64 * b) for b in BLOCKS if b <= 16384]


@pytest.mark.parametrize("seed", range(8))
def test_monotone(seed):
    r = random.Random(seed)
    for _ in range(150):
        hk = r.choice([1, 1, 2, 3, 8, 16, 64])
        batch, n_q = int(2 ** r.uniform(0, 9)), r.choice([1, 2, 5, int(2 ** r.uniform(0, 7)), r.randint(1, 128)])
        hq = hk * r.choice([1, 2, 3, 4, 7, 8, 16, 64])
        x = sizes(batch, hq, hk, n_q)
        rows = hq // hk * n_q
        assert all(a <= b for a, b in zip(x, x[1:])), (batch, hq, hk, n_q)
        assert len(set(x)) <= 3 and all(v % (4 * 130 * rows) == 0 for v in x)
        assert x[0] == 0 and x[-1] > 0


@pytest.mark.parametrize("rows", [1, 4, 5, 16, 17, 64, 65, 80, 96, 97, 128, 160, 161, 255, 256, 257, 512, 513, 4096, 4113, 524288])
def test_monotone_in_every_number_of_rows(rows):
    for batch in (1, 2, 31):
        n_q = next(d for d in range(min(rows, 128), 0, -1) if rows % d == 0 and rows // d <= 4096)
        x = sizes(batch, rows // n_q, 1, n_q)
        assert all(a <= b for a, b in zip(x, x[1:]))


def form(batch, hq, hk, n_q, n):
    rows, need = hq // hk * n_q, vs.cache_attend_workspace(batch, hq, hk, n_q, n)
    workers = need // (rows * 520) - batch * hk if need else 0
    return "head" if not need else "tile" if rows > 64 and workers == 256 // -(-rows // 256) else "row"


@pytest.mark.parametrize("batch, hq, hk, n_q, n, want", [
    # timed in each form; the faster by a tenth and more (16 sequences of 2000: where they are equally long)
    (1, 32, 8, 1, 500, "head"), (1, 32, 8, 1, 1500, "row"), (12, 32, 8, 1, 1500, "head"), (32, 32, 8, 1, 2000, "head"), (64, 32, 8, 1, 4000, "row"),
    (300, 4, 1, 1, 1500, "head"), (16, 32, 8, 1, 2000, "head"), (48, 4, 1, 1, 2000, "row"), (1, 32, 8, 5, 1000, "head"), (1, 32, 8, 5, 2000, "row"), (16, 32, 8, 5, 2000, "head"),
    (16, 32, 8, 5, 8000, "row"), (64, 32, 8, 5, 2000, "head"), (64, 32, 8, 5, 8000, "row"), (1, 32, 8, 50, 3000, "head"), (1, 32, 8, 50, 6000, "row"),
    (1, 32, 8, 100, 8000, "head"), (1, 32, 8, 100, 10000, "head"), (1, 32, 8, 100, 16000, "tile"), (1, 32, 8, 64, 10000, "row"), (1, 32, 8, 64, 24000, "tile"),
    (1, 32, 8, 40, 16000, "row"), (1, 32, 8, 40, 131072, "tile"), (1, 32, 8, 32, 131072, "tile"), (1, 32, 8, 16, 131072, "row"), (4, 32, 8, 25, 6000, "row"),
    (4, 16, 2, 20, 20000, "row"), (1, 16, 2, 32, 131072, "tile")])
def test_form(batch, hq, hk, n_q, n, want):
    assert form(batch, hq, hk, n_q, n) == want
