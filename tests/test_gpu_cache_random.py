"""stepprune_cache_attend on batches drawn once from fixed seeds, against the oracle: types,
head widths and ratios, pages, layouts, sequences from none to many, rows and runs of very
different lengths in one batch, groups anywhere, bounds at and above the lengths.
Tolerances are tests/cache_case.py's, derived there.
"""
import numpy as np
import pytest

from tests.cache_case import Batch

pytestmark = pytest.mark.gpu

HEADS = [(1, 1), (4, 2), (8, 8), (7, 1), (12, 4), (28, 4), (16, 16), (20, 1)]


def drawn(seed):
    rng = np.random.default_rng(1000 + seed)
    S = int(rng.choice([1, 2, 5, 17, 40, 66, 90]))
    Hq, Hk = HEADS[rng.integers(len(HEADS))]
    budget = 24000 // (Hq * max(1, S // 8))                  # the oracle's work
    tall = rng.random() < 0.5
    rows = lambda: int(rng.choice([0, 1, 1, 1, 2, 3, 9] + ([17, 40, 70, 130] if tall and S <= 17 else [])))
    counts = [rows() for _ in range(S)]
    reach = int(rng.choice([3, 40, 300, min(1500, max(300, budget))]))
    lens = [int(n + rng.integers(0, reach + 1)) if rng.random() < 0.9 else int(rng.integers(0, n + 1)) for n in counts]
    prefix, cuts = [], []
    if rng.random() < 0.6:
        G = int(rng.choice([1, 2, 5, S, S + 3]))
        cuts = sorted(int(c) for c in rng.integers(0, S + 1, G + 1))
        prefix = [int(rng.integers(0, int(rng.choice([2, 70, 700])))) for _ in range(G)]
    b = Batch(counts, lens, heads=(Hq, Hk), D=int(rng.choice([64, 128])), page=int(rng.choice([16, 32, 64, 128, 256])),
              dtype=str(rng.choice(["bf16", "bf16", "f32"])), layout=str(rng.choice(["packed", "padded"])),
              prefix=prefix, cuts=cuts, pad=int(rng.integers(0, 4)), seed=seed)
    slack = {}
    if rng.random() < 0.4:                                   # bounds above what there is
        slack = dict(max_rows=max(counts) + int(rng.integers(0, 100)), max_len=b.tables.shape[1] * b.page)
        if prefix:
            slack["max_prefix"] = b.prefix_tables.shape[1] * b.page
    return b, slack, bool(rng.random() < 0.3), int(rng.choice([0, 8, 64]))


@pytest.mark.parametrize("seed", range(48))
def test_random_batches(gpu_lib, seed):
    b, slack, see_all, extra = drawn(seed)
    b.upload(**slack)
    if b.rows == 0:
        pytest.skip("no rows drawn")
    b.check(*b.attend(see_all=see_all, ld_extra=extra), see_all=see_all)
