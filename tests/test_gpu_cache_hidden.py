"""Tokens that only later rows of a tile see, infinite or NaN: the rows before them are
computed again key by key (csrc/attend.hip).  Here in every kind of tile and chunk, against
the oracle, and with the accuracy that the tiles themselves have.
"""
import numpy as np
import pytest

from tests.cache_case import U32, Batch

pytestmark = pytest.mark.gpu


def place(b, table, at):
    return table[at // b.page], slice(None), at % b.page


def check_rows(b, got, lse, rows):
    """The given rows against the oracle, within tests/cache_case.py's bounds."""
    o, z = b.oracle()
    tol, tol_l = b.bounds(o, z)
    assert np.isfinite(got[rows]).all()
    assert (np.abs(got[rows] - o[rows]) <= tol[rows]).all(), np.max(np.abs(got[rows] - o[rows]) / tol[rows])
    assert (np.abs(lse[rows] - z[rows]) <= tol_l[rows]).all()


# rows and tokens of the sequences, their prefixes and groups: what computes the last sequence
KINDS = {
    "tall": ([70], [100], (), ()),
    "tall, prefix first": ([70], [100], (200,), (0, 1)),
    "tall, a ragged prefix": ([70], [70], (77,), (0, 1)),
    "tall, later chunks": ([70], [3000], (600,), (0, 1)),
    "thin, prefix taken itself": ([70, 5], [90, 41], (200,), (0, 2)),
    "thin, later chunks": ([1, 8], [4000, 3999], (), ()),
    "thin, a shared prefix": ([1, 8], [2100, 2050], (1500,), (0, 2)),
    "wide": ([1, 8], [30, 200], (), ()),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", KINDS)
def test_rows_before_a_hidden_token(gpu_lib, kind, D, bad, dtype):
    counts, lens, prefix, cuts = KINDS[kind]
    b = Batch(counts, lens, heads=(4, 2), D=D, dtype=dtype, prefix=prefix, cuts=cuts, seed=len(kind))
    s, n = len(counts) - 1, counts[-1]
    seen = n - n // 3 - 1                          # the token is row `seen`'s own
    where = place(b, b.tables[s], lens[s] - n + seen)
    b.v_cache[where] = 0.0                         # (the oracle's: those rows weigh it with nothing)
    rows = np.arange(b.rows)
    rows = rows[(rows < b.first[s] + seen) | (rows >= b.first[s] + n)]
    dirty = b.v_cache.copy()
    dirty[where] = bad
    clean, b.v_cache = b.v_cache, dirty
    b.upload()
    o, lse = b.attend()
    b.v_cache = clean
    check_rows(b, o, lse, rows)
    assert not np.isfinite(o[b.first[s] + seen:b.first[s] + n]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_other_sequences_keep_their_bits(gpu_lib, dtype, D):
    """A hidden token changes nothing, not the last bit, of the sequences beside its own."""
    outs = []
    for bad in (0.0, np.nan):
        b = Batch([60, 70, 3, 1], [60, 100, 50, 700], heads=(4, 2), D=D, dtype=dtype, prefix=[90], cuts=[0, 4], seed=5)
        where = place(b, b.tables[1], 30 + 41)
        b.v_cache[where] = bad
        b.upload()
        outs.append(b.attend())
    others = np.r_[0:60, 130:134]
    assert np.array_equal(outs[0][0][others], outs[1][0][others])
    assert np.array_equal(outs[0][1][others], outs[1][1][others])
    assert np.isfinite(outs[1][0][60:101]).all() and np.isnan(outs[1][0][101:130]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [0.0, np.nan])
def test_large_scores_in_float32(gpu_lib, bad, D):
    """Scores of about a thousand that differ by a few, float32.

    Every query is 8 in all elements and the keys are 8 plus eighths, so products and their
    sums are whole numbers below 2^14 that float32 holds: a score's only error is in the
    exponent, off by 2 U32 of its size (below 16 here, from the largest score, which is the
    first), so the weight by 32 U32; the exponential by 2^-22; the sums over 16 keys by 16
    U32 each; division, product and output by 4 U32.  Relative to A = sum p |v|: below
    (32 + 4 + 2 * 16 + 4) U32 = 72 U32.  An exponent rounded at the score's own size (1477
    and 2955 in powers of two) would be off by up to 2^-14 and 2^-13."""
    n = 16
    b = Batch([n], [n], heads=(1, 1), D=D, dtype="f32", seed=3)
    rng = np.random.default_rng(8)
    b.q[:] = 8.0
    eighths = rng.integers(-1, 2, (n, D))
    eighths = eighths[np.argsort(-eighths.sum(1), kind="stable")]           # the largest score first
    assert (eighths[0].sum() - eighths[-1].sum()) * 0.25 * 1.4427 < 16
    for p in range(n):
        b.k_cache[place(b, b.tables[0], p)] = 8.0 + eighths[p] / 8.0
    b.scale = 0.25
    last = place(b, b.tables[0], n - 1)
    b.v_cache[last] = 0.0
    o, lse = b.oracle()
    A, _ = b.oracle(v_cache=np.abs(b.v_cache))
    b.v_cache[last] = bad
    b.upload()
    got, z = b.attend()
    err = np.abs(got - o)[:n - 1] / A[:n - 1]
    assert err.max() <= 72 * U32, err.max() / U32
    assert np.abs(z - lse)[:n - 1].max() <= 6 * U32 * np.abs(lse).max()
