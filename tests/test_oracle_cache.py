"""The cache's oracle (oracle/cache.py) against other statements of the same things."""
import numpy as np

from oracle import cache as C


def _paged(rng, runs, Hk, D, page):
    need = [-(-n // page) for n in runs]
    order = rng.permutation(sum(need))
    at = np.concatenate([[0], np.cumsum(need)])
    tables = [order[at[i]:at[i + 1]] for i in range(len(runs))]
    shape = (sum(need), Hk, page, D)
    return rng.standard_normal(shape), rng.standard_normal(shape), tables


def test_attention_over_pages_is_attention_over_the_tokens():
    """Against a softmax matrix over the gathered tokens, prefix first; a prefix run is the
    same as those tokens in front of a sequence's own."""
    rng = np.random.default_rng(0)
    Hq, Hk, D, page = 6, 2, 8, 4
    n, L, P = 5, 9, 7
    k, v, tables = _paged(rng, [L, P], Hk, D, page)
    q = rng.standard_normal((n, Hq, D))
    o, lse = C.attend(q, k, v, [0], [n], [tables[0]], [L], 0.3, [tables[1]], [P], [0, 1])
    flat = lambda c, t, m: c[t].transpose(0, 2, 1, 3).reshape(-1, Hk, D)[:m]
    K = np.concatenate([flat(k, tables[1], P), flat(k, tables[0], L)]).repeat(Hq // Hk, 1)
    V = np.concatenate([flat(v, tables[1], P), flat(v, tables[0], L)]).repeat(Hq // Hk, 1)
    s = 0.3 * np.einsum("nhd,khd->hnk", q, K)
    s[:, np.arange(P + L)[None, :] > (P + L - n + np.arange(n))[:, None]] = -np.inf
    e = np.exp(s)
    assert np.allclose(o, np.einsum("hnk,khd->nhd", e / e.sum(-1, keepdims=True), V), atol=1e-12)
    assert np.allclose(lse, np.log(e.sum(-1)).T, atol=1e-12)


def test_rows_that_see_nothing():
    rng = np.random.default_rng(1)
    k, v, tables = _paged(rng, [2], 1, 4, 4)
    q = rng.standard_normal((4, 1, 4))
    o, lse = C.attend(q, k, v, [0], [4], tables, [2], 1.0)
    assert (o[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.isfinite(lse[2:]).all()
    assert np.allclose(o[2, 0], v[tables[0][0], 0, 0])                       # one token: its value


def test_rotation_keeps_lengths_and_depends_on_the_distance_alone():
    rng = np.random.default_rng(2)
    pairs, D = 6, 16
    freq = 50.0 ** (-np.arange(pairs) / pairs)
    table = np.stack([np.cos(np.arange(40)[:, None] * freq), np.sin(np.arange(40)[:, None] * freq)], -1)
    x, y = rng.standard_normal((2, D))
    for inter in (False, True):
        r = lambda z, p: C.rotate(z, table[p], inter)
        assert np.allclose(np.linalg.norm(r(x, 31)), np.linalg.norm(x))
        assert np.allclose(r(x, 5) @ r(y, 9), r(x, 25) @ r(y, 29))
        assert (r(x, 7)[2 * pairs:] == x[2 * pairs:]).all() and (r(x, 0) == x).all()


def test_append_then_read_back():
    rng = np.random.default_rng(3)
    Hq, Hk, D, page = 2, 1, 8, 4
    k, v, tables = _paged(rng, [9, 3], Hk, D, page)
    kn, vn, q = rng.standard_normal((5, Hk, D)), rng.standard_normal((5, Hk, D)), rng.standard_normal((5, Hq, D))
    qo, k2, v2 = C.append(k, v, q, kn, vn, [0, 4], [4, 1], tables, [9, 3])
    assert np.array_equal(qo, q)
    assert np.array_equal(C.run_tokens(k2, tables[0], 9)[5:], kn[:4])
    assert np.array_equal(C.run_tokens(v2, tables[1], 3)[2:], vn[4:])
    assert np.array_equal(C.run_tokens(k2, tables[0], 9)[:5], C.run_tokens(k, tables[0], 9)[:5])


def test_positions_follow_the_compaction():
    vis, txt = np.array([[10, 11, 12, 20, 21]]), np.array([[13, 14, 22]])
    out = C.compact_positions(vis, [0, 3, 5], txt, [0, 2, 3], [[0, 2], [1]], "packed", 0, np.full((1, 7), -1))
    assert out.tolist() == [[10, 12, 13, 14, 21, 22, -1]]
    out = C.compact_positions(vis, [0, 3, 5], txt, [0, 2, 3], [[0, 2], [1]], "padded", 5, np.full((1, 10), -1))
    assert out.tolist() == [[10, 12, 13, 14, -1, 21, 22, -1, -1, -1]]
