"""stepprune_cache_append and stepprune_compact_positions on the GPU against the
oracle (oracle/cache.py, 64 bits), and the cache's calls in a row behind the selection.

Tolerance of a rotated element x c - x' s: two products and a sum in float32 (the
fused one rounds once: two roundings in all, of at most |x c| + |x' s| each), then one
rounding to the working type: 2 U32 (|x c| + |x' s|) + half a step of the result.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import cache as oracle_cache
from paper_2609_13804_amd import binding as sp
from paper_2609_13804_amd import workloads as W
from paper_2609_13804_amd.runner import DeviceRun
from tests.cache_case import HALF_STEP, U32, Batch, device, ints, torch_type

pytestmark = pytest.mark.gpu


def angles(positions, pairs):
    a = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(pairs) / pairs)
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def append(b, rot, section=None, pos=None, interleaved=False, fused=True, queries=True, in_place=False, positions=None,
           check=True):
    """The call on b's rows; (q, k_cache, v_cache) as they come out, and the inputs."""
    Hq, Hk, D = b.Hq, b.Hk, b.D
    q, k, v = (b.values((b.rows, H, D)) for H in (Hq, Hk, Hk))
    up = lambda a: device(a, b.dtype).view(b.rows, -1)
    if fused and not in_place:
        qkv = torch.cat([up(q), up(k), up(v)], 1).contiguous()
        dq, dk, dv = qkv.split([Hq * D, Hk * D, Hk * D], 1)
    else:
        dq, dk, dv = up(q), up(k), up(v)
    cs = angles(max(b.lens + [1]) + 9 if positions is None else positions, max(1, rot // 2))
    d_cs = torch.from_numpy(cs).cuda()
    d_pos = None if pos is None else ints(pos)
    r = sp.cache_rotation(d_cs, rot, d_pos, section, interleaved) if rot else None
    q_out = dq if in_place else torch.full((b.rows, Hq * D), 7.0, dtype=torch_type(b.dtype), device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    sp.stepprune_cache_append(b.dims, dq if queries else None, dq.stride(0), dk, dk.stride(0), dv, dv.stride(0),
                              b.c_rows, b.c_runs, r, q_out if queries else None, b.d_k, b.d_v, ws, 256)
    torch.cuda.synchronize()
    code = sp.stepprune_read_device_error(ws)
    if check:
        assert code == sp.SP_DEV_OK
    back = lambda t, shape: t.double().cpu().numpy().reshape(shape)
    return (back(q_out, q.shape), back(b.d_k, b.k_cache.shape), back(b.d_v, b.v_cache.shape)), (q, k, v, cs), code


def compare(b, got, given, rot, section=None, pos=None, interleaved=False, queries=True, in_place=False):
    q, k, v, cs = given
    section = [rot // 2] if section is None else section
    turn = dict(cos_sin=cs, pos=pos, section=section, interleaved=interleaved) if rot else {}
    args = (b.first, b.counts, b.tables, b.lens)
    ref = oracle_cache.append(b.k_cache, b.v_cache, q, k, v, *args, **turn)
    # sum of the sizes of an element's two products: the same turn of |x| by (|c|, -|s|), and (|c|, |s|)
    size = [np.zeros_like(a) for a in ref]
    if rot:
        for sign in (-1.0, 1.0):
            t = dict(turn, cos_sin=np.abs(cs) * np.array([1.0, sign]))
            s = oracle_cache.append(np.zeros_like(b.k_cache), np.zeros_like(b.v_cache), np.abs(q), np.abs(k),
                                    np.abs(v), *args, **t)
            size = [np.maximum(x, y) for x, y in zip(size, s)]
    rows = b.live()
    other = np.setdiff1d(np.arange(b.rows), rows)
    if not in_place:
        assert (got[0][other] == 7.0).all()
    for i, (g, r, z) in enumerate(zip(got, ref, size)):
        if i == 0:
            if not queries:
                assert (g == 7.0).all()
                continue
            g, r, z = g[rows], r[rows], z[rows]
        assert (np.isnan(g) == np.isnan(r)).all()             # slots of no row are left alone
        d = np.where(np.isnan(r), 0.0, np.abs(g - r))
        tol = 2 * U32 * np.nan_to_num(z) + HALF_STEP[b.dtype] * np.abs(np.nan_to_num(r)) * (1 + 2.0 ** -7)
        if i == 2 or not rot:
            tol = 0 * tol                                      # copies
        assert (d <= tol).all(), (i, (d - tol).max())


CASES = [([1, 1, 1, 1, 1], [1, 16, 17, 100, 33]), ([5, 0, 33, 1, 70], [5, 0, 40, 200, 81]), ([130], [130])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["packed", "padded"])
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("interleaved", [False, True])
def test_append(gpu_lib, dtype, D, layout, case, interleaved):
    counts, lens = CASES[case]
    for rot in (D, D // 2, 16, 0):
        b = Batch(counts, lens, heads=(6, 2), D=D, dtype=dtype, layout=layout, page=32, pad=2, seed=case)
        b.upload()
        got, given, _ = append(b, rot, interleaved=interleaved)
        compare(b, got, given, rot, interleaved=interleaved)


@pytest.mark.parametrize("section", [[64], [16, 48], [16, 24, 24], [1, 0, 63], [7, 5, 52]])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_axes(gpu_lib, section, interleaved, dtype):
    b = Batch([9, 1, 3], [20, 50, 3], heads=(7, 1), dtype=dtype, seed=len(section))
    b.upload()
    pos = np.random.default_rng(1).integers(0, 300, (len(section), b.rows)).astype(np.int32)
    got, given, _ = append(b, 128, section, pos, interleaved, positions=300)
    compare(b, got, given, 128, section, pos, interleaved)


@pytest.mark.parametrize("heads", [(1, 1), (64, 8), (28, 4), (32, 32)])
def test_heads_and_queries(gpu_lib, heads):
    """Many and few heads to a wave; queries turned where they stand; none given."""
    for kw in (dict(), dict(in_place=True), dict(queries=False), dict(fused=False)):
        b = Batch([1, 40], [10, 47], heads=heads, D=64, seed=heads[0])
        b.upload()
        got, given, _ = append(b, 64, **kw)
        compare(b, got, given, 64, queries=kw.get("queries", True), in_place=kw.get("in_place", False))


def test_many_rows(gpu_lib):
    """Enough rows that a wave passes over a whole row's heads."""
    b = Batch([3000, 1200], [3000, 1300], heads=(12, 4), D=64, page=128, seed=2)
    b.upload()
    got, given, _ = append(b, 64)
    compare(b, got, given, 64)


@pytest.mark.parametrize("what", ["page", "position", "short", "offsets"])
def test_device_errors(gpu_lib, what):
    """The row or sequence at fault is left out and recorded; those before it are right."""
    b = Batch([2, 2, 2], [20, 21, 22], heads=(2, 1), D=64, seed=3)
    b.upload()
    pos = np.arange(6, dtype=np.int32)[None]
    want = {"page": sp.SP_DEV_BAD_PAGE, "position": sp.SP_DEV_BAD_POSITION, "short": sp.SP_DEV_BAD_OFFSETS,
            "offsets": sp.SP_DEV_BAD_OFFSETS}[what]
    if what == "page":
        b.d_tables[1, 1] = -5
    if what == "position":
        pos[0, 3] = 1000
    if what == "short":
        b.d_lens[1] = 1
    if what == "offsets":
        b.d_info[2] = 1
    got, given, code = append(b, 64, [32], pos, check=False)
    assert code == want
    if what == "offsets":                       # (they decide where every sequence's rows are)
        return
    ref = oracle_cache.append(b.k_cache, b.v_cache, *given[:3], b.first, b.counts, b.tables, b.lens, given[3],
                              np.minimum(pos, 9), [32])
    assert np.abs(got[0][:2] - ref[0][:2]).max() < 0.1
    assert (got[0][3] == 7.0).all()


@pytest.mark.parametrize("layout", ["padded", "packed"])
@pytest.mark.parametrize("axes", [1, 3])
def test_positions(gpu_lib, layout, axes):
    rng = np.random.default_rng(axes)
    sizes, texts = [40, 0, 300, 7], [5, 9, 0, 70]
    kept = [sorted(rng.permutation(n)[:k].tolist()) for n, k in zip(sizes, [11, 0, 290, 7])]
    off = lambda a: np.concatenate([[0], np.cumsum(a)]).astype(np.int32)
    io, to, ko = off(sizes), off(texts), off([len(k) + 1 for k in kept])
    idx = np.full(ko[-1], -1, np.int32)
    for b, k in enumerate(kept):
        idx[ko[b]:ko[b] + len(k)] = k
    vis = rng.integers(0, 9999, (axes, io[-1])).astype(np.int32)
    txt = rng.integers(0, 9999, (axes, to[-1])).astype(np.int32)
    per = 300 if layout == "padded" else 0
    rows = 4 * per if per else int(sum(map(len, kept)) + to[-1]) + 3
    pos = torch.full((axes, rows), -7, dtype=torch.int32, device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    code = sp.SP_LAYOUT_PADDED if per else sp.SP_LAYOUT_PACKED
    args = [ints(vis), int(io[-1]), ints(io), ints(txt), int(to[-1]), ints(to), axes, ints(idx), ints(ko),
            ints([len(k) for k in kept]), 4, code, per, rows]
    sp.stepprune_compact_positions(*args, pos, ws, 256)
    assert sp.stepprune_read_device_error(ws) == 0
    ref = oracle_cache.compact_positions(vis, io, txt, to, kept, layout, per, np.full((axes, rows), -7))
    assert np.array_equal(pos.cpu().numpy(), ref)
    # captured and replayed, on other positions each time
    d_vis, out = ints(vis), torch.full((axes, rows), -7, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sp.stepprune_compact_positions(d_vis, *args[1:], out, ws, 256)
    for n in (1, 2, 3):
        d_vis.copy_(ints(vis + n))
        g.replay()
        torch.cuda.synchronize()
        ref = oracle_cache.compact_positions(vis + n, io, txt, to, kept, layout, per, np.full((axes, rows), -7))
        assert np.array_equal(out.cpu().numpy(), ref)
    assert sp.stepprune_read_device_error(ws) == 0
    # what does not fit, and a kept index outside its image, are recorded
    bad = list(args)
    if per:
        bad[12], bad[13] = 289, rows
    else:
        bad[13] = rows - 4
    sp.stepprune_compact_positions(*bad, pos, ws, 256)
    assert sp.stepprune_read_device_error(ws) == sp.SP_DEV_OUTPUT_OVERFLOW
    bad = list(args)
    idx[2] = 40
    bad[7] = ints(idx)
    sp.stepprune_compact_positions(*bad, pos, ws, 256)
    assert sp.stepprune_read_device_error(ws) == sp.SP_DEV_BAD_OFFSETS


@pytest.mark.parametrize("layout", ["packed", "padded"])
def test_tokens_in_a_graph(gpu_lib, layout):
    """A captured step (append, then attend) replays while the runs grow by a token each
    time, on other streams' and eager work between the replays."""
    b = Batch([1] * 5, [3, 16, 40, 129, 15], heads=(4, 2), D=64, page=16, layout=layout, seed=4)
    b.upload(max_len=b.tables.shape[1] * 16)
    # pages for the tokens to come: those that no run has
    steps, free = 4, sorted(set(range(b.pages)) - {int(p) for p in b.tables.ravel() if p >= 0})
    for s in range(b.S):
        used = -(-b.lens[s] // 16)
        if -(-(b.lens[s] + steps) // 16) > used:
            b.tables[s, used] = free.pop()
    b.d_tables.copy_(ints(b.tables))
    Hq, Hk, D = b.Hq, b.Hk, b.D
    cs = angles(200, D // 2)
    d_cs = torch.from_numpy(cs).cuda()
    rot = sp.cache_rotation(d_cs, D)
    qkv = torch.zeros(b.rows, (Hq + 2 * Hk) * D, dtype=torch.bfloat16, device="cuda")
    dq, dk, dv = qkv.split([Hq * D, Hk * D, Hk * D], 1)
    q_out, o = (torch.full((b.rows, Hq * D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    nbytes = sp.stepprune_cache_workspace_bytes(b.dims, b.c_rows, b.c_runs)
    ws = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")

    def step():
        sp.stepprune_cache_append(b.dims, dq, dq.stride(0), dk, dk.stride(0), dv, dv.stride(0), b.c_rows, b.c_runs,
                                  rot, q_out, b.d_k, b.d_v, ws, nbytes)
        sp.stepprune_cache_attend(b.dims, q_out, Hq * D, b.c_rows, b.c_runs, None, None, b.scale, 0, b.d_k, b.d_v, o,
                                  None, ws, nbytes)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    host = lambda t, H: t.double().cpu().numpy().reshape(-1, H, D)
    for _ in range(steps):
        b.lens = [n + 1 for n in b.lens]
        b.d_lens.copy_(ints(b.lens))
        q, k, v = (b.values((b.rows, H, D)) for H in (Hq, Hk, Hk))
        qkv.copy_(torch.cat([device(t, "bf16").view(b.rows, -1) for t in (q, k, v)], 1))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (q_out, o, b.d_k, b.d_v)]
        ref = oracle_cache.append(b.k_cache, b.v_cache, q, k, v, b.first, b.counts, b.tables, b.lens, cs, None,
                                  [D // 2])
        live = b.live()
        for t, r in zip((host(got[0], Hq)[live], got[2].double().cpu().numpy(), got[3].double().cpu().numpy()),
                        (ref[0][live], ref[1], ref[2])):
            assert (np.isnan(t) == np.isnan(r)).all()
            r = np.nan_to_num(r)
            assert (np.abs(np.nan_to_num(t) - r) <= 2.0 ** -8 * np.abs(r) * 1.01 + 4 * U32 * 8).all()
        b.q = host(got[0], Hq)
        b.k_cache, b.v_cache = got[2].double().cpu().numpy(), got[3].double().cpu().numpy()
        b.check(host(got[1], Hq), None)
        step()                                          # the same tokens once more, eagerly
        torch.cuda.synchronize()
        for t, e in zip(got, (q_out, o, b.d_k, b.d_v)):
            assert torch.equal(torch.nan_to_num(t), torch.nan_to_num(e))
    assert sp.stepprune_read_device_error(ws) == 0


@pytest.mark.parametrize("name", ["tiny_bf16", "small_packed_bf16"])
def test_selection_to_attention(gpu_lib, name):
    """The calls in a row: select, compact, positions, the model's q/k/v product (torch),
    append, attend; then two questions' tokens on each image's prefix."""
    w = W.WORKLOADS[name]
    lay = W.make_layout(w)
    run = DeviceRun(w, W.make_inputs(w), lay, W.stop_bias(w))
    if run.out is None:
        pytest.skip("the workload's text has another width")
    run.run()
    T_vis, T_txt, B = run.sizes.T_vis, run.sizes.T_txt, run.sizes.B
    vis = np.concatenate([np.arange(n) for n in np.diff(lay.img_off)])[None].astype(np.int32)
    txt = np.concatenate([n + np.arange(L) for n, L in zip(np.diff(lay.img_off), np.diff(lay.text_off))])[None]
    pos = run.positions(ints(vis), ints(txt))
    kept = run.kept_lists()
    counts = [len(k) + int(L) for k, L in zip(kept, np.diff(lay.text_off))]
    ref_pos = oracle_cache.compact_positions(vis, lay.img_off, txt, lay.text_off, kept, w.layout, lay.rows_per_image,
                                             np.zeros((1, run.out_rows), np.int64))
    assert np.array_equal(pos.cpu().numpy(), ref_pos)

    Hq, Hk, D, page = 4, 2, 64, 16
    b = Batch(counts, counts, heads=(Hq, Hk), D=D, page=page, seed=1)
    b.k_cache[:], b.v_cache[:] = np.nan, np.nan
    b.upload()
    g = torch.Generator(device="cuda").manual_seed(0)
    Wm = torch.randn(w.d, (Hq + 2 * Hk) * D, device="cuda", generator=g) / w.d ** 0.5
    qkv = (torch.nan_to_num(run.out.float()) @ Wm).to(torch.bfloat16)
    q, k, v = qkv.split([Hq * D, Hk * D, Hk * D], 1)
    cs = torch.from_numpy(angles(int(ref_pos.max()) + 9, D // 2)).cuda()
    rows = run.cache_rows()
    rot = sp.cache_rotation(cs, D, pos)
    q_out = torch.full((run.out_rows, Hq * D), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(sp.stepprune_cache_workspace_bytes(b.dims, rows, b.c_runs), dtype=torch.uint8, device="cuda")
    sp.stepprune_cache_append(b.dims, q, q.stride(0), k, k.stride(0), v, v.stride(0), rows, b.c_runs, rot, q_out,
                              b.d_k, b.d_v, ws, ws.numel())
    o = torch.full((run.out_rows, Hq * D), 7.0, dtype=torch.bfloat16, device="cuda")
    sp.stepprune_cache_attend(b.dims, q_out, Hq * D, rows, b.c_runs, None, None, b.scale, 0, b.d_k, b.d_v, o, None,
                              ws, ws.numel())
    assert sp.stepprune_read_device_error(ws) == 0
    # the oracle on the model's rows, then its attention on the appended cache
    host = lambda t, H: t.double().cpu().numpy().reshape(-1, H, D)
    first = [i * lay.rows_per_image for i in range(B)] if w.layout == "padded" else \
        [int(f) for f in run.seq_info.cpu().numpy()[:-1]]
    rq, rk, rv = oracle_cache.append(b.k_cache, b.v_cache, host(q, Hq), host(k, Hk), host(v, Hk), first, counts,
                                     b.tables, b.lens, cs.cpu().numpy(), ref_pos, [D // 2])
    gk, gv = b.d_k.double().cpu().numpy(), b.d_v.double().cpu().numpy()
    live = np.concatenate([np.arange(f, f + n) for f, n in zip(first, counts)])
    close = lambda a, r: (np.abs(a - r) <= 2.0 ** -7 * np.abs(r) + 2.0 ** -8 * 1e-3).all()
    gq = host(q_out, Hq)
    assert close(gq[live], rq[live]) and close(gk[np.isfinite(rk)], rk[np.isfinite(rk)])
    assert (np.isnan(gk) == np.isnan(rk)).all() and (np.isnan(gv) == np.isnan(rv)).all()
    ref, _ = oracle_cache.attend(np.where(np.isfinite(gq), gq, 0), gk, gv, first, counts, b.tables, b.lens, b.scale)
    A, _ = oracle_cache.attend(np.where(np.isfinite(gq), gq, 0), gk, np.abs(gv), first, counts, b.tables, b.lens, b.scale)
    got = host(o, Hq)
    assert (np.abs(got[live] - ref[live]) <= (2.0 ** -8 + 2.0 ** -10) * A[live] + 2.0 ** -8 * np.abs(ref[live])).all()
    assert (got[np.setdiff1d(np.arange(run.out_rows), live)] == 7.0).all()

    # two questions on each image: the image's run is the prefix, one token a question
    S = 2 * B
    c = Batch([1] * S, [1] * S, heads=(Hq, Hk), D=D, page=page, spare=0, seed=2)
    c.pages = b.pages + S
    c.k_cache = np.concatenate([gk, np.full((S,) + gk.shape[1:], np.nan)])
    c.v_cache = np.concatenate([gv, np.full((S,) + gv.shape[1:], np.nan)])
    c.tables = np.asarray([[b.pages + s] for s in range(S)], np.int32)
    c.prefix, c.prefix_tables, c.cuts = counts, b.tables, list(range(0, S + 1, 2))
    c.upload()
    k1, v1 = c.values((S, Hk, D)), c.values((S, Hk, D))
    dk, dv = device(k1, "bf16").view(S, -1), device(v1, "bf16").view(S, -1)
    sp.stepprune_cache_append(c.dims, None, 0, dk, Hk * D, dv, Hk * D, c.c_rows, c.c_runs, None, None, c.d_k, c.d_v,
                              ws, ws.numel())
    c.k_cache, c.v_cache = c.d_k.double().cpu().numpy(), c.d_v.double().cpu().numpy()
    c.check(*c.attend())
