"""stepprune_cache_attend on the GPU against the oracle (oracle/cache.py, 64 bits).

Tolerances are tests/cache_case.py's, derived there.  The sizes are those at which the
work changes hands: blocks of 16 and 32 keys, tiles of 32 and 128 (row, head) pairs,
pages, chunks of keys, rows without a key.
"""
import numpy as np
import pytest
import torch

from tests.cache_case import Batch, device, ints, torch_type
from paper_2609_13804_amd import binding as sp

pytestmark = pytest.mark.gpu

LENS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 700]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [(2, 2), (7, 1), (8, 2)])
def test_single_tokens(gpu_lib, dtype, D, heads):
    b = Batch([1] * len(LENS), LENS, heads=heads, D=D, dtype=dtype, seed=D + heads[0])
    b.upload()
    b.check(*b.attend())


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_page_sizes(gpu_lib, page, dtype):
    b = Batch([1, 3, 1, 40], [page, page + 1, 3 * page - 1, 2 * page + 40], heads=(4, 2), D=64, page=page,
              dtype=dtype, layout="padded", prefix=[page - 1, page + 5], cuts=[0, 2, 4], pad=2, seed=page)
    b.upload()
    b.check(*b.attend(ld_extra=24))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["packed", "padded"])
def test_prompts(gpu_lib, dtype, D, layout):
    """Prompts of many lengths behind tokens of earlier calls; some sequences have no row,
    one has rows whose keys are not there (they see nothing)."""
    counts = [5, 0, 33, 64, 100, 1, 7, 130, 3]
    lens = [5, 40, 33, 200, 163, 9, 4, 131, 0]
    b = Batch(counts, lens, heads=(4, 2), D=D, dtype=dtype, layout=layout, pad=3, seed=7)
    b.upload()
    b.check(*b.attend())
    b.check(*b.attend(see_all=True), see_all=True)


@pytest.mark.parametrize("heads", [(40, 1), (64, 1), (33, 1), (28, 4), (5, 5)])
@pytest.mark.parametrize("D", [64, 128])
def test_head_groups(gpu_lib, heads, D):
    """More query heads to a key head than a tile has pairs, and odd numbers of them."""
    b = Batch([1, 2, 1, 5], [70, 300, 31, 5], heads=heads, D=D, seed=heads[0])
    b.upload()
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["packed", "padded"])
@pytest.mark.parametrize("prefix", [[0, 1, 16], [33, 600, 128], [257, 31, 64]])
def test_shared_prefixes(gpu_lib, dtype, layout, prefix):
    """Groups of several sequences, an empty group, sequences outside every group; tokens
    and short prompts together; runs of no token (cross attention)."""
    counts = [1, 1, 1, 9, 1, 2, 1, 0, 1]
    lens = [40, 1, 300, 9, 0, 30, 17, 50, 5]
    b = Batch(counts, lens, heads=(8, 2), dtype=dtype, layout=layout, prefix=[prefix[0], 7, prefix[1], prefix[2]],
              cuts=[1, 3, 3, 6, 8], pad=1, seed=prefix[0] + len(layout))
    b.upload()
    b.check(*b.attend())
    b.check(*b.attend(see_all=True), see_all=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("per_group", [2, 40])
def test_large_groups(gpu_lib, D, per_group):
    """Prefix rows in tall tiles (many sequences to a group) and in thin ones, the prefix
    in several chunks."""
    S = 2 * per_group
    b = Batch([1] * S, [1 + (7 * s) % 50 for s in range(S)], heads=(8, 2), D=D, prefix=[1500, 1111],
              cuts=[0, per_group, S], seed=per_group)
    b.upload()
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[1, 9], [3, 1, 11, 2]])
def test_empty_groups_behind_the_last(gpu_lib, dtype, counts):
    """Groups without a sequence at the end of the batch, behind a group of several tiles."""
    S = len(counts)
    b = Batch(counts, [n + 20 for n in counts], heads=(8, 2), dtype=dtype, prefix=[40, 90, 33, 5, 70],
              cuts=[0, 0, S - 1, S, S, S], seed=S)
    b.upload()
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["packed", "padded"])
@pytest.mark.parametrize("longest", [5, 90])
def test_more_segments_than_lanes(gpu_lib, dtype, layout, longest):
    """More than 64 sequences and more than 64 groups, of tokens, short and longer prompts."""
    S = 150
    counts = [(5 * s) % 4 for s in range(S)]
    for s in range(3, S, 9):
        counts[s] = longest - s % 5
    cuts = sorted([0, 2, 2] + list(range(4, 146, 2)) + [149])
    G = len(cuts) - 1
    b = Batch(counts, [n + (11 * s) % 60 for s, n in enumerate(counts)], heads=(4, 2), D=64, dtype=dtype, layout=layout,
              prefix=[(29 * g) % 140 for g in range(G)], cuts=cuts, seed=longest)
    assert G > 64
    b.upload()
    b.check(*b.attend())
    b.check(*b.attend(see_all=True), see_all=True)


def test_padded_slices_of_no_rows(gpu_lib):
    """Padded slices of no row: nothing is written, whatever rows the arrays have."""
    b = Batch([0, 0], [40, 700], heads=(4, 2), D=64, layout="padded", prefix=[30], cuts=[0, 2], seed=2)
    b.upload()
    assert b.per_seq == 0
    b.rows = 5
    b.q = np.ones((5, 4, 64))
    b.c_rows = sp.cache_rows(5, sp.SP_LAYOUT_PADDED, 0, b.d_info, 3)
    o, lse = b.attend()
    assert (o == 7.0).all() and (lse == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_runs_without_a_table(gpu_lib, dtype):
    """Runs of no token: their table may be NULL, whatever its width."""
    b = Batch([1, 3, 40], [0, 0, 0], heads=(4, 4), D=64, dtype=dtype, prefix=[77, 300], cuts=[0, 1, 3], seed=3)
    b.upload()
    b.c_runs.table, b.c_runs.table_width = None, 4
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("longest", [192, 2200])
def test_many_heads_and_sequences(gpu_lib, dtype, longest):
    """So many sequences and key heads that, while runs are short, each wave takes a head by
    itself; lengths from none to several chunks, some rows in groups."""
    S = 40
    lens = [(37 * s) % 90 for s in range(S)]
    lens[3], lens[11] = longest, 177
    b = Batch([1 + (s % 7 == 0) for s in range(S)], lens, heads=(64, 64), D=64, dtype=dtype, prefix=[50, 333],
              cuts=[2, 20, 31], seed=13)
    b.upload()
    b.check(*b.attend())
    dirty = Batch([2] * S, [2 + n for n in lens[:3]] + [40] * (S - 3), heads=(64, 64), D=64, dtype=dtype, seed=14)
    dirty.v_cache[dirty.tables[5][39 // 16], :, 39 % 16] = np.nan          # the last token of one run
    dirty.upload()
    o, lse = dirty.attend()
    assert np.isfinite(o[10]).all() and np.isnan(o[11]).all() and np.isfinite(np.delete(o, 11, 0)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cross_attention(gpu_lib, dtype):
    """Runs of no token at all: every row attends to its group's prefix alone."""
    b = Batch([20, 3, 50], [0, 0, 0], heads=(4, 4), D=64, dtype=dtype, prefix=[77, 300], cuts=[0, 1, 2], seed=3)
    b.upload()
    o, lse = b.attend()
    b.check(o, lse)
    assert (o[23:73] == 0).all() and np.isneginf(lse[23:73]).all()       # the last sequence has no group


def test_long_run_in_parts(gpu_lib):
    """A run over many chunks, joined; also with bounds far above the lengths."""
    b = Batch([1, 2], [9001, 37], heads=(7, 1), seed=11)
    b.upload()
    b.check(*b.attend())
    b.upload(max_len=b.tables.shape[1] * b.page, max_rows=2)
    b.check(*b.attend())


@pytest.mark.parametrize("layout", ["packed", "padded"])
@pytest.mark.parametrize("longest", [1300, 6001])
@pytest.mark.parametrize("prefix", [(), (700, 90)])
def test_prompts_and_tokens_in_parts(gpu_lib, layout, longest, prefix):
    """A few rows over long runs beside single tokens: the parts of both kinds of sequences,
    few and many of them, joined in one launch."""
    counts, lens = [40, 1, 3, 17, 0], [longest, longest - 7, 70, 500, 9]
    b = Batch(counts, lens, heads=(4, 1), D=64, page=32, layout=layout, prefix=prefix,
              cuts=[0, 2, 4] if prefix else (), seed=longest)
    b.upload()
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("D", [64, 128])
def test_hidden_tokens_have_no_influence(gpu_lib, dtype, bad, D):
    """Keys and values that are infinite or NaN at tokens that only later rows see: the
    rows before them get what they get without them, bit for bit."""
    n, L = 70, 100
    make = lambda: Batch([n], [L], heads=(4, 2), D=D, dtype=dtype, seed=5)
    clean, dirty = make(), make()
    at = L - n + 41                               # seen by rows 41 .. only
    for b, what in ((clean, 0.0), (dirty, bad)):
        where = b.tables[0][at // b.page], slice(None), at % b.page
        b.v_cache[where] = what
        if b is dirty:
            b.k_cache[where][0, ::3] = bad
        b.upload()
    oc, lc = clean.attend()
    od, ld = dirty.attend()
    tol, tol_l = clean.bounds(*clean.oracle())
    assert (np.abs(od[:41] - oc[:41]) <= 2 * tol[:41]).all()
    assert np.isfinite(od[:41]).all() and (np.abs(ld[:41] - lc[:41]) <= 2 * tol_l[:41]).all()
    assert not np.isfinite(od[41:, :2]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("longest", [130, 760, 1900])
def test_few_short_sequences(gpu_lib, dtype, D, longest):
    """A few sequences of one to eight rows, runs from none to several blocks a wave, some of
    less tokens than rows; tokens that only the last row sees are NaN in one of them."""
    counts, lens = [1, 8, 0, 3, 8, 2, 8], [0, 3, 9, longest, longest - 2, 2, 129]
    b = Batch(counts, lens, heads=(4, 2), D=D, dtype=dtype, layout="padded", pad=1, seed=D)
    b.upload()
    b.check(*b.attend())
    b.check(*b.attend(see_all=True), see_all=True)
    clean, _ = b.attend()
    tol, _ = b.bounds(*b.oracle())
    b.v_cache[b.tables[4][(lens[4] - 1) // 16], :, (lens[4] - 1) % 16] = np.nan
    b.upload()
    o, _ = b.attend()
    last = b.first[4] + 7
    assert np.isnan(o[last]).all()
    rows = np.setdiff1d(b.live(), [last])
    assert np.isfinite(o[rows]).all() and (np.abs(o[rows] - clean[rows]) <= 2 * tol[rows]).all()
    none = Batch([1, 2], [0, 0], heads=(4, 2), D=D, dtype=dtype)           # no token at all
    none.upload()
    none.c_runs.table = None
    o, lse = none.attend()
    assert (o == 0).all() and np.isneginf(lse).all()


def test_infinite_scores(gpu_lib):
    """A key that scores -inf weighs nothing, also when it comes first; rows whose every
    score is -inf give zeros."""
    b = Batch([1, 1], [40, 3], heads=(2, 2), D=64, seed=9)
    b.q = np.abs(b.q)
    for s, tokens in ((0, range(33)), (1, range(3))):
        for p in tokens:
            b.k_cache[b.tables[s][p // 16], :, p % 16, 0] = -np.inf
    b.upload()
    o, lse = b.attend()
    assert np.isfinite(o).all()
    assert (o[1] == 0).all() and np.isneginf(lse[1]).all()
    c = Batch([1, 1], [40, 3], heads=(2, 2), D=64, seed=9)
    c.q = b.q
    K = np.stack([c.k_cache[c.tables[0][p // 16], :, p % 16] for p in range(33, 40)])
    V = np.stack([c.v_cache[c.tables[0][p // 16], :, p % 16] for p in range(33, 40)])
    for h in range(2):
        p = np.exp(c.scale * K[:, h] @ c.q[0, h])
        ref = p @ V[:, h] / p.sum()
        assert np.abs(o[0, h] - ref).max() <= 2.0 ** -7 * (p @ np.abs(V[:, h]) / p.sum()).max()


def test_no_lse_and_same_bits(gpu_lib):
    b = Batch([1, 9, 60], [500, 333, 60], heads=(8, 2), prefix=[200], cuts=[0, 3], seed=4)
    b.upload()
    o, lse = b.attend()
    o2, _ = b.attend(lse=False)
    assert np.array_equal(o, o2)
    o3, lse3 = b.attend()
    assert np.array_equal(o, o3) and np.array_equal(lse, lse3)


def test_offsets_past_32_bits(gpu_lib):
    """Pages at the end of a cache of more than 2^32 bytes and 2^31 elements a side."""
    Hk, D, page = 8, 128, 256
    b = Batch([1, 4], [700, 300], heads=(8, 8), D=D, page=page, seed=21, spare=0)
    pages = (1 << 31) // (Hk * page * D) + b.pages + 5
    b.upload()
    small_k, small_v = b.d_k, b.d_v
    shape = (pages, Hk, page, D)
    b.d_k = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    b.d_v = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    shift = pages - b.pages
    b.d_k[shift:], b.d_v[shift:] = small_k, small_v
    b.d_tables += shift
    b.d_tables[ints(b.tables) < 0] = -1
    b.dims = sp.cache_dims(b.Hq, b.Hk, D, b.code(), page, pages)
    b.check(*b.attend())


@pytest.mark.parametrize("what", ["page", "len", "rows", "offsets", "group", "prefix_page"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_device_errors(gpu_lib, what, dtype):
    """Entries that contradict the bounds are recorded; the sequences beside them are right."""
    b = Batch([1, 2, 1], [50, 40, 30], heads=(4, 2), D=64, dtype=dtype, prefix=[20], cuts=[1, 2], seed=6)
    b.upload()
    want = {"page": sp.SP_DEV_BAD_PAGE, "prefix_page": sp.SP_DEV_BAD_PAGE, "len": sp.SP_DEV_GROUP_TOO_LARGE,
            "rows": sp.SP_DEV_GROUP_TOO_LARGE, "offsets": sp.SP_DEV_BAD_OFFSETS, "group": sp.SP_DEV_BAD_OFFSETS}[what]
    if what == "page":
        b.d_tables[1, 1] = b.pages
    if what == "prefix_page":
        b.d_ptables[0, 0] = -1
    if what == "len":
        b.d_lens[1] = 51
    if what == "rows":
        b.c_rows.max_rows = 1
    if what == "offsets":
        b.d_info[2] = 0
    if what == "group":
        b.d_off[1] = 9
    o, lse = b.attend(check=False)
    assert sp.stepprune_read_device_error(b.ws) == want
    ref, _ = b.oracle()
    if what not in ("offsets",):
        tol, _ = b.bounds(ref, _)
        assert (np.abs(o[0] - ref[0]) <= tol[0]).all()


def test_errors_of_prefixes_bounded_by_nothing(gpu_lib):
    """Groups' entries are looked at also where the prefixes' bound leaves them no token."""
    for what, want in (("len", sp.SP_DEV_GROUP_TOO_LARGE), ("group", sp.SP_DEV_BAD_OFFSETS)):
        b = Batch([1, 1], [50, 40], heads=(4, 2), D=64, prefix=[20], cuts=[0, 2], seed=6)
        b.upload(max_prefix=0)
        if what == "group":
            b.d_plens.zero_()
            b.d_off[1] = 3
        b.attend(check=False)
        assert sp.stepprune_read_device_error(b.ws) == want


def test_other_stream_and_graph(gpu_lib):
    """A captured call replays on lengths that grow within the bounds, with eager work
    between the replays."""
    b = Batch([1] * 6, [300, 20, 129, 64, 7, 255], heads=(8, 2), prefix=[150], cuts=[0, 4], seed=8)
    b.upload()
    full = [int(n) for n in b.lens]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        o, lse = b.attend(stream=side)
    b.check(o, lse)
    q = device(b.q, "bf16").view(b.rows, -1)
    out = torch.zeros_like(q)
    nbytes = sp.stepprune_cache_workspace_bytes(b.dims, b.c_rows, b.c_runs, b.c_prefix)
    ws = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")
    call = lambda: sp.stepprune_cache_attend(b.dims, q, q.shape[1], b.c_rows, b.c_runs, b.c_prefix, b.d_off, b.scale,
                                             0, b.d_k, b.d_v, out, None, ws, nbytes)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for back in (6, 3, 1, 0, 0):
        b.lens = [n - back for n in full]
        b.d_lens.copy_(ints(b.lens))
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        b.check(got.double().cpu().numpy().reshape(b.rows, b.Hq, b.D), None)
        out.fill_(7.0)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
    assert sp.stepprune_read_device_error(ws) == 0


def test_two_streams_at_once(gpu_lib):
    """Two batches on two streams, each with its own workspace, get what they get alone."""
    batches = [Batch([1] * 9, [900 + 7 * s for s in range(9)], heads=(8, 2), prefix=[700], cuts=[0, 9], seed=1),
               Batch([130, 60, 1], [700, 60, 300], heads=(8, 2), seed=2)]
    calls, alone, outs = [], [], []
    for b in batches:
        b.upload()
        o, lse = b.attend()
        b.check(o, lse)
        q = device(b.q, "bf16").view(b.rows, -1)
        out = torch.full_like(q, 7.0)
        nbytes = sp.stepprune_cache_workspace_bytes(b.dims, b.c_rows, b.c_runs, b.c_prefix)
        ws = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")
        calls.append(lambda b=b, q=q, out=out, ws=ws, nbytes=nbytes: sp.stepprune_cache_attend(
            b.dims, q, q.shape[1], b.c_rows, b.c_runs, b.c_prefix, b.d_off, b.scale, 0, b.d_k, b.d_v, out, None, ws,
            nbytes))
        alone.append(o)
        outs.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    for _ in range(8):
        for call, stream in zip(calls, streams):
            with torch.cuda.stream(stream):
                call()
    torch.cuda.synchronize()
    for b, o, out in zip(batches, alone, outs):
        assert np.array_equal(out.double().cpu().numpy().reshape(o.shape)[b.live()], o[b.live()])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["packed", "padded"])
@pytest.mark.parametrize("prefix", [[1, 0, 129], [128, 400, 17], [500, 3, 383]])
def test_few_sequences_with_their_prefixes(gpu_lib, D, layout, prefix):
    """Few sequences that each take their prefix themselves: groups of several and of none,
    sequences outside every group, runs of no token, rows whose last token is NaN for the
    last of them alone, NaN behind every run's and prefix's end."""
    counts, lens = [1, 4, 1, 0, 3, 1, 4], [90, 4, 0, 5, 100, 17, 60]
    b = Batch(counts, lens, heads=(8, 2), D=D, layout=layout, prefix=prefix, cuts=[1, 3, 3, 6], pad=1, seed=D)
    b.upload()
    clean, _ = b.attend()
    b.check(clean, _)
    b.check(*b.attend(see_all=True), see_all=True)
    tol, _ = b.bounds(*b.oracle())
    b.v_cache[b.tables[4][99 // 16], :, 99 % 16] = np.inf
    b.upload()
    o, _ = b.attend()
    last = b.first[4] + 2
    assert not np.isfinite(o[last]).any()
    rows = np.setdiff1d(b.live(), [last])
    assert np.isfinite(o[rows]).all() and (np.abs(o[rows] - clean[rows]) <= 2 * tol[rows]).all()
