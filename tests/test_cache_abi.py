"""The cache's calls on the host: what they refuse before any device work (the pointers
are fake and never dereferenced), the workspace query, and, of the generated code of
csrc/attend.hip, what its direct-to-LDS loads rely on.
"""
import os
import re
import subprocess

import pytest

from paper_2609_13804_amd import build as B
from tests.test_codegen import IMPLICIT_M0, _instructions

FAKE, MISALIGNED = 0x10000, 0x10008
OTHER = 0x20000


@pytest.fixture(scope="module")
def sp():
    from paper_2609_13804_amd import binding
    return binding


class Table:                     # what cache_runs asks of a tensor
    def __init__(self, count, width, ptr=FAKE):
        self.shape, self.ptr = (count, width), ptr

    def data_ptr(self):
        return self.ptr


def _dims(sp, **kw):
    a = dict(q_heads=8, kv_heads=2, head_dim=128, dtype=sp.SP_BF16, page_size=16, pages=10)
    a.update(kw)
    return sp.cache_dims(**a)


def _rows(sp, **kw):
    a = dict(rows=4, layout=sp.SP_LAYOUT_PACKED, rows_per_seq=0, seq_info=FAKE, max_rows=4)
    a.update(kw)
    return sp.cache_rows(**a)


def _runs(sp, count=2, width=3, max_len=48, ptr=FAKE, len_ptr=FAKE):
    return sp.cache_runs(Table(count, width, ptr), len_ptr, max_len)


def _rot(sp, **kw):
    class T:
        shape = (100, 64, 2)

        def data_ptr(self):
            return kw.get("cos_sin", FAKE)
    r = sp.cache_rotation(T(), kw.get("rot_dim", 128), kw.get("pos"), kw.get("section"))
    for k in ("positions", "interleaved", "axes"):
        if k in kw:
            setattr(r, k, kw[k])
    return r


DIMS = [(dict(q_heads=0), "EINVAL"), (dict(kv_heads=0), "EINVAL"), (dict(kv_heads=3), "EINVAL"),
        (dict(q_heads=1026, kv_heads=2), "EUNSUPPORTED"), (dict(head_dim=96), "EUNSUPPORTED"),
        (dict(head_dim=0), "EINVAL"), (dict(dtype=2), "EUNSUPPORTED"), (dict(page_size=8), "EUNSUPPORTED"),
        (dict(page_size=48), "EUNSUPPORTED"), (dict(page_size=512), "EUNSUPPORTED"), (dict(page_size=0), "EINVAL"),
        (dict(pages=0), "EINVAL")]
ROWS = [(dict(rows=-1), "EINVAL"), (dict(max_rows=-1), "EINVAL"), (dict(layout=2), "EINVAL"),
        (dict(seq_info=0), "EINVAL"), (dict(layout=0, rows_per_seq=3), "EINVAL"),
        (dict(layout=0, rows_per_seq=-1), "EINVAL"), (dict(rows=1 << 26), "EUNSUPPORTED"),
        (dict(rows=(1 << 23) + 1), "EUNSUPPORTED")]
RUNS = [(dict(count=-1), "EINVAL"), (dict(max_len=49), "EINVAL"), (dict(max_len=-1), "EINVAL"),
        (dict(width=(1 << 26) + 1, max_len=(1 << 30) + 1), "EUNSUPPORTED"),
        (dict(count=(1 << 24) + 1), "EUNSUPPORTED"), (dict(ptr=0), "EINVAL"), (dict(len_ptr=0), "EINVAL"),
        (dict(width=-1, max_len=0), "EINVAL")]


def _append(sp, dims=None, rows=None, runs=None, **kw):
    a = dict(Q=FAKE, ldq=1024, K=FAKE, ldk=256, V=FAKE, ldv=256, rot=_rot(sp), Q_out=OTHER, k_cache=FAKE,
             v_cache=FAKE, ws=FAKE, ws_bytes=0)
    a.update(kw)
    return sp.stepprune_cache_append(dims or _dims(sp), a["Q"], a["ldq"], a["K"], a["ldk"], a["V"], a["ldv"],
                                     rows or _rows(sp), runs or _runs(sp), a["rot"], a["Q_out"], a["k_cache"],
                                     a["v_cache"], a["ws"], a["ws_bytes"], stream=0, raise_on_error=False)


def _attend(sp, dims=None, rows=None, runs=None, **kw):
    a = dict(Q=FAKE, ldq=1024, prefix=None, grp_off=None, scale=0.1, flags=0, k_cache=FAKE, v_cache=FAKE, O=OTHER,
             lse=None, ws=FAKE, ws_bytes=0)
    a.update(kw)
    return sp.stepprune_cache_attend(dims or _dims(sp), a["Q"], a["ldq"], rows or _rows(sp), runs or _runs(sp),
                                     a["prefix"], a["grp_off"], a["scale"], a["flags"], a["k_cache"], a["v_cache"],
                                     a["O"], a["lse"], a["ws"], a["ws_bytes"], stream=0, raise_on_error=False)


@pytest.mark.parametrize("call", [_append, _attend])
def test_structs_are_checked(sp, call):
    """Everything in order comes as far as the workspace's size."""
    assert call(sp) == sp.SP_EWORKSPACE
    for make, name, cases in ((_dims, "dims", DIMS), (_rows, "rows", ROWS), (_runs, "runs", RUNS)):
        for kw, want in cases:
            assert call(sp, **{name: make(sp, **kw)}) == getattr(sp, "SP_" + want), (name, kw)


def test_append_refusals(sp):
    for kw in (dict(Q=0), dict(Q_out=0), dict(K=0), dict(V=0), dict(k_cache=0), dict(v_cache=0), dict(ws=0),
               dict(Q=MISALIGNED), dict(K=MISALIGNED), dict(V=MISALIGNED), dict(Q_out=MISALIGNED),
               dict(k_cache=MISALIGNED), dict(v_cache=MISALIGNED), dict(ws=MISALIGNED), dict(ldq=1016),
               dict(ldk=248), dict(ldv=248), dict(ldq=1028), dict(ldk=260), dict(ldv=260), dict(Q_out=FAKE, ldq=1032)):
        assert _append(sp, **kw) == sp.SP_EINVAL, kw
    assert _append(sp, Q=0, Q_out=0) == sp.SP_EWORKSPACE                       # keys and values only
    assert _append(sp, Q_out=FAKE) == sp.SP_EWORKSPACE                         # in place
    assert _append(sp, rot=None) == sp.SP_EWORKSPACE
    for kw in (dict(cos_sin=0), dict(cos_sin=MISALIGNED), dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=144),
               dict(positions=0), dict(interleaved=2), dict(axes=2), dict(axes=0), dict(section=[60]),
               dict(pos=FAKE, section=[30, 20]), dict(pos=FAKE, section=[65, -1]),
               dict(pos=FAKE, section=[16, 24, 24], axes=4)):
        assert _append(sp, rot=_rot(sp, **kw)) == sp.SP_EINVAL, kw
    assert _append(sp, rot=_rot(sp, pos=FAKE, section=[16, 24, 24])) == sp.SP_EWORKSPACE


def test_attend_refusals(sp):
    for kw in (dict(Q=0), dict(O=0), dict(O=FAKE), dict(k_cache=0), dict(v_cache=0), dict(ws=0), dict(Q=MISALIGNED),
               dict(O=MISALIGNED), dict(k_cache=MISALIGNED), dict(v_cache=MISALIGNED), dict(ws=MISALIGNED),
               dict(ldq=1016), dict(ldq=1028), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(scale=1e-44), dict(scale=3e38), dict(flags=2), dict(prefix=_runs(sp)),
               dict(grp_off=FAKE)):
        assert _attend(sp, **kw) == sp.SP_EINVAL, kw
    ok = dict(prefix=_runs(sp, count=1), grp_off=FAKE)
    assert _attend(sp, **ok) == sp.SP_EWORKSPACE
    for kw, want in RUNS:
        assert _attend(sp, prefix=_runs(sp, **kw), grp_off=FAKE) == getattr(sp, "SP_" + want), kw


def test_workspace_query(sp):
    ws = lambda **kw: sp.stepprune_cache_workspace_bytes(kw.pop("dims", _dims(sp)), kw.pop("rows", _rows(sp)),
                                                         kw.pop("runs", _runs(sp)), kw.pop("prefix", None))
    base = ws()
    assert base >= 256 + 4 * 4
    # few sequences take a short prefix by themselves: no parts; of a long one, a part of the
    # prefix and of the row's own run: m, l and the output of every (row, head)
    assert ws(prefix=_runs(sp, count=1)) == base
    assert ws(prefix=_runs(sp, count=1, width=1 << 10, max_len=4096)) >= 256 + 4 * 4 + 4 * 8 * 2 * (128 + 2) * 4
    long = _runs(sp, count=1, width=1 << 16, max_len=1 << 20)
    assert ws(runs=long) > base
    for kw, _ in DIMS:
        assert ws(dims=_dims(sp, **kw)) == 0, kw
    for kw, _ in ROWS:
        if "seq_info" not in kw:
            assert ws(rows=_rows(sp, **kw)) == 0, kw
    assert ws(runs=_runs(sp, max_len=49)) == 0
    assert ws(runs=_runs(sp, ptr=0, len_ptr=0)) == base            # device pointers are not read


def test_largest_bounds(sp):
    """Bounds at their limits: the split stays within its integers, and what no launch holds
    is refused."""
    ws = lambda rows, runs, prefix, **kw: sp.stepprune_cache_workspace_bytes(_dims(sp, **kw), rows, runs, prefix)
    long = lambda n: _runs(sp, count=n, width=1 << 22, max_len=1 << 30)
    for heads in (1, 8, 1024):
        kw = dict(q_heads=heads, kv_heads=heads, page_size=256)
        n = ws(_rows(sp, rows=64, max_rows=64), long(1), long(1), **kw)       # parts of each (row, head)
        assert 0 < n <= 3 * 64 * heads * 1024 * 130 * 4 + 4096, (heads, n)
    # many items: one chunk would be prefix and run together, 2^31 keys
    many = dict(q_heads=1024, kv_heads=1024, page_size=256)
    n = ws(_rows(sp, rows=64, max_rows=64), long(1), long(1), **many)
    assert 0 < n < 1 << 36, n
    # a wave to each (row, head) to join with the prefix
    big = dict(q_heads=1024, kv_heads=1024, page_size=16, dtype=sp.SP_F32)
    few = _runs(sp, count=1)
    assert ws(_rows(sp, rows=1 << 15, max_rows=1 << 15), few, few, **big) > 0
    assert ws(_rows(sp, rows=1 << 17, max_rows=1 << 17), few, few, **big) == 0
    assert _attend(sp, dims=_dims(sp, **big), rows=_rows(sp, rows=1 << 17, max_rows=1 << 17), ldq=1 << 17,
                   prefix=few, grp_off=FAKE) == sp.SP_EUNSUPPORTED
    # 2^24 and more workgroups for the tokens: with a wave to a head a quarter of the heads each
    assert ws(_rows(sp, rows=1 << 15, max_rows=1), _runs(sp, count=1 << 15), None, **big) > 0
    assert ws(_rows(sp, rows=1 << 16, max_rows=1), _runs(sp, count=1 << 16), None, **big) == 0
    # runs of no tokens need no table
    assert _attend(sp, runs=_runs(sp, ptr=0, max_len=0)) == sp.SP_EWORKSPACE


def test_no_rows_is_no_work(sp):
    """Nothing to do is not an error, and nothing is launched (there is no GPU here)."""
    n = 1 << 20
    for rows, runs in ((_rows(sp, rows=0), _runs(sp)), (_rows(sp), _runs(sp, count=0))):
        assert _append(sp, rows=rows, runs=runs, ws_bytes=n) == sp.SP_OK
        assert _attend(sp, rows=rows, runs=runs, ws_bytes=n) == sp.SP_OK


def test_positions_refusals(sp):
    def call(**kw):
        a = dict(vis=FAKE, T_vis=10, img_off=FAKE, txt=FAKE, T_txt=5, text_off=FAKE, axes=1, idx=FAKE, off=FAKE,
                 cnt=FAKE, B=2, layout=1, per=0, out=15, pos=FAKE, ws=FAKE, ws_bytes=0)
        a.update(kw)
        return sp.stepprune_compact_positions(a["vis"], a["T_vis"], a["img_off"], a["txt"], a["T_txt"], a["text_off"],
                                              a["axes"], a["idx"], a["off"], a["cnt"], a["B"], a["layout"], a["per"],
                                              a["out"], a["pos"], a["ws"], a["ws_bytes"], stream=0,
                                              raise_on_error=False)
    assert call() == sp.SP_EWORKSPACE
    for kw in (dict(vis=0), dict(txt=0), dict(img_off=0), dict(text_off=0), dict(idx=0), dict(off=0), dict(cnt=0),
               dict(pos=0), dict(ws=0), dict(ws=MISALIGNED), dict(B=0), dict(T_vis=-1), dict(T_txt=-1), dict(out=-1),
               dict(axes=0), dict(axes=4), dict(layout=2), dict(layout=0, per=8), dict(layout=0, per=-1)):
        assert call(**kw) == sp.SP_EINVAL, kw


def test_m0_is_written_only_by_the_lds_load(tmp_path):
    """As for the other users of the direct-to-LDS load: M0 is set by its own statement
    alone and read by nothing else."""
    dst = str(tmp_path / "attend.s")
    flags = [f for f in B.HIPCC_FLAGS if f != "-fPIC"]
    r = subprocess.run([B._hipcc(), *flags, *B.EXTRA_FLAGS.get("attend.hip", []), "--cuda-device-only", "-S",
                        os.path.join(B.CSRC, "attend.hip"), "-o", dst], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    ins = list(_instructions(open(dst).read().splitlines()))
    writes = 0
    for k, (_, s) in enumerate(ins):
        assert not IMPLICIT_M0.match(s), s
        ops = s.split(None, 1)
        if len(ops) == 2 and re.match(r"m0\s*,", ops[1]):
            assert re.fullmatch(r"s_mov_b32\s+m0,\s*s\d+", s), s
            assert ins[k + 1][1] == "s_nop 0", ins[k + 1][1]
            assert ins[k + 2][1].startswith("global_load_lds_dwordx4"), ins[k + 2][1]
            writes += 1
    assert writes > 0
