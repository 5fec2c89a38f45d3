"""The cache's structs as binding.py makes them from tensors (CPU: the structs hold
addresses only, nothing is launched).
"""
import gc
import weakref

import pytest
import torch


@pytest.fixture(scope="module")
def sp():
    from paper_2609_13804_amd import binding
    return binding


def _ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


STRUCTS = {
    "rows": lambda sp, t: sp.cache_rows(4, sp.SP_LAYOUT_PACKED, 0, t("info", _ints(3)), 4),
    "runs": lambda sp, t: sp.cache_runs(t("table", _ints(2, 3)), t("len", _ints(2)), 48),
    "rotation": lambda sp, t: sp.cache_rotation(t("cos_sin", torch.zeros(100, 32, 2)), 64, t("pos", _ints(1, 4))),
}


@pytest.mark.parametrize("name", STRUCTS)
def test_structs_keep_their_tensors(sp, name):
    """A tensor that a call alone refers to (cache_rotation(cos_sin, D, run.positions(..)))
    lives as long as the struct that holds its address, and no longer."""
    seen = []

    def temporary(what, tensor):
        seen.append((what, weakref.ref(tensor)))
        return tensor

    struct = STRUCTS[name](sp, temporary)
    gc.collect()
    for what, ref in seen:
        assert ref() is not None, what
    del struct
    gc.collect()
    for what, ref in seen:
        assert ref() is None, what


def test_tensors_that_are_not_what_the_structs_say(sp):
    """The structs carry an address and sizes: a tensor of another type, or one whose rows
    are apart (the first columns of a wider table), would be read as something else."""
    wide = torch.arange(12, dtype=torch.int32).reshape(2, 6)
    table, length, info = wide[:, :3].contiguous(), _ints(2), _ints(3)
    angles, pos = torch.zeros(100, 32, 2), _ints(2, 4)
    runs = lambda t, n: sp.cache_runs(t, n, 48)
    rows = lambda i: sp.cache_rows(4, sp.SP_LAYOUT_PACKED, 0, i, 4)
    turn = lambda a, p, dim=64, section=(16, 16): sp.cache_rotation(a, dim, p, section)
    runs(table, length), rows(info), turn(angles, pos), turn(angles, None, section=None)
    turn(angles, _ints(4), section=None)                              # one axis: [rows] will do
    runs(wide.t()[:0].t(), length)                                    # no columns: nothing is read
    for call in (lambda: runs(wide[:, :3], length), lambda: runs(wide.t()[:3].t(), length),
                 lambda: runs(table.long(), length), lambda: runs(table, length.long()),
                 lambda: runs(table, wide[:, 0]), lambda: runs(table, _ints(1)), lambda: runs(table.reshape(-1), length),
                 lambda: rows(info.long()), lambda: rows(_ints(6)[::2]),
                 lambda: turn(angles.double(), pos), lambda: turn(angles[:, :, :1], pos),
                 lambda: turn(torch.zeros(100, 64, 2), pos), lambda: turn(torch.zeros(100, 64, 2)[:, :32], pos),
                 lambda: turn(angles, pos.long()), lambda: turn(angles, _ints(4, 2).t()),
                 lambda: turn(angles, _ints(3, 4)), lambda: turn(angles, _ints(4))):
        with pytest.raises(ValueError):
            call()
