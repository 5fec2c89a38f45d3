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
