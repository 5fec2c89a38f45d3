"""DeviceRun.positions on its arguments (CPU: the run is a shell around sizes, and the
launch is caught before it).
"""
from types import SimpleNamespace

import pytest
import torch

T_VIS, T_TXT, ROWS = 10, 5, 9


@pytest.fixture
def run(monkeypatch):
    from paper_2609_13804_amd import binding, runner
    r = runner.DeviceRun.__new__(runner.DeviceRun)
    r.sizes = SimpleNamespace(T_vis=T_VIS, T_txt=T_TXT, B=2)
    r.X = torch.zeros(1)
    r.out_rows, r.layout_code, r.rows_per_image = ROWS, binding.SP_LAYOUT_PACKED, 0
    r.img_off = r.text_off = r.kept_idx = r.kept_off = r.kept_cnt = None
    r.ws, r.ws_bytes = [None] * 3, [0] * 3
    r.calls = []
    monkeypatch.setattr(binding, "stepprune_compact_positions", lambda *a, **k: r.calls.append(a))
    return r


def _ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_shapes_are_the_runs(run):
    """The kernel takes sizes from the run and axes from vis_pos: fewer axes or tokens in
    the other arrays would be read and written out of range."""
    for axes in (1, 3):
        pos = run.positions(_ints(axes, T_VIS), _ints(axes, T_TXT))
        assert tuple(pos.shape) == (axes, ROWS) and pos.dtype == torch.int32 and not pos.any()
        mine = _ints(axes, ROWS)
        assert run.positions(_ints(axes, T_VIS), _ints(axes, T_TXT), pos=mine) is mine
    assert len(run.calls) == 4
    vis, txt, pos = _ints(3, T_VIS), _ints(3, T_TXT), _ints(3, ROWS)
    for bad in ((vis, txt[:1], None), (vis[:, :-1].contiguous(), txt, None), (vis, txt[:, :-1].contiguous(), None),
                (vis.long(), txt, None), (vis, txt.long(), None), (vis, txt, pos[:2]), (vis, txt, pos[:, 1:].contiguous()),
                (vis, txt, pos.long()), (_ints(T_VIS, 3).t(), txt, None), (vis, _ints(T_TXT, 3).t(), None),
                (vis, txt, _ints(ROWS, 3).t()), (vis[0], txt[0], None), (_ints(3, T_VIS + 1), txt, None)):
        with pytest.raises(ValueError):
            run.positions(*bad)
    assert len(run.calls) == 4
