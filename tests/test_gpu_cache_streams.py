"""What the runner puts ahead of a launch is on the launch's stream."""
import numpy as np
import pytest
import torch

from oracle import cache as oracle_cache
from paper_2609_13804_amd import workloads as W
from paper_2609_13804_amd.runner import DeviceRun
from tests.cache_case import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", ["stream", "handle", "current", "default"])
@pytest.mark.parametrize("name", ["tiny_bf16", "small_packed_bf16"])
def test_positions_on_another_stream(gpu_lib, name, how):
    """The array that positions() makes is cleared before its launch, also while the current
    stream is far behind; rows of no image stay zero."""
    w = W.WORKLOADS[name]
    lay = W.make_layout(w)
    run = DeviceRun(w, W.make_inputs(w), lay, W.stop_bias(w))
    run.run()
    vis = np.concatenate([3 + np.arange(n) for n in np.diff(lay.img_off)])[None].astype(np.int32)
    txt = 500 + np.arange(run.sizes.T_txt)[None].astype(np.int32)
    d_vis, d_txt = ints(vis), ints(txt)
    torch.cuda.synchronize()
    ref = oracle_cache.compact_positions(vis, lay.img_off, txt, lay.text_off, run.kept_lists(), w.layout,
                                         lay.rows_per_image, np.zeros((1, run.out_rows), np.int64))
    side = torch.cuda.Stream()
    stream = {"stream": side, "handle": side.cuda_stream, "current": None, "default": 0}[how]
    a = torch.zeros(4096, 4096, device="cuda")
    b = torch.empty_like(a)
    torch.cuda.synchronize()
    with torch.cuda.stream(side if how == "default" else torch.cuda.current_stream()):
        for _ in range(20):                          # tens of milliseconds of work on the current stream
            torch.mm(a, a, out=b)
        pos = run.positions(d_vis, d_txt, stream=stream)
    torch.cuda.synchronize()
    assert np.array_equal(pos.cpu().numpy(), ref)
    assert run.device_errors() == [0, 0, 0]
