"""RMS norm backward on both sides of what decides how many threads a row has: its length, whether it is whole pieces, and the
number of rows."""
import pytest
import torch

from test_gpu_rms import _check_backward, _normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("cols", [4096, 4097, 4104, 5113, 5120, 5121])
@pytest.mark.parametrize("rows", [512, 513, 2047, 2048])
def test_threads_of_a_row(rows, cols, dtype):
    import paper_2307_02031_amd as g
    x, dy, dres = (_normal(rows, cols, dtype=dtype, seed=cols + i) for i in range(3))
    w = _normal(cols, dtype=torch.float32, seed=4, spread=0.3, middle=1.0)
    rstd = torch.rand(rows, generator=torch.Generator().manual_seed(rows)).cuda() + 0.5
    need = g.gbmw_rms_norm_workspace(x, w)
    whole = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    dx, dw = g.gbmw_rms_norm_backward(dy, x, w, rstd, dres=dres, workspace=whole[:need])
    _check_backward(dx, dw, dy, x, w, rstd, dres)
    assert bool((whole[need:] == 0x5a).all())
