"""Layer norm where a workgroup takes several rows one after the other: rows on their way while one is worked on, sums
over rows, scratch memory that is used again, a last turn that not all have."""
import pytest
import torch

from test_gpu_layer import _check_norm, _normal

pytestmark = pytest.mark.gpu

# Rows beyond what all workgroups take at a time, forward (2048 workgroups of four rows of 64 threads or one of 256, 256
# to 512 of 1024) and backward (256 to 512 workgroups of 512 threads or more); lengths for each count of threads and
# of pieces a thread, whole pieces and not, in 32 bits (four values a piece) and 16 (eight).
SHAPES = [(8203, 40), (8195, 64), (8300, 1283), (4200, 1000), (2101, 2049), (2105, 5120), (1100, 3500), (517, 7000), (603, 8193), (301, 16385), (300, 32768)]
TYPES = pytest.mark.parametrize("dtype,wdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.float16, torch.float16)],
                                ids=["f32", "bf16-f32", "f16"])


@TYPES
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_several_rows_a_workgroup(rows, cols, dtype, wdtype):
    import paper_2307_02031_amd as g
    x = _normal(rows, cols, dtype=dtype, seed=cols, spread=2.0, middle=0.5)
    dy = _normal(rows, cols, dtype=dtype, seed=cols + 3)
    w = _normal(cols, dtype=wdtype, seed=cols + 1, spread=0.3, middle=1.0)
    b = _normal(cols, dtype=wdtype, seed=cols + 2, spread=0.3)
    y, mean, rstd, dx, dw, db = _check_norm(x, w, b, dy)
    # over their inputs, and in rows that lie apart: the same bits
    wide = torch.empty(rows, cols + 24, dtype=dtype, device="cuda")[:, 5:5 + cols]
    wide.copy_(x)
    for given in (wide, x.clone()):
        got = g.gbmw_layer_norm_forward(given, w, b, y=given)
        assert all(torch.equal(p, q) for p, q in zip((y, mean, rstd), got))
    wide.copy_(dy)
    for given in (wide, dy.clone()):
        got = g.gbmw_layer_norm_backward(given, x, w, mean, rstd, dx=given)
        assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), got))
