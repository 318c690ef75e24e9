"""What a NaN, an infinity, or squares that 32 bits do not hold leave of a row, its scales and its codes."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


@pytest.mark.parametrize("qtype", [F8, torch.int8], ids=["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("cols", [300, 1283, 5120])
@pytest.mark.parametrize("group", [0, 64, 128])
def test_rows_that_are_not_finite(group, cols, dtype, qtype):
    import paper_2307_02031_amd as g
    x = torch.randn(4, cols, generator=torch.Generator().manual_seed(cols)).to(dtype).cuda()
    x[0, 17], x[1, 200], x[2, 70] = float("-inf"), float("nan"), 3e19
    r = g.gbmw_rms_norm_forward(x, qtype=qtype, group=group)
    groups = -(-cols // group) if group else 1
    assert r.scale.shape == (4, groups)
    own = torch.arange(groups, device="cuda") == 17 // (group or cols)
    # an infinity: itself NaN, and its group's scale; the others 0, with the least scale
    assert float(r.rstd[0]) == 0.0 and bool(torch.isnan(r.y[0, 17])) and bool(torch.isnan(r.scale[0][own]).all())
    rest = torch.arange(cols, device="cuda") != 17
    assert bool((r.y[0][rest] == 0).all()) and bool((r.scale[0][~own] == 2.0 ** -126).all())
    each = torch.arange(cols, device="cuda") // (group or cols)
    assert bool((r.q[0][~own[each]].float() == 0).all())
    # a NaN: the row
    assert bool(torch.isnan(r.rstd[1])) and bool(torch.isnan(r.y[1]).all()) and bool(torch.isnan(r.scale[1]).all())
    # squares beyond 32 bits: zeros
    assert float(r.rstd[2]) == 0.0 and bool((r.y[2] == 0).all())
    assert bool((r.scale[2] == 2.0 ** -126).all()) and bool((r.q[2].float() == 0).all())
    # the row beside them is as it is alone
    one = g.gbmw_rms_norm_forward(x[3:], qtype=qtype, group=group)
    assert torch.equal(r.y[3:], one.y) and torch.equal(r.q[3:].view(torch.uint8), one.q.view(torch.uint8)) and torch.equal(r.scale[3:], one.scale)
