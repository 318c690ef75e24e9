"""A norm written over its input: the call returns no h, which a backward call would take for the rows that were normed."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_no_h_is_left(dtype):
    import paper_2307_02031_amd as g
    x, dy = (torch.randn(7, 300, generator=torch.Generator().manual_seed(i)).to(dtype).cuda() for i in range(2))
    w = torch.ones(300, device="cuda")
    base = g.gbmw_rms_norm_forward(x, w)
    assert base.h is x
    for y in (lambda t: t, lambda t: t.view(7, 300), lambda t: t[:]):       # the tensor itself, or another one of its memory
        over = x.clone()
        r = g.gbmw_rms_norm_forward(over, w, y=y(over))
        assert r.h is None and torch.equal(over, base.y) and torch.equal(r.rstd, base.rstd)
        with pytest.raises(g.GbmwError):
            g.gbmw_rms_norm_backward(dy, r.h, w, r.rstd)
    # with a residual the sum is there, in place or not
    a, res = x.clone(), dy.clone()
    r = g.gbmw_rms_norm_forward(a, w, residual=res, y=a)
    assert torch.equal(r.h, x + dy)
    assert g.gbmw_rms_norm_forward(x[:0], w, y=x[:0]).h is not None
