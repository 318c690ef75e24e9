"""RMS norm's values in 8 bits, bit for bit: the header's formula in 32 bits, each operation rounded, from the h and rstd
that the call returns."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


def _check(r, weight, qtype, group):
    y = r.h.float() * r.rstd[..., None]
    if weight is not None:
        y = y * weight.float()
    cols, top = y.shape[-1], 448 if qtype == F8 else 127
    parts = torch.nn.functional.pad(y, (0, -cols % (group or cols))).unflatten(-1, (-1, group or cols))
    scale = (parts.abs().amax(-1) * float(np.float32(1) / np.float32(top))).clamp_min(2.0 ** -126)
    c = (parts / scale[..., None]).flatten(-2)[..., :cols]
    want = c.to(F8).view(torch.uint8) if qtype == F8 else torch.round(c).clamp(-127, 127).to(torch.int8).view(torch.uint8)
    off = int((scale.view(torch.int32) != r.scale.view(torch.int32)).sum()), int((want != r.q.view(torch.uint8)).sum())
    assert off == (0, 0), off


@pytest.mark.parametrize("qtype", [F8, torch.int8], ids=["e4m3", "int8"])
@pytest.mark.parametrize("rows,cols,group,dtype", [(8192, 5120, 128, torch.bfloat16), (8192, 5120, 0, torch.bfloat16),
                                                   (20000, 1000, 32, torch.float16), (4000, 2049, 64, torch.float32),
                                                   (300, 20001, 0, torch.float32), (70000, 100, 0, torch.float16)])
def test_codes_are_the_quotient(rows, cols, group, dtype, qtype):
    import paper_2307_02031_amd as g
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x, res = (torch.randn(rows, cols, generator=gen, device="cuda").to(dtype) for _ in range(2))
    w = torch.randn(cols, generator=gen, device="cuda") * 0.2 + 1.0
    _check(g.gbmw_rms_norm_forward(x, w, residual=res, qtype=qtype, group=group, want_y=False), w, qtype, group)
    _check(g.gbmw_rms_norm_forward(x, qtype=qtype, group=group), None, qtype, group)


@pytest.mark.parametrize("qtype", [F8, torch.int8], ids=["e4m3", "int8"])
@pytest.mark.parametrize("size", [1e-38, 1e-36, 1e-30, 1e-20, 1e30])
def test_codes_of_far_sizes(size, qtype):
    """Scales from the least on, and within a group values of many sizes."""
    import paper_2307_02031_amd as g
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(500, 1280, generator=gen, device="cuda")
    w = torch.randn(1280, generator=gen, device="cuda") * size
    w *= 2.0 ** torch.randint(-30, 1, (1280,), generator=gen, device="cuda").float()
    for group in (0, 64):
        _check(g.gbmw_rms_norm_forward(x, w, qtype=qtype, group=group), w, qtype, group)
