"""More rows than a launch has workgroups for: each takes a second turn, and what it kept of the first is in nobody's way."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
TURN = 1 << 21      # workgroups at most


# 256 and 128 threads a row (one, and two rows a workgroup), 64 (four) and 16 (sixteen); the most codes are 8.7 GB
@pytest.mark.parametrize("cols,per", [(1540, 1), (2064, 2), (400, 4), (24, 16)])
def test_a_second_turn(cols, per):
    import paper_2307_02031_amd as g
    rows = TURN * per + 70
    # rows that overlap, each one value further on: all differ, in little memory
    x = torch.randn(rows + cols, generator=torch.Generator(device="cuda").manual_seed(cols), device="cuda").bfloat16()
    x = x * torch.exp2((torch.arange(rows + cols, device="cuda") % 1000 / 100).float()).bfloat16()
    x = torch.as_strided(x, (rows, cols), (1, 1))
    w = torch.randn(cols, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    for group in (0, 32):
        r = g.gbmw_rms_norm_forward(x, w, qtype=F8, group=group, want_y=False)
        for part in (slice(0, 40), slice(TURN * per - 30, rows)):
            q = g.gbmw_rms_norm_forward(x[part], w, qtype=F8, group=group, want_y=False)
            assert torch.equal(q.rstd, r.rstd[part]) and torch.equal(q.scale, r.scale[part])
            assert torch.equal(q.q.view(torch.uint8), r.q[part].view(torch.uint8))
    del r, q
    torch.cuda.empty_cache()
