"""As many workgroups as a launch of the attention kernels may have."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_eight_million_heads(dtype):
    """2^23 heads of one row and 128 keys, the same head over and over (strides of 0): each has that head's results."""
    import paper_2307_02031_amd as g
    gen = torch.Generator().manual_seed(3)
    new = lambda *s: torch.randn(*s, generator=gen).to(dtype).cuda()
    q, k, v, dout = new(1, 1, 1, 1), new(1, 128, 1, 1), new(1, 128, 1, 1), new(1, 1, 1, 1)
    out, lse = g.gbmw_attention_forward(q, k, v)
    base = g.gbmw_attention_backward(dout, q, k, v, out, lse)
    B, H = 1 << 13, 1 << 10
    many = lambda t: t.expand(B, t.shape[1], H, 1)
    print("attention backward", B, H, dtype, flush=True)
    got = g.gbmw_attention_backward(many(dout), many(q), many(k), many(v), many(out), lse.expand(B, H, 1).contiguous())
    for a, b in zip(got, base):
        assert bool((a == b).all())
