"""Scales at the ends of what is accepted."""
import pytest
import torch

from test_gpu_attention import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Lq,Lk", [(70, 90), (3, 200), (5, 6)])
@pytest.mark.parametrize("scale,size", [(1e-31, 3e14), (1e-36, 1e17), (4e-38, 5e17)])
def test_scales_of_large_queries_and_keys(scale, size, Lq, Lk):
    """Scores of a few hundredths from products that only bfloat16's range holds.  The bounds are relative to the terms, as
    everywhere; gradients of q and k are as small as the keys and queries are large."""
    q, k, v, dout = _inputs(1, Lq, Lk, 2, 2, 16, torch.bfloat16, seed=Lq)
    q, k = ((t.float() * size).bfloat16() for t in (q, k))
    _check(q, k, v, dout, scale=scale)
    _check(q, k, v, dout, scale=scale, causal=True)


@pytest.mark.parametrize("Lq,Lk", [(70, 90), (3, 200), (5, 6)])
def test_the_largest_scale_of_scores_of_zero(Lq, Lk):
    """All keys count alike."""
    import paper_2307_02031_amd as g
    q, k, v, dout = _inputs(1, Lq, Lk, 2, 2, 16, torch.bfloat16, seed=Lq)
    q[:] = 0
    out, lse = g.gbmw_attention_forward(q, k, v, scale=3.4e38)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    base = g.gbmw_attention_forward(q, k, v, scale=1.0)
    assert torch.equal(out, base[0]) and torch.equal(lse, base[1])
