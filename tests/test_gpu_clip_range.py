"""Clipping where the norm or the factor leaves 32 bits' normal numbers."""
import math

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,value,max_norm,scale", [
    (1000, 3e38, 1.0, 1.0),            # norm 9.5e39: not a number of 32 bits; factor 1e-40
    (70001, 3.4e38, 1e-3, 0.5),
    (5, 1e38, 1e-20, 1.0),             # factor 6e-59
    (40000, 3e38, 1e-30, 1.0),         # outputs of 6e-33 from a factor of 2e-71
    (100, 1e30, 1e-9, 1.0),            # factor 1e-40, a norm that 32 bits hold
    (100, 1e30, 1e30, 0.25),           # an ordinary factor
    (100, 1e38, math.inf, 1e-40),      # a scale below the normal numbers is taken as it is
    (100, 1.0, math.inf, 1e-40)])
def test_factors_of_any_size(n, value, max_norm, scale):
    """Bound: the factor and the product are each rounded to 24 bits, and a result below the normal numbers to its step."""
    import paper_2307_02031_amd as g
    print("clip", n, value, max_norm, scale, flush=True)
    gen = torch.Generator().manual_seed(n)
    x = (value * (1.0 - torch.rand(n, generator=gen, dtype=torch.float64) * 0.5)).float()
    x[::3] *= -1
    x64, s64, m64 = x.double(), float(torch.tensor(scale)), float(torch.tensor(max_norm))
    want = s64 * math.sqrt(math.fsum((x64 * x64).tolist()))
    factor = s64 * (m64 / want) if want > m64 else s64
    for in_place in (False, True):
        grad = x.cuda()
        out = grad if in_place else torch.zeros_like(grad)
        lst = g.gbmw_gradient_list_create([grad], [out])
        norm = float(g.gbmw_clip_gradients(lst, max_norm, scale))
        assert norm == math.inf if want > 3.5e38 else abs(norm - want) <= 2.0 ** -22 * want + 2.0 ** -149
        y = x64 * factor
        ref.assert_close("out", out, y, 3 * 2.0 ** -24 * y.abs() + 2.0 ** -150)
        g.gbmw_gradient_list_destroy(lst)
