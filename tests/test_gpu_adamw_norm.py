"""The norm and the step that clips by it, called one after the other as documented: with one scale of the loss in both, and
the gradients left as they are."""
import math

import pytest
import torch

import layer_reference as ref
from test_gpu_adamw import HOW, SIZES, _check, _copy, _list, _tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale,max_norm", [(1.0, 0.5), (0.25, 0.5), (0.25, 1e6), (3.0, 1.0), (2.0 ** -10, 1e-4)])
def test_norm_and_step_with_a_loss_scale(scale, max_norm, bits, gdtype):
    import paper_2307_02031_amd as g
    decay = [0.01] * len(SIZES)
    t = _tensors(bits, torch.float32, gdtype, 4100)
    before = _copy(t)
    norm = g.gbmw_clip_gradients(g.gbmw_gradient_list_create(t["grad"], norm_only=True), max_norm, scale)
    g.gbmw_adamw_step(_list(g, t, decay), step=3, scale=scale, norm=norm, max_norm=max_norm, **HOW)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(t["grad"], before["grad"]))
    total = float(torch.cat([ref.f64(x) for x in before["grad"]]).norm()) * scale
    assert abs(float(norm) - total) <= 2.0 ** -23 * total     # a sum in 64 bits, rounded once
    _check(before, t, 3, decay, scale * (max_norm / total if total > max_norm else 1.0))


def test_a_list_for_the_norm_alone():
    """The same norm as with outputs, of nothing, of NaN, and in a graph; no tensor is written."""
    import paper_2307_02031_amd as g
    xs = [torch.randn(n, generator=torch.Generator().manual_seed(n)).cuda().half() for n in (1, 40000, 0, 777)]
    before = [x.clone() for x in xs]
    only = g.gbmw_gradient_list_create(xs, norm_only=True)
    outs = [torch.zeros(x.shape, device="cuda") for x in xs]
    for max_norm, scale in ((1e-3, 1.0), (math.inf, 0.5)):
        want = g.gbmw_clip_gradients(g.gbmw_gradient_list_create(xs, outs), max_norm, scale)
        assert torch.equal(g.gbmw_clip_gradients(only, max_norm, scale), want)
        assert all(torch.equal(x, y) for x, y in zip(xs, before))
    norm = torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.gbmw_clip_gradients(only, math.inf, 0.5, norm=norm)
    for k in range(3):
        xs[1].mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, g.gbmw_clip_gradients(only, math.inf, 0.5))
    xs[3][5] = float("nan")
    assert math.isnan(float(g.gbmw_clip_gradients(only, 1.0)))
    assert float(g.gbmw_clip_gradients(g.gbmw_gradient_list_create([], norm_only=True), 1.0)) == 0.0
    with pytest.raises(g.GbmwError):
        g.gbmw_gradient_list_create(xs, outs, norm_only=True)
