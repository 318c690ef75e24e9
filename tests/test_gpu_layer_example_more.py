"""A present-day decoder layer's whole step with the operators together (RMS norm that adds, rotary positions, attention,
the gradients' norm, AdamW that clips), against torch's own differentiation and the formula in 64 bits."""
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


def _plain(w, x, head, n):
    """The same layer in 64 bits, sample by sample; rows beyond a sample's length see and are seen by nothing."""
    h = x.shape[-1]
    norm = lambda t, a: t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-5) * a
    half = head // 2
    freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64) * 2 / head)
    rows = []
    for b in range(x.shape[0]):
        t = norm(x[b], w["norm1"]) @ w["qkv"].T + w["qkv_bias"]
        q, k, v = t.view(-1, 3, h // head, head).permute(1, 2, 0, 3)
        angle = torch.arange(x.shape[1], dtype=torch.float64)[:, None] * freq
        turn = lambda a: torch.cat([a[..., :half] * angle.cos() - a[..., half:] * angle.sin(),
                                    a[..., :half] * angle.sin() + a[..., half:] * angle.cos()], -1)
        s = (turn(q) @ turn(k).transpose(1, 2)) * head ** -0.5
        i = torch.arange(x.shape[1])
        m = (i[None, :] < n[b]) & (i[:, None] < n[b]) & (i[None, :] <= i[:, None])
        p = torch.softmax(torch.where(m, s, -torch.inf), 2)
        o = torch.where(m.any(1)[:, None], torch.nan_to_num(p) @ v, 0.0).permute(1, 0, 2).reshape(-1, h)
        rows.append(x[b] + o @ w["proj"].T + w["proj_bias"])
    y = torch.stack(rows)
    a = torch.nn.functional.gelu(norm(y, w["norm2"]) @ w["up"].T + w["up_bias"])
    return y + a @ w["down"].T + w["down_bias"]


@pytest.mark.parametrize("bits", [32, 8])
def test_a_layers_step_with_its_optimizer(bits):
    import paper_2307_02031_amd as g
    from paper_2307_02031_amd.layer_example import Layer
    B, L, hidden, head = 3, 70, 128, 32
    layer = Layer(g, hidden, head, True, dtype=torch.float16, rms=True, rotary=True)
    layer.optimizer(bits)
    gen = torch.Generator().manual_seed(3)
    x, dz = (torch.randn(B, L, hidden, generator=gen).half().cuda() for _ in range(2))
    n = torch.tensor([70, 1, 33], dtype=torch.int32, device="cuda")
    z = layer.forward(x, n)
    dx = layer.backward(dz)
    before = {k: t.clone() for k, t in layer.param.items()}
    norm = layer.step(1e-3, 0.5)
    torch.cuda.synchronize()

    w = {k: (t.half() if k in layer.grad and layer.grad[k].dtype == torch.float16 else t).cpu().double().requires_grad_()
         for k, t in before.items()}
    x64 = x.cpu().double().requires_grad_()
    want = _plain(w, x64, head, n.tolist())
    grads = torch.autograd.grad(want, [x64, *w.values()], dz.cpu().double())
    # values pass about a dozen roundings to 11 bits on their way, at random: 12 ** 0.5 * 2 ** -12 is under 2 ** -10
    off = lambda a, b: float((a.cpu().double() - b).norm() / b.norm())
    assert off(z, want.detach()) < 2.0 ** -9
    assert off(dx, grads[0]) < 2.0 ** -8
    assert list(layer.grad) == list(w)
    for (name, got), ref in zip(layer.grad.items(), grads[1:]):
        assert off(got, ref) < 2.0 ** -8, name
    total = float(torch.cat([t.double().flatten() for t in layer.grad.values()]).norm())
    assert abs(float(norm) - total) <= 1e-6 * total
    # the first step of AdamW: m / c1 is the clipped gradient, and v / c2 its square, whatever the states' bits
    for name, t in layer.param.items():
        clipped = layer.grad[name].double() * min(1.0, 0.5 / total)
        keep = 1.0 - 1e-3 * (0.1 if t.dim() == 2 else 0.0)
        ref = before[name].double() * keep - 1e-3 * clipped / (clipped.abs() + 1e-8)
        # a step of 1e-3, off by 2^-20 of itself, and the roundings of parameters of order 1
        assert float((t.double() - ref).abs().max()) < 1e-3 * 2.0 ** -20 + 2.0 ** -22 * float(before[name].abs().max() + 1)
        if layer.w[name] is not t:
            assert torch.equal(layer.w[name], t.half())
    layer.backward(dz)     # and once more, with the states and weights that the step left
    assert float(layer.step(1e-3, 0.5)) > 0 and all(bool(torch.isfinite(t).all()) for t in layer.param.values())


@pytest.mark.parametrize("more", [[], ["--norm", "rms", "--rotary", "--states", "8"], ["--states", "32"]],
                         ids=["plain", "rms-rotary-8", "32"])
def test_the_command(more, monkeypatch, capsys):
    from paper_2307_02031_amd import layer_example
    monkeypatch.setattr(sys, "argv", ["layer_example", "--model", "BERT-Huge-32", "--batch", "1", "--steps", "1", *more])
    layer_example.main()
    said = capsys.readouterr().out
    assert "forward" in said and "best: batch" in said and ("step" in said.splitlines()[0]) == ("--states" in more)
