"""Calls so large that another path takes them, and places beyond 32 bits: the bits of small calls."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
FAR = (1 << 31) + 24


def _normal(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def test_norm_of_more_than_the_cache_holds():
    import paper_2307_02031_amd as g
    x, res, dy, dres = (_normal(12288, 5120, seed=i).bfloat16() for i in range(4))
    w = _normal(5120, seed=5)
    r = g.gbmw_rms_norm_forward(x, w, residual=res, qtype=F8, group=64)
    dx, dw = g.gbmw_rms_norm_backward(dy, r.h, w, r.rstd, dres=dres)
    for part in (slice(0, 3000), slice(9300, 12288)):
        q = g.gbmw_rms_norm_forward(x[part], w, residual=res[part], qtype=F8, group=64)
        for a, b in zip(r, q):
            assert torch.equal(a[part].view(torch.uint8), b.view(torch.uint8))
        assert torch.equal(dx[part], g.gbmw_rms_norm_backward(dy[part], q.h, w, q.rstd, dres=dres[part])[0])
    want = (dy.double() * (r.h.double() * r.rstd.double()[:, None])).sum(0)
    # 12288 products of order 1, in 32 bits: a thread's rows in a row, then the workgroups' shares
    assert float((dw.double() - want).abs().max()) < 2.0 ** -24 * 12288 * 2
    # rows that are no whole lines, and in place
    wide = torch.zeros(12288, 5128, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:5123] = x
    h = wide[:, 3:5123]
    again = g.gbmw_rms_norm_forward(h, w, residual=res, h=h)
    assert torch.equal(again.y, r.y) and torch.equal(h, r.h)
    assert bool((wide[:, :3] == 0).all()) and bool((wide[:, 5123:] == 0).all())


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "pairs"])
@pytest.mark.parametrize("D,rot", [(128, 128), (256, 128)])
def test_rotary_of_more_than_the_cache_holds(D, rot, interleaved):
    import paper_2307_02031_amd as g
    B, L = 4, 4096 * 128 // D
    q, k = (_normal(B, L, H, D, seed=H).bfloat16() for H in (32, 8))
    freq = g.gbmw_rotary_frequencies(rot)
    got = g.gbmw_rotary_forward(q, k, freq, interleaved=interleaved)
    for b in range(B):
        one = g.gbmw_rotary_forward(q[b:b + 1], k[b:b + 1], freq, interleaved=interleaved)
        assert torch.equal(got[0][b:b + 1], one[0]) and torch.equal(got[1][b:b + 1], one[1])
    g.gbmw_rotary_forward(q, k, freq, interleaved=interleaved, q_out=q, k_out=k)
    assert torch.equal(q, got[0]) and torch.equal(k, got[1])


def test_rows_beyond_32_bits():
    import paper_2307_02031_amd as g
    stride = (1 << 29) - 8      # as far apart as rows of a norm may be: the last of six is beyond 2^31 elements
    near = [_normal(6, 300, seed=i).half() for i in range(4)]
    room = torch.empty(5 * stride + 300, dtype=torch.float16, device="cuda")

    def far(t):     # one array at a time lies so far apart
        v = torch.as_strided(room, (6, 300), (stride, 1))
        v.copy_(t)
        return v

    w = _normal(300, seed=9)
    base = g.gbmw_rms_norm_forward(near[0], w, residual=near[1])
    back = g.gbmw_rms_norm_backward(near[2], base.h, w, base.rstd, dres=near[3])
    for kw in (dict(x=far), dict(residual=far), dict(y=far), dict(h=far)):
        args = dict(x=near[0], residual=near[1])
        name = next(iter(kw))
        args[name] = far(args.get(name, torch.zeros_like(near[0])))
        r = g.gbmw_rms_norm_forward(weight=w, **args)
        assert torch.equal(r.y, base.y) and torch.equal(r.h, base.h), name
    for i in range(3):
        args = [near[2], base.h, near[3]]
        args[i] = far(args[i])
        dx, dw = g.gbmw_rms_norm_backward(args[0], args[1], w, base.rstd, dres=args[2])
        assert torch.equal(dx, back[0]) and torch.equal(dw, back[1])
    assert torch.equal(g.gbmw_rms_norm_backward(near[2], base.h, w, base.rstd, dres=near[3], dx=far(near[0]))[0], back[0])

    freq = g.gbmw_rotary_frequencies(100)
    x = near[0][:2].view(2, 1, 3, 100)
    turned = g.gbmw_rotary_forward(x, None, freq)[0]
    at = torch.as_strided(room, (2, 1, 3, 100), (FAR, 300, 100, 1))
    at.copy_(x)
    assert torch.equal(g.gbmw_rotary_forward(at, None, freq)[0], turned)
    assert torch.equal(g.gbmw_rotary_forward(x, None, freq, q_out=at)[0], turned)
    # heads and rows so far apart
    y = near[1][:2].view(1, 2, 3, 100)
    turned = g.gbmw_rotary_forward(y, None, freq)[0]
    at = torch.as_strided(room, (1, 2, 3, 100), (0, FAR, 100, 1))
    at.copy_(y)
    assert torch.equal(g.gbmw_rotary_forward(at, None, freq, q_out=at)[0], turned)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_tensor_beyond_32_bits(bits):
    """The last elements of a tensor of 2^31 and more get what a short tensor of theirs does, where no random numbers
    are in it."""
    import paper_2307_02031_amd as g
    n, tail = FAR, 256 * 5 + FAR % 256
    kind = F8 if bits == 8 else torch.float32
    p, grad = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.uint8 if bits == 8 else kind, device="cuda").view(kind) for _ in range(2))
    scales = [torch.zeros((n + 255) // 256, device="cuda") for _ in range(2)] if bits == 8 else None
    p[-tail:], grad[-tail:] = _normal(tail, seed=1).bfloat16(), _normal(tail, seed=2).bfloat16()
    short = [t[-tail:].clone() for t in (p, grad, m, v)]
    few = [torch.zeros((tail + 255) // 256, device="cuda") for _ in range(2)] if bits == 8 else None

    def make(p, grad, m, v, s):
        return g.gbmw_adamw_list_create([p], [grad], [m], [v], m_scales=s and s[:1], v_scales=s and s[1:], weight_decay=0.1)

    a, b = make(p, grad, m, v, scales), make(*short, few)
    for step in (1, 2):
        for lst in (a, b):
            g.gbmw_adamw_step(lst, 1e-2, step)
    torch.cuda.synchronize()
    for x, y in zip((p, m, v), (short[0], short[2], short[3])):
        assert torch.equal(x[-tail:].view(torch.uint8), y.view(torch.uint8))
    assert bool((p[:1 << 20] == 0).all())
    if bits == 8:
        assert all(torch.equal(x[-len(y):], y) for x, y in zip(scales, few))
