"""AdamW over many tensors against a plain form in 64 bits.

Bounds, worked out before any run: each product and each sum is rounded by 2^-24 relative, and so are the factors that all
elements share, so the moments are off by 2^-22 of their terms' sizes, a step by the first moment's error and 2^-20 of
itself, the parameter by those, a rounding of each of its two terms, and half a step of its type."""
import math

import numpy as np
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
SIZES = [1, 0, 7, 255, 256, 257, 5000, 16384, 16385, 70001, 3]
HOW = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8)


def _normal(n, seed, spread=1.0):
    return torch.randn(n, generator=torch.Generator().manual_seed(seed)) * spread


def _coded(x):
    """Codes and scales of blocks of 256, to the nearest."""
    blocks = torch.nn.functional.pad(x, (0, -len(x) % 256)).view(-1, 256)
    scale = (blocks.abs().amax(1) / 448).clamp_min(2.0 ** -126)
    return (blocks / scale[:, None]).view(-1)[:len(x)].to(F8), scale


def _held(code, scale):
    return code.cpu().double() * scale.cpu().double().repeat_interleave(256)[:len(code)]


def _tensors(bits, dtype, gdtype, seed, sizes=SIZES, copy=None, zero=False):
    """Tensors as dicts, all of one kind end to end in one buffer, at odd places."""
    def flat(parts, dtype):
        whole = torch.zeros(sum(len(p) for p in parts) + 3, device="cuda").to(dtype)
        for p, view in zip(parts, whole[3:].split([len(p) for p in parts])):
            view.copy_(p)
        return list(whole[3:].split([len(p) for p in parts]))

    z = 0.0 if zero else 1.0
    m = [_normal(n, seed + 100 + i, 0.01 * z) for i, n in enumerate(sizes)]
    v = [(_normal(n, seed + 200 + i, 0.01).abs() + 0.003) ** 2 * z for i, n in enumerate(sizes)]
    t = dict(param=flat([_normal(n, seed + i, 0.05) for i, n in enumerate(sizes)], dtype),
             grad=flat([_normal(n, seed + 300 + i, 10.0 ** -(1 + i % 3)) for i, n in enumerate(sizes)], gdtype))
    if bits == 32:
        t.update(m=flat(m, torch.float32), v=flat(v, torch.float32))
    else:
        cm, cv = [_coded(x) for x in m], [_coded(x.sqrt()) for x in v]
        t.update(m=flat([c for c, _ in cm], F8), v=flat([c for c, _ in cv], F8),
                 m_scale=flat([s for _, s in cm], torch.float32), v_scale=flat([s for _, s in cv], torch.float32))
    if copy is not None:
        t["copy"] = flat([torch.zeros(n) for n in sizes], copy)
    return t


def _list(g, t, decay):
    return g.gbmw_adamw_list_create(t["param"], t["grad"], t["m"], t["v"], m_scales=t.get("m_scale"), v_scales=t.get("v_scale"),
                                    copies=t.get("copy"), weight_decay=decay)


def _copy(t):
    return {n: [x.clone() for x in xs] for n, xs in t.items()}


def _want(t, i, step, decay, factor=1.0, lr=HOW["lr"]):
    """param, m, v of tensor i after a step from t, each with its bound, in 64 bits."""
    b1, b2, eps = HOW["beta1"], HOW["beta2"], HOW["eps"]
    p, grad = ref.f64(t["param"][i]), ref.f64(t["grad"][i]) * factor
    if "m_scale" in t:
        m, v = _held(t["m"][i], t["m_scale"][i]), _held(t["v"][i], t["v_scale"][i]) ** 2
    else:
        m, v = ref.f64(t["m"][i]), ref.f64(t["v"][i])
    em = 2.0 ** -22 * (b1 * m.abs() + (1 - b1) * grad.abs()) + 1e-45
    m, v = b1 * m + (1 - b1) * grad, b2 * v + (1 - b2) * grad ** 2
    ev = 2.0 ** -21 * v + 1e-44
    den = torch.sqrt(v / (1 - b2 ** step)) + eps
    by = lr / (1 - b1 ** step)
    change = by * m / den
    want = p * (1 - lr * decay) - change
    ep = (by / den * em + 2.0 ** -20 * change.abs() + 2.0 ** -22 * (p.abs() + change.abs()) +
          ref.U[t["param"][i].dtype] * want.abs() + ref.TINY[t["param"][i].dtype])
    return (want, ep), (m, em), (v, ev)


def _check(before, t, step, decay, factor=1.0, lr=HOW["lr"], seed=0):
    for i, n in enumerate(len(x) for x in before["param"]):
        if not n:
            continue
        p, m, v = _want(before, i, step, decay[i], factor, lr)
        ref.assert_close(f"param {i}", t["param"][i], *p)
        if "copy" in t:
            assert torch.equal(t["copy"][i], t["param"][i].to(t["copy"][i].dtype))
        if "m_scale" not in t:
            ref.assert_close(f"m {i}", t["m"][i], *m)
            ref.assert_close(f"v {i}", t["v"][i], *v)
            continue
        r = torch.sqrt(v[0])
        for name, x, off in (("m", m[0], m[1]), ("v", r, 2.0 ** -21 * r)):
            pad = torch.nn.functional.pad(x.abs(), (0, -n % 256)).view(-1, 256)
            scale = (pad.amax(1) / 448).clamp_min(2.0 ** -126)
            worst = torch.nn.functional.pad(off, (0, -n % 256)).view(-1, 256).amax(1)
            ref.assert_close(f"{name} scale {i}", t[name + "_scale"][i], scale, 2.0 ** -22 * scale + worst / 448)
            each = t[name + "_scale"][i].cpu().double().repeat_interleave(256)[:n]
            c, code = x / each, t[name][i].cpu().double()
            step_of = 2.0 ** (torch.floor(torch.log2(c.abs().clamp_min(2.0 ** -6))) - 3)
            # the nearest is half a step away, a neighbour at random less than a whole one; a root that is not 0 is not held as 0
            most = step_of * (0.5 if seed == 0 else 1.0) * 1.0001 + off / each
            if name == "v":
                assert bool(((code > 0) | (x == 0)).all())
                most = torch.where(c < 2.0 ** -9, 2.0 ** -9, most)
            ref.assert_close(f"{name} codes {i}", code, c, most)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,gdtype,copy", [(torch.float32, torch.float32, None), (torch.float32, torch.bfloat16, torch.bfloat16),
                                               (torch.float32, torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16, None),
                                               (torch.float16, torch.float32, None), (torch.bfloat16, torch.float16, None)])
def test_steps(bits, dtype, gdtype, copy):
    import paper_2307_02031_amd as g
    t = _tensors(bits, dtype, gdtype, 1000, copy=copy)
    decay = [0.1 * (i % 2) for i in range(len(SIZES))]
    lst = _list(g, t, decay)
    for step, seed in ((1, 0), (2, 5), (3, 0), (70000, 123456789)):
        print("adamw", bits, dtype, gdtype, step, flush=True)
        before = _copy(t)
        g.gbmw_adamw_step(lst, step=step, seed=seed, **HOW)
        torch.cuda.synchronize()
        _check(before, t, step, decay, seed=seed)
    g.gbmw_adamw_list_destroy(lst)


@pytest.mark.parametrize("bits", [32, 8])
def test_from_zeroed_states(bits):
    """The first step moves every parameter by about lr, whatever the gradient's size; zero gradients move nothing."""
    import paper_2307_02031_amd as g
    t = _tensors(bits, torch.float32, torch.float32, 2000, zero=True)
    t["grad"][3].zero_()
    if bits == 8:
        for n in ("m", "v", "m_scale", "v_scale"):
            for x in t[n]:
                x.view(torch.uint8).zero_()
    before = _copy(t)
    g.gbmw_adamw_step(_list(g, t, 0.0), step=1, **HOW)
    torch.cuda.synchronize()
    _check(before, t, 1, [0.0] * len(SIZES))
    assert torch.equal(t["param"][3], before["param"][3])
    moved = (t["param"][5] - before["param"][5]).abs()
    assert bool((moved > 0.9 * HOW["lr"]).all()) and bool((moved < 1.1 * HOW["lr"]).all())


def test_rounding_at_random_is_right_on_average_and_as_documented():
    """Codes from the hash of seed, step and place, worked out here again; their errors add up to no more than chance
    allows: n numbers of variance at most a quarter of a step's square."""
    import paper_2307_02031_amd as g
    sizes = [300, 70000, 1000]
    t = _tensors(8, torch.float32, torch.float32, 3000, sizes=sizes)
    before = _copy(t)
    seed, step = 77, 9
    g.gbmw_adamw_step(_list(g, t, 0.0), step=step, seed=seed, **HOW)
    torch.cuda.synchronize()

    def bits(x):
        x = (x * 0x9E3779B1) & 0xFFFFFFFF
        x = ((x ^ (x >> 15)) * 0x85EBCA77) & 0xFFFFFFFF
        return x ^ (x >> 13)

    key, block = bits((seed + step * 0x9E3779B9) & 0xFFFFFFFF), 0
    for i, n in enumerate(sizes):
        word = bits(torch.arange(block * 256, block * 256 + n) ^ key)
        block += (n + 255) // 256
        _, m, v = _want(before, i, step, 0.0)
        for name, x, part in (("m", m[0], word >> 16), ("v", torch.sqrt(v[0]), word & 65535)):
            each = t[name + "_scale"][i].cpu().double().repeat_interleave(256)[:n]
            c = x / each
            unit = 2.0 ** (torch.floor(torch.log2(c.abs().clamp_min(2.0 ** -6))) - 3)
            up = c.abs() / unit + (part + 0.5) / 65536
            sure = (up - torch.round(up)).abs() > 1e-3      # 32 bits decide the others
            got = t[name][i].cpu().double()
            want = torch.copysign(torch.floor(up) * unit, c)
            assert bool(sure.double().mean() > 0.99) and torch.equal(got[sure], want[sure])
            off = ((got - c) / unit)[c.abs() > 2.0 ** -6]
            assert abs(float(off.mean())) < 6 * 0.5 / math.sqrt(len(off))
    # another seed, other codes; the same again, the same
    a, b, c = (_copy(before) for _ in range(3))
    for x, s in ((a, seed), (b, seed), (c, seed + 1)):
        g.gbmw_adamw_step(_list(g, x, 0.0), step=step, seed=s, **HOW)
    raw = lambda x: x["m"][1].view(torch.uint8)
    assert torch.equal(raw(a), raw(t)) and torch.equal(raw(a), raw(b)) and not torch.equal(raw(a), raw(c))
    assert torch.equal(a["param"][1], c["param"][1])


@pytest.mark.parametrize("bits", [32, 8])
def test_clips_as_it_reads(bits):
    """With the norm that the clipping call leaves: the step of clipped gradients; without a finite norm, none."""
    import paper_2307_02031_amd as g
    decay = [0.01] * len(SIZES)
    for scale, max_norm in ((1.0, 0.5), (0.25, 1e6), (2.0, 0.1)):
        t = _tensors(bits, torch.float32, torch.bfloat16, 4000)
        before = _copy(t)
        norm = g.gbmw_clip_gradients(g.gbmw_gradient_list_create(t["grad"]), float("inf"), 1.0)
        lst = _list(g, t, decay)
        norm *= scale
        g.gbmw_adamw_step(lst, step=3, scale=scale, norm=norm, max_norm=max_norm, **HOW)
        torch.cuda.synchronize()
        total = float(torch.cat([ref.f64(x) for x in before["grad"]]).norm()) * scale
        factor = scale * (max_norm / total if total > max_norm else 1.0)
        assert all(torch.equal(a, b) for a, b in zip(t["grad"], before["grad"]))
        _check(before, t, 3, decay, factor)
        for bad in (float("nan"), float("inf")):
            held = _copy(t)
            g.gbmw_adamw_step(lst, step=4, norm=torch.full((1,), bad, device="cuda"), max_norm=1.0, **HOW)
            torch.cuda.synchronize()
            for n, xs in t.items():
                assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(xs, held[n])), n


def test_numbers_read_on_the_device_and_a_graph():
    """A captured step takes the rate, the step's number and the norm of the moment."""
    import paper_2307_02031_amd as g
    for bits in (32, 8):
        t = _tensors(bits, torch.float32, torch.bfloat16, 5000, copy=torch.bfloat16)
        other = _copy(t)
        lr, step = torch.tensor([1e-3], device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
        norm = torch.ones(1, device="cuda")
        how = dict(beta1=0.9, beta2=0.99, seed=11, max_norm=1.0)
        lst, plain = _list(g, t, 0.1), _list(g, other, 0.1)
        state = _copy(t)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step += 1
            g.gbmw_adamw_step(lst, lr, step, norm=norm, **how)
        assert all(torch.equal(a, b) for a, b in zip(t["param"], state["param"]))     # captured, not run
        for i in range(1, 5):
            lr.fill_(1e-3 / i)
            norm.fill_(0.5 * i)
            graph.replay()
            torch.cuda.synchronize()
            assert int(step) == i
            g.gbmw_adamw_step(plain, float(lr), i, norm=norm, **how)
            torch.cuda.synchronize()
            for n, xs in t.items():
                assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(xs, other[n])), (bits, i, n)


def test_streams_nothing_and_neighbours():
    import paper_2307_02031_amd as g
    g.gbmw_adamw_step(g.gbmw_adamw_list_create([], [], [], []), step=1, **HOW)
    for bits in (32, 8):
        t = _tensors(bits, torch.float32, torch.float32, 6000)
        other = _copy(t)
        g.gbmw_adamw_step(_list(g, t, 0.0), step=2, **HOW)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        lst = _list(g, other, 0.0)
        g.gbmw_adamw_step(lst, step=2, stream=side, **HOW)
        side.synchronize()
        for n, xs in t.items():
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(xs, other[n])), n
        # only every other tensor is in a list: the ones between stay
        t = _tensors(bits, torch.float32, torch.float32, 7000, copy=torch.float16)
        before = _copy(t)
        some = {n: xs[::2] for n, xs in t.items()}
        g.gbmw_adamw_step(_list(g, some, 0.0), step=2, **HOW)
        torch.cuda.synchronize()
        for n in t:
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(t[n][1::2], before[n][1::2])), n


def test_nan_and_infinities_stay_in_their_block():
    import paper_2307_02031_amd as g
    for bits in (32, 8):
        for bad in (float("nan"), float("inf")):
            t = _tensors(bits, torch.float32, torch.float32, 8000, sizes=[1000])
            t["grad"][0][300] = bad
            before = _copy(t)
            for step in (1, 2):
                g.gbmw_adamw_step(_list(g, t, 0.0), step=step, seed=step - 1, **HOW)
            torch.cuda.synchronize()
            fine = torch.ones(1000, dtype=torch.bool)
            fine[256:512 if bits == 8 else 301] = False
            if bits == 32:
                fine[256:300] = True
            else:
                assert bool(torch.isnan(_held(t["m"][0], t["m_scale"][0])[256:512]).all()) or bad == float("inf")
                assert not bool(torch.isfinite(t["m_scale"][0][1]))
            assert bool(torch.isfinite(t["param"][0][fine.cuda()]).all()) and not bool(torch.isfinite(t["param"][0][300]))


def test_refusals():
    import paper_2307_02031_amd as g
    p, q, m, v = (torch.zeros(600, device="cuda") for _ in range(4))
    make = g.gbmw_adamw_list_create
    s = lambda: [torch.zeros(3, device="cuda")]
    e = lambda: [torch.zeros(600, device="cuda", dtype=F8)]
    whole = torch.zeros(1200, device="cuda")
    half = torch.zeros(600, device="cuda", dtype=torch.float16)
    for args, kw in [(([p], [q], [m], [m]), {}), (([p], [p], [m], [v]), {}), (([p, p], [q, q], [m, v], [v, m]), {}),
                     (([p], [q[:5]], [m], [v]), {}), (([p], [q], [m], []), {}), (([p], [q], [m], [v]), dict(m_scales=s(), v_scales=s())),
                     (([p], [q], e(), e()), {}), (([p], [q], e(), e()), dict(m_scales=s(), v_scales=[torch.zeros(2, device="cuda")])),
                     (([p], [q], e(), [v]), dict(m_scales=s(), v_scales=s())), (([p], [q], [m], [v]), dict(copies=[torch.zeros(600, device="cuda")])),
                     (([half], [q], [m], [v]), dict(copies=[torch.zeros_like(half)])), (([p.cpu()], [q], [m], [v]), {}),
                     (([p], [q], [m], [v]), dict(weight_decay=-1.0)), (([p], [q], [m], [v]), dict(weight_decay=[0.0, 0.0])),
                     (([whole[:600]], [q], [whole[500:1100]], [v]), {}), (([whole[::2]], [q], [m], [v]), {})]:
        with pytest.raises(g.GbmwError) as err:
            make(*args, **kw)
        assert err.value.status == g.GBMW_ERR_INVALID_ARG
    lst = make([p, whole[:600]], [q, q], [m, whole[600:]], [v, torch.zeros(600, device="cuda")])     # gradients may be shared
    for kw in (dict(lr=-1.0), dict(lr=math.nan), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(eps=1e-40), dict(scale=0.0), dict(max_norm=0.0), dict(step=0)):
        with pytest.raises(g.GbmwError) as err:
            g.gbmw_adamw_step(lst, **{**HOW, "step": 1, **kw})
        assert err.value.status == g.GBMW_ERR_INVALID_ARG
    for kw in (dict(lr=torch.zeros(1)), dict(step=torch.ones(1, device="cuda")), dict(norm=torch.ones(0, device="cuda"))):
        with pytest.raises(g.GbmwError):
            g.gbmw_adamw_step(lst, **{**HOW, "step": 1, **kw})


@pytest.mark.parametrize("seed", [0, 5])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("grad", [1e-15, 1e-18, -1e-19])
def test_gradients_whose_squares_are_below_the_normal_numbers(grad, bits, seed):
    import paper_2307_02031_amd as lib

    # v is g^2 (1 - beta2), with two roundings of half a step of 2^-149; a first step goes by lr g / |g|.  All values of the
    # block are its largest, so its codes are 448 whatever the rounding
    n = 300
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), grad, device="cuda")
    m, v = (torch.zeros(n, device="cuda").to(F8 if bits == 8 else torch.float32) for _ in range(2))
    scales = [torch.zeros(2, device="cuda") for _ in range(2)]
    how = dict(m_scales=scales[:1], v_scales=scales[1:]) if bits == 8 else {}
    lst = lib.gbmw_adamw_list_create([p], [g], [m], [v], **how)
    lib.gbmw_adamw_step(lst, 1.0, 1, beta1=0.9, beta2=0.999, eps=2.0 ** -126, seed=seed)
    value = float(np.float32(grad))
    square = value * value * 1e-3
    off = 2.0 ** -149 / square / 2 + 2.0 ** -20
    root = _held(v, scales[1]) if bits == 8 else v.cpu().double().sqrt()
    assert ((root - math.sqrt(square)).abs() <= off * math.sqrt(square)).all()
    want = -value / (abs(value) + 2.0 ** -126)
    assert ((p.cpu().double() - want).abs() <= off).all()
