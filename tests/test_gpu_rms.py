"""RMS norm, with a residual and to 8 bits, against plain forms in 64 bits.

Bounds are worked out before any run.  A sum of n squares in 32 bits, a thread's own values in a row and then a tree, is
off by at most (16 + log2 n + n / 256) 2^-24 of itself; half of that, and four roundings, is rstd's.  Everything after it
is products: each rounds by 2^-24 relative, and an output by half a step of its type."""
import math

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
TYPES = [(torch.float32, torch.float32), (torch.float16, torch.float16), (torch.float16, torch.float32),
         (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)]
IDS = ["f32", "f16", "f16-f32", "bf16", "bf16-f32"]


def _normal(*shape, dtype, seed, spread=1.0, middle=0.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=gen) * spread + middle).to(dtype).cuda()


def _sum_error(n):
    return 2.0 ** -24 * (16 + math.log2(n) + n / 256)


def _rel(n):
    return _sum_error(n) / 2 + 2.0 ** -22


def _forward(x, res, w, eps):
    """h (rounded, as it is normed), rstd, y in 64 bits."""
    h = ref.f64(x) if res is None else (x.float().cpu() + res.float().cpu()).to(x.dtype).double()
    rstd = 1.0 / torch.sqrt((h * h).mean(-1) + eps)
    y = h * rstd[..., None]
    return h, rstd, y if w is None else y * ref.f64(w)


def _check_forward(r, x, res, w, eps=1e-5, qtype=None, group=0):
    h, rstd, y = _forward(x, res, w, eps)
    n = x.shape[-1]
    if res is None:
        assert r.h is x
    else:
        assert torch.equal(r.h.cpu().double(), h)
    ref.assert_close("rstd", r.rstd, rstd, _rel(n) * rstd)
    off = _rel(n) + 2.0 ** -22
    if r.y is not None:
        ref.assert_close("y", r.y, y, (off + ref.U[x.dtype]) * y.abs() + ref.TINY[x.dtype])
    if qtype is None:
        assert r.q is None and r.scale is None
        return
    top, size = (448.0, group or n) if qtype == F8 else (127.0, group or n)
    parts = [c.abs().amax(-1) for c in y.split(size, -1)]
    scale = (torch.stack(parts, -1) / top).clamp_min(2.0 ** -126)
    assert r.scale.shape == (*x.shape[:-1], len(parts)) and r.q.dtype == qtype
    ref.assert_close("scale", r.scale, scale, (off + 2.0 ** -23) * scale)
    c = y / scale.repeat_interleave(size, -1)[..., :n]
    half = 0.5 if qtype == torch.int8 else torch.where(c.abs() < 2.0 ** -6, 2.0 ** -10, c.abs() * 2.0 ** -4)
    ref.assert_close("q", r.q.float(), c, half + (2 * off + 2.0 ** -21) * c.abs())


def _check_backward(dx, dw, dy, h, w, rstd, dres=None):
    n, rows = h.shape[-1], max(1, h.numel() // h.shape[-1])
    h64, dy64, r = ref.f64(h), ref.f64(dy), ref.f64(rstd)[..., None]
    w64 = torch.ones(n, dtype=torch.float64) if w is None else ref.f64(w)
    xhat, g = h64 * r, dy64 * w64
    c, mean_abs = (g * xhat).mean(-1, keepdim=True), (g * xhat).abs().mean(-1, keepdim=True)
    normed = (g - xhat * c) * r
    want = normed if dres is None else normed + ref.f64(dres)
    # rstd is given, so what is off is the sum, and a few roundings of each of the terms
    bound = r * (2.0 ** -21 * g.abs() + xhat.abs() * mean_abs * (_sum_error(n) + 2.0 ** -21))
    bound = bound + (ref.U[h.dtype] + 2.0 ** -23) * want.abs() + 2.0 ** -23 * normed.abs() + ref.TINY[h.dtype]
    ref.assert_close("dx", dx, want, bound)
    if w is None:
        assert dw is None
        return
    axes = tuple(range(h.dim() - 1))
    ref.assert_close("dweight", dw, (dy64 * xhat).sum(axes), (ref.U[w.dtype] + 2.0 ** -24) * (dy64 * xhat).sum(axes).abs() +
                     2.0 ** -24 * (20 + rows) * (dy64 * xhat).abs().sum(axes) + ref.TINY[w.dtype])


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (5, 7), (4, 63), (9, 64), (2, 257), (33, 500), (7, 1023), (6, 1283),
                                       (5, 2049), (3, 5120), (2, 8192), (3, 8193), (2, 16385), (1, 32768), (1500, 40),
                                       (4100, 136), (3000, 1544), (40, 2057), (5000, 392), (9, 12289), (3, 6145)])
def test_sizes(rows, cols, types):
    import paper_2307_02031_amd as g
    dtype, wdtype = types
    print("rms", rows, cols, dtype, wdtype, flush=True)
    x, res = (_normal(rows, cols, dtype=dtype, seed=cols + i, spread=1.0 + i) for i in range(2))
    w = _normal(cols, dtype=wdtype, seed=cols + 2, spread=0.3, middle=1.0)
    dy, dres = (_normal(rows, cols, dtype=dtype, seed=cols + 3 + i, spread=0.1) for i in range(2))
    for residual, weight, grad in ((res, w, dres), (None, w, None), (res, None, None), (None, None, dres)):
        r = g.gbmw_rms_norm_forward(x, weight, residual=residual)
        dx, dw = g.gbmw_rms_norm_backward(dy, r.h, weight, r.rstd, dres=grad)
        torch.cuda.synchronize()
        _check_forward(r, x, residual, weight)
        _check_backward(dx, dw, dy, r.h, weight, r.rstd, grad)


@pytest.mark.parametrize("qtype", [F8, torch.int8], ids=["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
def test_8_bits(group, dtype, qtype):
    import paper_2307_02031_amd as g
    for rows, cols in ((1, 1), (3, 5), (2, 31), (5, 33), (4, 128), (3, 129), (2, 1283), (3, 1531), (600, 260), (2, 5120),
                       (3, 9000), (1, 32768), (1, 32761)):
        print("rms 8 bits", rows, cols, dtype, qtype, group, flush=True)
        x, res = (_normal(rows, cols, dtype=dtype, seed=cols + i) for i in range(2))
        w = _normal(cols, dtype=dtype, seed=cols + 2, spread=0.3, middle=1.0)
        both = g.gbmw_rms_norm_forward(x, w, residual=res, qtype=qtype, group=group)
        only = g.gbmw_rms_norm_forward(x, w, residual=res, qtype=qtype, group=group, want_y=False)
        torch.cuda.synchronize()
        _check_forward(both, x, res, w, qtype=qtype, group=group)
        assert only.y is None and torch.equal(only.q.view(torch.uint8), both.q.view(torch.uint8))
        assert torch.equal(only.scale, both.scale) and torch.equal(only.h, both.h)


def test_8_bits_of_zeros_small_values_infinities_and_nan():
    import paper_2307_02031_amd as g
    x = torch.zeros(6, 300, device="cuda")
    x[1] = 1e-30                  # far below eps: y = x / sqrt(eps)
    x[2, 17], x[3, 200] = float("inf"), float("nan")
    x[4, :128] = _normal(128, dtype=torch.float32, seed=1)
    x[5] = _normal(300, dtype=torch.float32, seed=2) * 1e-36
    for group in (0, 128):
        r = g.gbmw_rms_norm_forward(x, qtype=F8, group=group)
        code, scale, y = r.q.float(), r.scale, r.y
        assert bool((code[0] == 0).all()) and bool((scale[0] == 2.0 ** -126).all())
        held = code * scale.repeat_interleave(group or 300, 1)[:, :300]
        for i in (1, 4, 5):
            # half a step of the largest of a group's, where scales and codes are normal numbers
            step = scale[i].repeat_interleave(group or 300)[:300] * 2.0 ** -10
            assert bool(((held[i] - y[i]).abs() <= y[i].abs() * (2.0 ** -4 + 1e-5) + step * 1.001).all())
        if group:
            assert bool((code[4, 128:] == 0).all()) and scale[4, 1] == 2.0 ** -126
        # an infinity makes rstd 0 and itself NaN, a NaN makes the row NaN
        assert bool(torch.isnan(y[2, 17])) and r.rstd[2] == 0 and bool(torch.isnan(y[3]).all())
        assert bool(torch.isnan(scale[3]).all()) and bool(torch.isnan(scale[2, 17 // (group or 300)]))


def test_fused_is_an_addition_and_a_norm():
    """The same bits as the norm of the sum, in every output and in the backward pass."""
    import paper_2307_02031_amd as g
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        x, res, dy = (_normal(70, 1283, dtype=dtype, seed=40 + i) for i in range(3))
        w = _normal(1283, dtype=torch.float32, seed=44)
        h = x + res
        a, b = (g.gbmw_rms_norm_forward(*p, qtype=F8, group=64) for p in ((x, w, 1e-5, res), (h, w, 1e-5)))
        assert torch.equal(a.h, h)
        for p, q in zip(a, b):
            assert torch.equal(p.view(torch.uint8), q.view(torch.uint8))


def test_strides_places_and_no_rows():
    import paper_2307_02031_amd as g
    x, res, dy, dres = (_normal(6, 5, 131, dtype=torch.bfloat16, seed=11 + i) for i in range(4))
    w = _normal(131, dtype=torch.float32, seed=15)
    base = g.gbmw_rms_norm_forward(x, w, residual=res, qtype=F8, group=32)
    grads = g.gbmw_rms_norm_backward(dy, base.h, w, base.rstd, dres=dres)
    same = lambda p, q: torch.equal(p.contiguous().view(torch.uint8), q.contiguous().view(torch.uint8))

    def wide(t, fill=7.0):
        big = torch.full((6, 5, 200), fill, device="cuda").to(t.dtype)
        big[..., 3:134] = t
        return big[..., 3:134]

    def untouched(t, fill=7.0):
        big = torch.as_strided(t, (6, 5, 200), (1000, 200, 1), t.storage_offset() - 3).float()
        return bool((big[..., :3] == fill).all()) and bool((big[..., 134:] == fill).all())

    zero = torch.zeros_like(x)
    out = dict(y=wide(zero), h=wide(zero), q=wide(torch.zeros(6, 5, 131, device="cuda").to(F8)))
    for p, q in zip(base, g.gbmw_rms_norm_forward(wide(x), w, residual=wide(res), qtype=F8, group=32, **out)):
        assert same(p, q)
    dx = wide(zero)
    for p, q in zip(grads, g.gbmw_rms_norm_backward(wide(dy), wide(base.h), w, base.rstd, dres=wide(dres), dx=dx)):
        assert same(p, q)
    assert all(untouched(t) for t in (*out.values(), dx))
    one = x[0, 0].expand(6, 5, 131)     # one row for all
    for p, q in zip(g.gbmw_rms_norm_forward(one.contiguous(), w, residual=res), g.gbmw_rms_norm_forward(one, w, residual=res)):
        assert p is q is None or same(p, q)
    # results over their inputs
    a, b = x.clone(), res.clone()
    r = g.gbmw_rms_norm_forward(a, w, residual=b, h=b, y=a)
    assert r.h is b and r.y is a and same(a, base.y) and same(b, base.h)
    a, b = x.clone(), res.clone()
    g.gbmw_rms_norm_forward(a, w, residual=b, h=a, y=b)
    assert same(b, base.y) and same(a, base.h)
    for over in range(2):
        d = [dy.clone(), dres.clone()]
        got = g.gbmw_rms_norm_backward(d[0], base.h, w, base.rstd, dres=d[1], dx=d[over])
        assert got[0] is d[over] and same(got[0], grads[0]) and same(got[1], grads[1])
    none = x[:0]
    r = g.gbmw_rms_norm_forward(none, w, residual=none, qtype=F8)
    dx, dw = g.gbmw_rms_norm_backward(none, none, w, r.rstd)
    torch.cuda.synchronize()
    assert r.y.shape == none.shape and r.scale.shape == (0, 5, 1) and dx.shape == none.shape and bool((dw == 0).all())


def test_same_bits_on_streams_and_in_a_graph():
    import paper_2307_02031_amd as g
    x, res, dy, dres = (_normal(700, 1280, dtype=torch.bfloat16, seed=21 + i) for i in range(4))
    w = _normal(1280, dtype=torch.float32, seed=25)

    def run(**kw):
        r = g.gbmw_rms_norm_forward(x, w, residual=res, qtype=F8, group=128, **kw)
        return [t.view(torch.uint8) for t in (*r, *g.gbmw_rms_norm_backward(dy, r.h, w, r.rstd, dres=dres, **kw))]

    base = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = run(stream=side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(base, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed in range(3):
        x.copy_(_normal(700, 1280, dtype=torch.bfloat16, seed=30 + seed))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(run(), got))


def test_workspace_of_just_the_bytes_asked_for():
    import paper_2307_02031_amd as g
    assert g.gbmw_rms_norm_workspace(torch.empty(2, 3, device="cuda")) == 0     # one workgroup writes dweight itself
    for rows, cols in ((200, 3), (700, 1280), (40, 9001)):
        x, dy = (_normal(rows, cols, dtype=torch.float16, seed=50 + i) for i in range(2))
        w = _normal(cols, dtype=torch.float16, seed=52)
        r = g.gbmw_rms_norm_forward(x, w)
        base = g.gbmw_rms_norm_backward(dy, x, w, r.rstd)
        need = g.gbmw_rms_norm_workspace(x, w)
        whole = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
        got = g.gbmw_rms_norm_backward(dy, x, w, r.rstd, workspace=whole[:need])
        assert all(torch.equal(p, q) for p, q in zip(base, got)) and bool((whole[need:] == 0x5a).all())
        with pytest.raises(g.GbmwError):
            g.gbmw_rms_norm_backward(dy, x, w, r.rstd, workspace=whole[:need - 4])


def test_gradients_against_differences():
    """Of sum(y * dy) + sum(h * dres), in float32: a step d moves the sum by its gradient times 2 d and an error of
    order d^3; what is left is the sums' own rounding."""
    import paper_2307_02031_amd as g
    x, res, dy, dres = (_normal(3, 50, dtype=torch.float32, seed=60 + i) for i in range(4))
    w = _normal(50, dtype=torch.float32, seed=64, middle=1.0)
    r = g.gbmw_rms_norm_forward(x, w, residual=res)
    dx, dw = g.gbmw_rms_norm_backward(dy, r.h, w, r.rstd, dres=dres)

    def total(x, w):
        r = g.gbmw_rms_norm_forward(x, w, residual=res)
        return float((r.y.double() * dy.double()).sum() + (r.h.double() * dres.double()).sum())

    d = 2.0 ** -6
    for i, j in ((0, 0), (1, 17), (2, 49)):
        hi, lo = x.clone(), x.clone()
        hi[i, j] += d
        lo[i, j] -= d
        # 150 values of order 1, each off by 2^-22: 1e-5 of the sum at most, over 2 d; d^2 = 2.4e-4 times a third derivative below 1
        assert abs((total(hi, w) - total(lo, w)) / (2 * d) - float(dx[i, j])) < 2e-3
        hi, lo = w.clone(), w.clone()
        hi[j] += d
        lo[j] -= d
        assert abs((total(x, hi) - total(x, lo)) / (2 * d) - float(dw[j])) < 2e-3


def test_shapes_of_one_axis_and_of_many():
    import paper_2307_02031_amd as g
    x, res, dy = (_normal(2, 3, 4, 130, dtype=torch.float16, seed=70 + i) for i in range(3))
    w = _normal(130, dtype=torch.float16, seed=74)
    r = g.gbmw_rms_norm_forward(x, w, residual=res, qtype=F8, group=64)
    dx, dw = g.gbmw_rms_norm_backward(dy, r.h, w, r.rstd)
    _check_forward(r, x, res, w, qtype=F8, group=64)
    _check_backward(dx, dw, dy, r.h, w, r.rstd)
    assert r.rstd.shape == (2, 3, 4) and r.scale.shape == (2, 3, 4, 3)
    one = g.gbmw_rms_norm_forward(x[1, 2, 3], w, residual=res[1, 2, 3], qtype=F8, group=64)
    assert one.rstd.shape == () and one.scale.shape == (3,)
    assert torch.equal(one.y, r.y[1, 2, 3]) and torch.equal(one.scale, r.scale[1, 2, 3]) and one.rstd == r.rstd[1, 2, 3]
    dx1, dw1 = g.gbmw_rms_norm_backward(dy[1, 2, 3], one.h, w, one.rstd)
    assert torch.equal(dx1, dx[1, 2, 3]) and dw1.shape == (130,)
    # rows that are not one stride apart have no row stride
    with pytest.raises(g.GbmwError):
        g.gbmw_rms_norm_forward(x[:, ::2, 1:], w)


def test_the_binding_refuses():
    import paper_2307_02031_amd as g
    x, w = _normal(4, 64, dtype=torch.bfloat16, seed=1), _normal(64, dtype=torch.float32, seed=2)
    r = g.gbmw_rms_norm_forward(x, w)
    for kw in (dict(weight=w[:5]), dict(weight=w.half()), dict(residual=x[:2]), dict(residual=x.float()), dict(residual=x.cpu()), dict(h=x.clone()),
               dict(q=x.to(F8)), dict(qtype=torch.uint8), dict(qtype=F8, group=16), dict(qtype=F8, group=-1), dict(qtype=F8, q=x), dict(y=x.float()),
               dict(y=x[:, :1].expand(4, 64)), dict(want_y=False), dict(eps=-1.0), dict(eps=math.inf), dict(residual=x[:1].expand(4, 64), h=x[:1].expand(4, 64)),
               dict(weight=torch.zeros(128, device="cuda")[::2])):
        with pytest.raises(g.GbmwError) as e:
            g.gbmw_rms_norm_forward(x, **{"weight": w, **kw})
        assert e.value.status == g.GBMW_ERR_INVALID_ARG, kw
    for args, kw in (((x[:2], x, w, r.rstd), {}), ((x, x, w, r.rstd[:2]), {}), ((x, x, w, r.rstd.half()), {}), ((x, x, w, r.rstd), dict(dres=x[:1])),
                     ((x, x, w, r.rstd), dict(dx=x.float())), ((x.float(), x, w, r.rstd), {})):
        with pytest.raises(g.GbmwError) as e:
            g.gbmw_rms_norm_backward(*args, **kw)
        assert e.value.status == g.GBMW_ERR_INVALID_ARG
