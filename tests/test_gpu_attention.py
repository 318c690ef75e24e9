"""Attention against a plain form in 64 bits: head layouts, types, lengths from zero on, sizes off every tile edge,
masks that leave rows empty, strides, streams, graphs."""
import itertools

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu


def _inputs(B, Lq, Lk, Hq, Hk, D, dtype, seed=0, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    new = lambda *s: (torch.randn(*s, generator=gen) * spread).to(dtype).cuda()
    return new(B, Lq, Hq, D), new(B, Lk, Hk, D), new(B, Lk, Hk, D), new(B, Lq, Hq, D)


def _check(q, k, v, dout, backward=True, **mask):
    import paper_2307_02031_amd as g
    print("attention", tuple(q.shape), tuple(k.shape), q.dtype, {n: getattr(m, "tolist", lambda: m)() for n, m in mask.items()},
          flush=True)
    out, lse = g.gbmw_attention_forward(q, k, v, **mask)
    got = dict(out=out, lse=lse)
    if backward:
        got["dq"], got["dk"], got["dv"] = g.gbmw_attention_backward(dout, q, k, v, out, lse, **mask)
    torch.cuda.synchronize()
    want = ref.attention(q, k, v, dout=dout if backward else None, out_given=out, **mask)
    for n, t in got.items():
        assert t.shape == want[n][0].shape
        ref.assert_close(n, t, *want[n])
    return got


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("D", [1, 8, 17, 32, 40, 48, 64, 72, 80, 96, 100, 128])
def test_head_sizes(D, dtype):
    _check(*_inputs(2, 70, 150, 2, 2, D, dtype, seed=D))
    _check(*_inputs(1, 130, 130, 2, 1, D, dtype, seed=D + 1), causal=True)


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("Lq,Lk", [(1, 1), (1, 2), (1, 64), (1, 65), (2, 1), (3, 700), (31, 33), (32, 32), (64, 63), (65, 64),
                                   (127, 129), (128, 128), (129, 127), (197, 197), (256, 1), (300, 20), (20, 300), (513, 512)])
def test_lengths(Lq, Lk, causal):
    """More queries than keys under a causal mask: the first rows see nothing."""
    got = _check(*_inputs(1, Lq, Lk, 2, 2, 64, torch.bfloat16, seed=Lq * 1000 + Lk), causal=causal)
    if causal and Lq > Lk:
        assert bool((got["out"][:, :Lq - Lk] == 0).all()) and bool(torch.isneginf(got["lse"][:, :, :Lq - Lk]).all())
        assert bool((got["dq"][:, :Lq - Lk] == 0).all())


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (4, 4), (4, 1), (6, 2), (7, 1), (5, 5), (32, 4)])
def test_shared_heads(Hq, Hk):
    for i, (Lq, Lk, causal) in enumerate([(1, 90, True), (50, 50, True), (33, 70, False), (80, 40, True)]):
        _check(*_inputs(2, Lq, Lk, Hq, Hk, 80, torch.float16, seed=Hq * 10 + i), causal=causal)


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_lengths_of_samples(causal):
    """Samples from empty to full, and values outside the arrays: what lies beyond a length is not used, NaN or not."""
    nq = torch.tensor([0, 1, 130, 77, 64, 130, 999, -3], dtype=torch.int32, device="cuda")
    nk = torch.tensor([5, 0, 1, 64, 200, 200, 999, 10], dtype=torch.int32, device="cuda")
    q, k, v, dout = _inputs(8, 130, 200, 4, 2, 64, torch.bfloat16, seed=3)
    for b in range(8):
        n, m = min(max(int(nq[b]), 0), 130), min(max(int(nk[b]), 0), 200)
        q[b, n:], dout[b, n:], k[b, m:], v[b, m:] = float("nan"), float("inf"), float("nan"), float("-inf")
    got = _check(q, k, v, dout, causal=causal, len_q=nq, len_k=nk)
    for b in range(8):
        n, m = min(max(int(nq[b]), 0), 130), min(max(int(nk[b]), 0), 200)
        assert bool((got["out"][b, n:] == 0).all()) and bool((got["dq"][b, n:] == 0).all())
        assert bool((got["dk"][b, m:] == 0).all()) and bool((got["dv"][b, m:] == 0).all())
        assert bool(torch.isneginf(got["lse"][b, :, n:]).all())


def test_no_rows_or_no_keys():
    import paper_2307_02031_amd as g
    for B, Lq, Lk in [(0, 5, 5), (2, 0, 5), (2, 5, 0), (1, 0, 0)]:
        q, k, v, dout = _inputs(B, Lq, Lk, 2, 2, 64, torch.float16)
        out, lse = g.gbmw_attention_forward(q, k, v)
        dq, dk, dv = g.gbmw_attention_backward(dout, q, k, v, out, lse)
        torch.cuda.synchronize()
        assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())
        assert all(bool((t == 0).all()) for t in (dq, dk, dv))


def test_scores_of_any_size():
    """Probabilities of 0 and 1 in the type, and a scale of 0: the mean of the values that are seen."""
    q, k, v, dout = _inputs(1, 150, 150, 2, 2, 64, torch.bfloat16, seed=9, spread=3.0)
    _check(q, k, v, dout, causal=True)
    _check(q, k, v, dout, causal=True, scale=0.0)
    _check(q, k, v, dout, scale=1e-4)
    # scores of +-1e4: one key takes all, or none of them counts
    import paper_2307_02031_amd as g
    q, k, v, _ = _inputs(1, 64, 64, 1, 1, 16, torch.bfloat16, seed=10)
    q[..., 1:], k[..., 1:], q[..., 0] = 0, 0, 100
    k[0, :, 0, 0] = -100
    k[0, 5, 0, 0] = 100
    out, lse = g.gbmw_attention_forward(q, k, v, scale=1.0)
    assert bool((out == v[:, 5:6]).all()) and bool((lse == 1e4).all())
    k[0, 5, 0, 0] = -100
    out, lse = g.gbmw_attention_forward(q, k, v, scale=1.0)
    want = v.double().mean(1, keepdim=True).expand(out.shape)
    ref.assert_close("out", out, want.cpu(), 2.0 ** -6 * v.double().abs().mean(1, keepdim=True).expand(out.shape).cpu())


def test_a_nan_in_a_row_stays_in_its_rows():
    """A NaN query makes its own row NaN and no other; a NaN key every row that sees it."""
    import paper_2307_02031_amd as g
    q, k, v, _ = _inputs(1, 100, 100, 1, 1, 64, torch.bfloat16, seed=11)
    q[0, 40] = float("nan")
    out, lse = g.gbmw_attention_forward(q, k, v)
    bad = torch.isnan(out).any(-1).flatten()
    assert bool(bad[40]) and int(bad.sum()) == 1 and int(torch.isnan(lse).sum()) == 1
    q, k, v, _ = _inputs(1, 100, 100, 1, 1, 64, torch.bfloat16, seed=11)
    k[0, 90] = float("nan")
    out, _ = g.gbmw_attention_forward(q, k, v)
    assert bool(torch.isnan(out).any(-1).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_strides_and_alignment(dtype):
    """Heads before rows, parts of one product, every second row, arrays that start at any element, broadcast keys:
    the same bits as from dense arrays."""
    import paper_2307_02031_amd as g
    B, L, H, D = 2, 90, 3, 72
    q, k, v, dout = _inputs(B, L, L, H, H, D, dtype, seed=21)

    def run(q, k, v, dout, outs=None):
        out, lse = g.gbmw_attention_forward(q, k, v, causal=True, out=None if outs is None else outs[0])
        grads = g.gbmw_attention_backward(dout, q, k, v, out, lse, causal=True,
                                          **({} if outs is None else dict(zip(("dq", "dk", "dv"), outs[1:]))))
        return [out, lse, *grads]

    base = run(q, k, v, dout)

    def heads_first(t):
        return t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)

    def every_second(t):
        w = torch.full((B, 2 * L, H, D + 5), float("nan"), dtype=dtype, device="cuda")
        w[:, ::2, :, 3:3 + D] = t
        return w[:, ::2, :, 3:3 + D]

    def part_of_product(t):
        w = torch.full((B, L, 3 * H * D), float("nan"), dtype=dtype, device="cuda")
        w[:, :, H * D:2 * H * D] = t.flatten(2)
        return w[:, :, H * D:2 * H * D].unflatten(2, (H, D))

    def off_by_one(t):
        w = torch.empty(t.numel() + 1, dtype=dtype, device="cuda")
        w[1:] = t.flatten()
        return w[1:].view(t.shape)

    for how in (heads_first, every_second, part_of_product, off_by_one):
        print(how.__name__, flush=True)
        outs = [how(torch.zeros_like(q)) for _ in range(4)]
        for x, y in zip(base, run(*map(how, (q, k, v, dout)), outs)):
            assert torch.equal(x, y)
    one = k[:1, :, :1].expand(B, L, H, D)
    for x, y in zip(run(q, one.contiguous(), v, dout), run(q, one, v, dout)):
        assert torch.equal(x, y)


def test_offsets_beyond_32_bits():
    """Samples and heads that lie more than 2^32 bytes apart."""
    import paper_2307_02031_amd as g
    q, k, v, dout = _inputs(2, 70, 130, 2, 2, 64, torch.bfloat16, seed=31)
    base = g.gbmw_attention_forward(q, k, v, causal=True)
    far = torch.empty((5 << 30) // 2, dtype=torch.bfloat16, device="cuda")

    def spread(t, at):
        L = t.shape[1]
        s = torch.as_strided(far, t.shape, ((3 << 30) // 2 - 4096, 3 * 64, (1 << 30) // 2 + 64, 1), at)
        s.copy_(t)
        return s

    qf, kf, vf = spread(q, 0), spread(k, 1 << 20), spread(v, 2 << 20)
    out, lse = g.gbmw_attention_forward(qf, kf, vf, causal=True)
    assert torch.equal(out, base[0]) and torch.equal(lse, base[1])
    for x, y in zip(g.gbmw_attention_backward(dout, q, k, v, *base, causal=True),
                    g.gbmw_attention_backward(dout, qf, kf, vf, out, lse, causal=True)):
        assert torch.equal(x, y)


def test_same_bits_again_and_on_another_stream():
    import paper_2307_02031_amd as g
    q, k, v, dout = _inputs(2, 200, 333, 4, 2, 128, torch.bfloat16, seed=41)

    def run(**kw):
        out, lse = g.gbmw_attention_forward(q, k, v, **kw)
        return [out, lse, *g.gbmw_attention_backward(dout, q, k, v, out, lse, **kw)]

    base = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        for x, y in zip(base, run()):
            assert torch.equal(x, y)
        got = run(stream=side)
        junk = [torch.full_like(t, 7) for t in base]     # memory of this stream, asked for while the side stream runs
        side.synchronize()
        for x, y in zip(base, got):
            assert torch.equal(x, y)
        with torch.cuda.stream(side):
            got = run()
        side.synchronize()
        for x, y in zip(base, got):
            assert torch.equal(x, y)


def test_in_a_graph():
    import paper_2307_02031_amd as g
    q, k, v, dout = _inputs(1, 100, 260, 2, 1, 64, torch.float16, seed=51)

    def run():
        out, lse = g.gbmw_attention_forward(q, k, v, causal=True)
        return [out, lse, *g.gbmw_attention_backward(dout, q, k, v, out, lse, causal=True)]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed in range(3):
        for t, new in zip((q, k, v, dout), _inputs(1, 100, 260, 2, 1, 64, torch.float16, seed=60 + seed)):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(run(), got):
            assert torch.equal(x, y)


def test_gradients_against_differences():
    """The loss sum(out * w) along random directions, from the plain form in 64 bits at both ends."""
    import paper_2307_02031_amd as g
    q, k, v, w = _inputs(1, 40, 50, 4, 2, 32, torch.float16, seed=71)
    nk = torch.tensor([45], dtype=torch.int32, device="cuda")
    out, lse = g.gbmw_attention_forward(q, k, v, causal=True, len_k=nk)
    grads = g.gbmw_attention_backward(w, q, k, v, out, lse, causal=True, len_k=nk)
    gen = torch.Generator().manual_seed(5)
    x = [t.cpu().double() for t in (q, k, v)]
    want = ref.attention(q, k, v, causal=True, len_k=nk, dout=w, out_given=out)
    h = 1e-4

    def loss(*a):
        # the plain form takes its type's bounds from q; values stay 64 bits
        Lq, Lk = a[0].shape[1], a[1].shape[1]
        m = ref.sees(Lq, Lk, True, Lq, 45)
        total = 0.0
        for hq in range(4):
            s = torch.where(m, a[0][0, :, hq] @ a[1][0, :, hq // 2].T * 32 ** -0.5, -torch.inf)
            total = total + (torch.softmax(s[:, :45], 1) @ a[2][0, :45, hq // 2] * w[0, :, hq].cpu().double()).sum()
        return float(total)

    for which in range(3):
        d = torch.randn(x[which].shape, generator=gen, dtype=torch.float64)
        ends = [loss(*[t + s * h * d if n == which else t for n, t in enumerate(x)]) for s in (1, -1)]
        slope = (ends[0] - ends[1]) / (2 * h)
        name = ("dq", "dk", "dv")[which]
        allowed = float((want[name][1] * d.abs()).sum()) + 1e-5 * float((want[name][0] * d).abs().sum())
        assert abs(float((grads[which].cpu().double() * d).sum()) - slope) <= allowed, name


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_small_gradients_keep_their_digits(dtype):
    """Gradients of a thousandth, spread over a thousand keys: score gradients far below float16's normal numbers."""
    q, k, v, dout = _inputs(1, 64, 1000, 1, 1, 64, dtype, seed=81)
    dout = (dout.float() * 1e-3).to(dtype)
    import paper_2307_02031_amd as g
    out, lse = g.gbmw_attention_forward(q, k, v)
    dq, dk, dv = g.gbmw_attention_backward(dout, q, k, v, out, lse)
    want = ref.attention(q, k, v, dout=dout, out_given=out)
    for n, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        value = want[n][0]
        off = (ref.f64(t) - value).norm() / value.norm()
        # two roundings of half an ulp at most, and the outputs' own steps (dk in float16 is below its normal numbers)
        steps = ref.TINY[dtype] * value.numel() ** 0.5 / value.norm()
        assert off <= 2 * ref.U[dtype] + steps, (n, float(off))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("B,Lq,Lk,Hq,Hk,D", [(1, 1, 5000, 8, 2, 128), (2, 1, 4097, 4, 4, 64), (1, 8, 3001, 8, 2, 80), (3, 5, 700, 6, 6, 40),
                                             (1, 33, 2500, 2, 2, 96), (1, 200, 1700, 2, 1, 64), (1, 1, 1100, 3, 1, 17),
                                             (1, 32, 6000, 1, 1, 128), (1, 40, 1300, 1, 1, 127)])
def test_few_rows_and_many_keys(B, Lq, Lk, Hq, Hk, D, dtype):
    """Where several workgroups, and several waves of one, share the keys of a row."""
    q, k, v, dout = _inputs(B, Lq, Lk, Hq, Hk, D, dtype, seed=Lk)
    _check(q, k, v, dout)
    _check(q, k, v, dout, causal=True)
    nk = torch.tensor([Lk - 70, 3, 0][:B], dtype=torch.int32, device="cuda")
    nq = torch.tensor([Lq, max(1, Lq - 1), Lq][:B], dtype=torch.int32, device="cuda")
    _check(q, k, v, dout, causal=True, len_q=nq, len_k=nk)


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_few_keys_and_many_rows(causal):
    """Where several workgroups share the rows that see a key."""
    _check(*_inputs(1, 2100, 130, 2, 1, 64, torch.bfloat16, seed=91), causal=causal)
    _check(*_inputs(1, 1500, 1500, 4, 1, 40, torch.float16, seed=92), causal=causal)


def test_strides_of_extents_of_one():
    """They may hold anything, and count for nothing."""
    import paper_2307_02031_amd as g
    q, k, v, dout = _inputs(1, 1, 1, 1, 1, 64, torch.bfloat16, seed=95)
    base = g.gbmw_attention_forward(q, k, v)
    odd = [torch.as_strided(t, t.shape, (1 << 50, 7, 3, 1)) for t in (q, k, v, dout)]
    got = g.gbmw_attention_forward(*odd[:3])
    assert torch.equal(base[0], got[0]) and torch.equal(base[1], got[1]) and torch.equal(base[0], v)
    for x, y in zip(g.gbmw_attention_backward(dout, q, k, v, *base), g.gbmw_attention_backward(odd[3], *odd[:3], *got)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("B,Lq,Lk,Hq,Hk,D", [(1, 1, 1, 1, 1, 8), (3, 8, 8, 6, 6, 64), (5, 3, 19, 4, 2, 96), (2, 16, 8, 2, 2, 128), (4, 4, 32, 3, 3, 40),
                                             (2, 2, 7, 8, 1, 17), (3, 0, 9, 2, 2, 64), (9, 11, 11, 2, 1, 80)])
def test_gradients_of_few_rows_and_keys_are_rounded_once(B, Lq, Lk, Hq, Hk, D, dtype):
    """Few terms do not average their roundings out.  Bound: the result's rounding; probabilities from a log-sum-exp and
    an exponential good to 2^-18 (1 + |lse|), |lse| < 7 here, so 2^-15 of each term; up to 11 x 2 rows or 32 keys and
    256 products in 32 bits, far less.  Past the kernel's sizes (11 x 11 rows of two heads) the usual bound."""
    import paper_2307_02031_amd as g
    q, k, v, dout = _inputs(B, Lq, Lk, Hq, Hk, D, dtype, seed=17)
    wide = torch.full((B, Lk, 2 * Hk, D), float("nan"), dtype=dtype, device="cuda")
    wide[:, :, :Hk] = k
    k = wide[:, :, :Hk]                                            # heads of a larger row
    n = torch.arange(B, dtype=torch.int32, device="cuda")
    for mask in (dict(), dict(causal=True), dict(causal=True, len_q=(Lq - n).clamp(0), len_k=(Lk - 2 * n).clamp(0)), dict(scale=0.4)):
        got = _check(q, k, v, dout, **mask)
        if Lq * Hq // Hk * Lk > 128:
            continue
        want = ref.attention(q, k, v, dout=dout, out_given=got["out"], **mask)
        terms = _terms(q, k, v, dout, **mask)
        u = ref.U[dtype]
        for name in ("dq", "dk", "dv"):
            bound = u * want[name][0].abs() + 2.0 ** -15 * terms[name] + ref.TINY[dtype]
            ref.assert_close(name, got[name], want[name][0], bound)


def _terms(q, k, v, dout, causal=False, scale=None, len_q=None, len_k=None):
    """The sums of the terms' sizes in dq, dk and dv."""
    q, k, v, dout = (ref.f64(t) for t in (q, k, v, dout))
    (B, Lq, Hq, D), (Lk, Hk) = q.shape, k.shape[1:3]
    scale = D ** -0.5 if scale is None else scale
    res = dict(dq=torch.zeros_like(q), dk=torch.zeros_like(v), dv=torch.zeros_like(v))
    for b, h in itertools.product(range(B), range(Hq)):
        nq, nk = (L if n is None else int(n[b]) for L, n in ((Lq, len_q), (Lk, len_k)))
        m, kh = ref.sees(Lq, Lk, causal, nq, nk)[:nq, :nk], h * Hk // Hq
        qq, dd, kk, vv = q[b, :nq, h], dout[b, :nq, h], k[b, :nk, kh], v[b, :nk, kh]
        p = torch.where(m, torch.softmax(torch.where(m, scale * qq @ kk.T, -1e300), 1), 0.0)
        dp = dd.abs() @ vv.abs().T
        ds = p * (dp + (p * dp).sum(1, keepdim=True))
        res["dq"][b, :nq, h] = scale * ds @ kk.abs()
        res["dk"][b, :nk, kh] += scale * ds.T @ qq.abs()
        res["dv"][b, :nk, kh] += p.T @ dd.abs()
    return res
