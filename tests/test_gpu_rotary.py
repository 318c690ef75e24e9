"""Rotary positions against a plain form in 64 bits.

Bounds, worked out before any run: the angle's fraction of a turn is rounded to 32 bits (2^-26 of a turn, 2^-23 radians),
cos and sin and their product with the factor are off by three more roundings, so each of an output's two products is off
by at most 2^-21 of its size, and the output by half a step of its type.  The angle itself is off by 2^-51 of its size
(the frequency over 2 pi, and the product with the position)."""
import math

import numpy as np
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.float16, torch.bfloat16]
IDS = ["f32", "f16", "bf16"]


def _normal(*shape, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=gen).to(dtype).cuda()


def _turned(x, freq, positions, interleaved, factor, sign):
    """value and bound in 64 bits; positions int64 [B][L]."""
    x64, rot = ref.f64(x), 2 * len(freq)
    angle = positions.cpu().numpy().astype(np.longdouble)[..., None] * freq.cpu().numpy().astype(np.longdouble)
    cos, sin = (torch.from_numpy(f(angle).astype(np.float64))[:, :, None] * factor for f in (np.cos, np.sin))
    sin = sin * sign
    far = torch.from_numpy(np.abs(angle).astype(np.float64))[:, :, None] * 2.0 ** -51 * abs(factor)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    out, bound = x64.clone(), torch.zeros_like(x64)
    u, v = x64[..., a], x64[..., b]
    out[..., a], out[..., b] = u * cos - v * sin, u * sin + v * cos
    size = (u.abs() + v.abs()) * (2.0 ** -21 * abs(factor) + far)
    bound[..., a] = size + ref.U[x.dtype] * out[..., a].abs() + ref.TINY[x.dtype]
    bound[..., b] = size + ref.U[x.dtype] * out[..., b].abs() + ref.TINY[x.dtype]
    return out, bound


def _check(q, k, freq, positions=None, interleaved=False, factor=1.0):
    import paper_2307_02031_amd as g
    B, L = q.shape[:2]
    pos = torch.arange(L).expand(B, L) if positions is None else positions.long()
    for call, sign in ((g.gbmw_rotary_forward, 1.0), (g.gbmw_rotary_backward, -1.0)):
        got = call(q, k, freq, positions=positions, interleaved=interleaved, factor=factor)
        torch.cuda.synchronize()
        for name, x, y in (("q", q, got[0]), ("k", k, got[1])):
            if x is None:
                assert y is None
            else:
                ref.assert_close(name, y, *_turned(x, freq, pos, interleaved, factor, sign))
        if k is not None:
            places = [q.clone(), k.clone()]
            here = call(*places, freq, positions=positions, interleaved=interleaved, factor=factor, q_out=places[0], k_out=places[1])
            assert here[0] is places[0] and all(torch.equal(a, b) for a, b in zip(here, got))


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "pairs"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_sizes(dtype, interleaved):
    import paper_2307_02031_amd as g
    for B, L, Hq, Hk, D, rot in [(1, 1, 1, 1, 2, 2), (2, 3, 1, 1, 1, 0), (1, 5, 3, 1, 7, 4), (3, 17, 4, 2, 40, 40), (2, 33, 5, 5, 80, 32),
                                 (1, 9, 2, 1, 96, 38), (2, 70, 8, 2, 128, 128), (1, 40, 40, 40, 64, 64), (2, 5, 1, 1, 64, 6),
                                 (1, 3, 70, 2, 16, 8), (1, 2, 3, 1, 512, 512), (1, 2, 2, 2, 300, 258), (5, 1, 32, 8, 128, 64),
                                 (1, 4500, 1, 1, 8, 8), (2, 9, 6, 3, 45, 44), (1, 6, 2, 2, 511, 2)]:
        print("rotary", dtype, interleaved, (B, L, Hq, Hk, D, rot), flush=True)
        q, k = _normal(B, L, Hq, D, dtype=dtype, seed=D + L), _normal(B, L, Hk, D, dtype=dtype, seed=D + L + 1)
        freq = g.gbmw_rotary_frequencies(rot)
        _check(q, k, freq, interleaved=interleaved)
        _check(q, None, freq, interleaved=interleaved, factor=-0.5)


def test_far_and_negative_positions():
    import paper_2307_02031_amd as g
    q, k = _normal(4, 6, 3, 64, dtype=torch.float32, seed=1), _normal(4, 6, 1, 64, dtype=torch.float32, seed=2)
    starts = torch.tensor([[0], [131072], [-70], [2 ** 31 - 6]])
    pos = (starts + torch.arange(6)).to(torch.int32).cuda()
    for scaling in (dict(), dict(scaling="linear", by=4.0), dict(scaling="base", by=8.0),
                    dict(scaling="ramp", by=8.0, original=4096.0), dict(scaling="ramp", by=2.0, original=512.0, slow=0.5, fast=4.0)):
        _check(q, k, g.gbmw_rotary_frequencies(64, 500000.0, **scaling), positions=pos, factor=1.25)
    _check(q, k, torch.tensor([0.0, 3.0, -1.0], dtype=torch.float64, device="cuda"), positions=pos)
    # one row of positions for all samples
    one = torch.arange(100, 106, dtype=torch.int32, device="cuda").expand(4, 6)
    _check(q, k, g.gbmw_rotary_frequencies(32), positions=one)


def test_values_turn_by_relative_position():
    """<turned q, turned k> depends on the distance alone: at far positions as at near ones."""
    import paper_2307_02031_amd as g
    q, k = (_normal(1, 1, 1, 128, dtype=torch.float32, seed=i) for i in (5, 6))
    freq = g.gbmw_rotary_frequencies(128)
    at = lambda x, p: g.gbmw_rotary_forward(x, None, freq, positions=torch.tensor([[p]], dtype=torch.int32, device="cuda"))[0]
    near = float((at(q, 7).double() * at(k, 3).double()).sum())
    far = float((at(q, 1000007).double() * at(k, 1000003).double()).sum())
    size = float(q.double().norm() * k.double().norm())
    assert abs(near - far) < 8 * 2.0 ** -21 * size


@pytest.mark.parametrize("D,rot", [(64, 64), (80, 40), (33, 10)])
def test_lengths_and_strides(D, rot):
    """Rows from a sample's length on are neither read nor written; inputs and outputs are parts of wider arrays."""
    import paper_2307_02031_amd as g
    B, L, Hq, Hk = 4, 21, 6, 2
    n = torch.tensor([21, 0, 7, 1], dtype=torch.int32, device="cuda")
    qkv = _normal(B, L, (Hq + 2 * Hk) * D, dtype=torch.bfloat16, seed=9)
    dense = [t.unflatten(2, (-1, D)).contiguous() for t in qkv.split([Hq * D, Hk * D, Hk * D], 2)]
    freq = g.gbmw_rotary_frequencies(rot)
    want = g.gbmw_rotary_forward(dense[0], dense[1], freq)
    for b, m in enumerate(n.tolist()):
        qkv[b, m:] = float("nan")
    q, k, v = (t.unflatten(2, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], 2))
    outs = [torch.full((B, L, H, D + 5), 3.0, dtype=torch.bfloat16, device="cuda") for H in (Hq, Hk)]
    got = g.gbmw_rotary_forward(q, k, freq, len_x=n, q_out=outs[0][..., 2:D + 2], k_out=outs[1][..., 2:D + 2])
    torch.cuda.synchronize()
    for b, m in enumerate(n.tolist()):
        for out, res, ref_ in zip(outs, got, want):
            assert torch.equal(res[b, :m], ref_[b, :m])
            assert bool((out[b, m:] == 3).all()) and bool((out[..., :2] == 3).all()) and bool((out[..., D + 2:] == 3).all())
    # lengths beyond the rows, and below none
    off = g.gbmw_rotary_forward(dense[0], None, freq, len_x=torch.tensor([L + 9, -3, 7, 2 ** 31 - 1], dtype=torch.int32, device="cuda"),
                                q_out=torch.zeros_like(dense[0]))[0]
    for b, m in enumerate((L, 0, 7, L)):
        assert torch.equal(off[b, :m], want[0][b, :m]) and bool((off[b, m:] == 0).all())
    # in place in the product's own array: v and the rows behind stay
    before = qkv.clone()
    g.gbmw_rotary_forward(q, k, freq, len_x=n, q_out=q, k_out=k)
    torch.cuda.synchronize()
    assert torch.equal(torch.nan_to_num(v), torch.nan_to_num(before[..., (Hq + Hk) * D:].unflatten(2, (-1, D))))
    for b, m in enumerate(n.tolist()):
        assert torch.equal(q[b, :m], want[0][b, :m]) and torch.equal(k[b, :m], want[1][b, :m])
        assert bool(torch.isnan(qkv[b, m:]).all())
    # heads before rows, and values broadcast over samples
    heads = dense[0].transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(g.gbmw_rotary_forward(heads, None, freq)[0], want[0])
    one = dense[0][:1].expand(B, L, Hq, D)
    assert torch.equal(g.gbmw_rotary_forward(one, None, freq)[0], want[0][:1].expand(B, L, Hq, D))


def test_backward_is_the_transpose():
    """<forward(x), y> = <x, backward(y)>, and a forward call undoes a backward one where the factor is 1."""
    import paper_2307_02031_amd as g
    x, y = (_normal(2, 50, 4, 80, dtype=torch.float32, seed=i) for i in (20, 21))
    freq = g.gbmw_rotary_frequencies(40)
    for inter in (False, True):
        a = g.gbmw_rotary_forward(x, None, freq, interleaved=inter, factor=1.5)[0]
        b = g.gbmw_rotary_backward(y, None, freq, interleaved=inter, factor=1.5)[0]
        size = float(x.double().norm() * y.double().norm())
        assert abs(float((a.double() * y.double()).sum() - (x.double() * b.double()).sum())) < 4 * 2.0 ** -21 * size
        back = g.gbmw_rotary_backward(g.gbmw_rotary_forward(x, None, freq, interleaved=inter)[0], None, freq, interleaved=inter)[0]
        assert float((back - x).abs().max()) < 8 * 2.0 ** -21 * float(x.abs().max())


def test_no_rows_streams_and_a_graph():
    import paper_2307_02031_amd as g
    freq = g.gbmw_rotary_frequencies(64)
    q, k = _normal(3, 100, 8, 64, dtype=torch.bfloat16, seed=1), _normal(3, 100, 2, 64, dtype=torch.bfloat16, seed=2)
    assert g.gbmw_rotary_forward(q[:0], k[:0], freq)[0].shape == (0, 100, 8, 64)
    assert g.gbmw_rotary_forward(q[:, :0], k[:, :0], freq)[1].shape == (3, 0, 2, 64)
    pos = torch.arange(100, dtype=torch.int32, device="cuda").expand(3, 100).contiguous()
    base = g.gbmw_rotary_forward(q, k, freq, positions=pos)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = g.gbmw_rotary_forward(q, k, freq, positions=pos, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(base, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = g.gbmw_rotary_forward(q, k, freq, positions=pos)
    for i in range(3):
        pos += 1000
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(g.gbmw_rotary_forward(q, k, freq, positions=pos), got))


def test_the_binding_refuses():
    import paper_2307_02031_amd as g
    freq = g.gbmw_rotary_frequencies(8)
    q, k = _normal(2, 3, 4, 8, dtype=torch.float32, seed=1), _normal(2, 3, 2, 8, dtype=torch.float32, seed=2)
    pos = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    for args, kw in [((q[0], k, freq), {}), ((q, k[:, :2], freq), {}), ((q, k.half(), freq), {}), ((q, k, freq.float()), {}),
                     ((q, k, torch.zeros(5, dtype=torch.float64, device="cuda")), {}), ((q, k, freq.cpu()), {}),
                     ((q, k, freq), dict(positions=pos.long())), ((q, k, freq), dict(positions=pos[:1])),
                     ((q, k, freq), dict(positions=pos.t().contiguous().t())), ((q, k, freq), dict(len_x=pos[0])), ((q, k, freq), dict(factor=1e39)), ((q, k, freq), dict(factor=math.nan)),
                     ((q, k, freq), dict(q_out=k)), ((q, None, freq), dict(k_out=k)), ((q, k, freq), dict(factor=math.inf)),
                     ((q, k, freq), dict(q_out=q[:1].expand(2, 3, 4, 8))), ((q.transpose(1, 3).contiguous().transpose(1, 3), k, freq), {})]:
        with pytest.raises(g.GbmwError) as e:
            g.gbmw_rotary_forward(*args, **kw)
        assert e.value.status == g.GBMW_ERR_INVALID_ARG
