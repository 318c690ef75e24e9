"""What RMS norm, rotary positions and AdamW refuse, through the C entry points and without a device, and the rotary
frequencies, which the host computes."""
import ctypes as ct
import math

import numpy as np
import pytest
import torch

no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="checks the host side with made-up addresses, without a device")


def _rms(g, **over):
    p = g.gbmw_rms_norm_problem()
    for i, n in enumerate(("x", "residual", "weight", "h", "y", "q", "scale", "rstd", "dy", "dres", "dx", "dweight", "workspace")):
        setattr(p, n, (i + 1) << 20)
    p.dtype, p.wdtype, p.rows, p.cols, p.eps, p.qtype, p.group = g.GBMW_BF16, g.GBMW_F32, 1000, 64, 1e-5, g.GBMW_E4M3, 32
    for n in ("x", "residual", "h", "y", "q", "dy", "dres", "dx"):
        setattr(p, n + "_stride", 64)
    p.workspace_bytes = 1 << 20
    for n, x in over.items():
        setattr(p, n, x)
    return p


@no_device
def test_rms_refuses():
    import paper_2307_02031_amd as g
    fwd, bwd = g._lib.gbmw_rms_norm_forward, g._lib.gbmw_rms_norm_backward
    both = [(dict(dtype=3), "dtype"), (dict(wdtype=g.GBMW_F16), "wdtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"),
            (dict(cols=0), "cols"), (dict(cols=32769), "cols"), (dict(x=None), "x is null"), (dict(x=(1 << 20) + 1), "x is not aligned"),
            (dict(x_stride=-1), "x: row stride"), (dict(rstd=2), "rstd"), (dict(weight=(1 << 20) + 2), "weight")]
    only = {0: [(dict(eps=-1.0), "eps"), (dict(eps=math.nan), "eps"), (dict(y=None, q=None), "neither"), (dict(y_stride=63), "y: row stride"),
                (dict(h_stride=3), "h: row stride"), (dict(q_stride=63), "q: row stride"), (dict(qtype=2), "qtype"), (dict(group=16), "group"),
                (dict(group=-1), "group"), (dict(scale=None), "scale"), (dict(scale=2), "scale"), (dict(residual=3), "residual"),
                (dict(y=1 << 20, x_stride=65), "y is x"), (dict(h=2 << 20, residual_stride=70), "h is residual"),
                (dict(h=5 << 20), "one array")],
            1: [(dict(dy=None), "dy"), (dict(dx=None), "dx"), (dict(rstd=None), "rstd"), (dict(dx_stride=3), "dx: row stride"),
                (dict(dres=(1 << 20) + 1), "dres"), (dict(workspace=None), "workspace"), (dict(workspace_bytes=64), "workspace"),
                (dict(workspace=(1 << 20) + 8), "workspace"), (dict(dweight=(1 << 20) + 2), "dweight"), (dict(dx=9 << 20, dx_stride=70), "dx is dy"),
                (dict(dx=10 << 20, dx_stride=70), "dx is dres")]}
    for i, call in enumerate((fwd, bwd)):
        assert call(None) == g.GBMW_ERR_INVALID_ARG
        for over, word in both + only[i]:
            assert call(ct.byref(_rms(g, **over))) == g.GBMW_ERR_INVALID_ARG, over
            assert word in g.gbmw_last_error(), (over, g.gbmw_last_error())
    assert fwd(ct.byref(_rms(g, rows=0, x=None, y=None))) == g.GBMW_OK
    assert bwd(ct.byref(_rms(g, rows=0, x=None, dweight=None))) == g.GBMW_OK
    assert g._lib.gbmw_rms_norm_workspace(ct.byref(_rms(g, cols=0))) == -1
    assert g._lib.gbmw_rms_norm_workspace(ct.byref(_rms(g))) >= 64 * 4


def _rotary(g, **over):
    p = g.gbmw_rotary_problem()
    for i, n in enumerate(("freq", "positions", "len", "q", "k", "q_out", "k_out")):
        setattr(p, n, (i + 1) << 20)
    p.dtype, p.B, p.L, p.Hq, p.Hk, p.D, p.rot, p.factor, p.position_stride = g.GBMW_BF16, 2, 10, 4, 2, 64, 32, 1.0, 10
    for n, H in (("q", 4), ("k", 2), ("q_out", 4), ("k_out", 2)):
        setattr(p, n + "_stride", (ct.c_int64 * 3)(10 * H * 64, H * 64, 64))
    for n, x in over.items():
        setattr(p, n, (ct.c_int64 * 3)(*x) if n.endswith("_stride") and n != "position_stride" else x)
    return p


@no_device
def test_rotary_refuses():
    import paper_2307_02031_amd as g
    for call in (g._lib.gbmw_rotary_forward, g._lib.gbmw_rotary_backward):
        assert call(None) == g.GBMW_ERR_INVALID_ARG
        for over, word in [(dict(dtype=5), "dtype"), (dict(B=-1), "negative"), (dict(L=-1), "negative"), (dict(Hq=0), "Hq"), (dict(Hk=-1), "Hk"),
                           (dict(D=0), "D="), (dict(D=513), "D="), (dict(rot=31), "rot"), (dict(rot=66), "rot"), (dict(rot=-2), "rot"),
                           (dict(interleaved=2), "interleaved"), (dict(factor=math.nan), "factor"), (dict(factor=math.inf), "factor"),
                           (dict(B=1 << 16, L=1 << 16), "too many"), (dict(freq=None), "freq"), (dict(freq=4), "freq"), (dict(positions=2), "positions"),
                           (dict(position_stride=-1), "positions"), (dict(len=2), "len"), (dict(q=None), "q is null"), (dict(k=None), "k is null"),
                           (dict(q_out=None), "q_out is null"), (dict(k_out=3), "k_out is not aligned"), (dict(q_stride=(1, -1, 1)), "stride"),
                           (dict(q_out_stride=(2560, 256, 63)), "overlap"), (dict(q_out_stride=(0, 256, 64)), "overlap"),
                           (dict(k_out_stride=(1280, 64, 64)), "overlap"), (dict(q_out=4 << 20, q_out_stride=(3000, 256, 64)), "other strides"),
                           (dict(k_out=5 << 20, k_out_stride=(3000, 128, 64)), "other strides"), (dict(k_out=6 << 20), "one array")]:
            assert call(ct.byref(_rotary(g, **over))) == g.GBMW_ERR_INVALID_ARG, over
            assert word in g.gbmw_last_error(), (over, g.gbmw_last_error())
        assert call(ct.byref(_rotary(g, B=0, q=None, k=None))) == g.GBMW_OK


def test_frequencies():
    import paper_2307_02031_amd as g

    def freq(rot, theta=10000.0, scaling=0, by=1.0, original=0.0, slow=1.0, fast=32.0):
        out = np.full(max(0, rot // 2) + 1, 7.0)
        st = g._lib.gbmw_rotary_frequencies(rot, theta, scaling, by, original, slow, fast, out.ctypes.data)
        assert out[-1] == 7.0
        return st, out[:-1]

    i = np.arange(32)
    plain = 10000.0 ** (-2 * i / 64)
    near = lambda a, b: np.allclose(a, b, rtol=1e-14, atol=0)
    assert freq(64)[0] == g.GBMW_OK and near(freq(64)[1], plain) and freq(64)[1][0] == 1.0
    assert near(freq(64, scaling=1, by=4.0)[1], plain / 4)
    base = freq(64, scaling=2, by=4.0)[1]
    assert near(base, (10000.0 * 4.0 ** (64 / 62)) ** (-2 * i / 64)) and near(base[-1], plain[-1] / 4) and base[0] == 1.0
    ramp = freq(64, scaling=3, by=4.0, original=4096.0)[1]
    turns = 4096 * plain / (2 * np.pi)
    assert near(ramp[turns >= 32], plain[turns >= 32]) and near(ramp[turns <= 1], plain[turns <= 1] / 4)
    w = ((turns - 1) / 31)[(turns > 1) & (turns < 32)]
    assert len(w) > 3 and near(ramp[(turns > 1) & (turns < 32)], (plain * 0.25)[(turns > 1) & (turns < 32)] * (1 + 3 * w))
    assert freq(0)[0] == g.GBMW_OK
    for kw, word in [(dict(rot=3), "rot"), (dict(rot=514), "rot"), (dict(rot=-2), "rot"), (dict(rot=8, theta=0.0), "theta"),
                     (dict(rot=8, theta=math.inf), "theta"), (dict(rot=8, scaling=4), "scaling"), (dict(rot=8, scaling=1, by=0.0), "by"),
                     (dict(rot=2, scaling=2, by=2.0), "rot=2"), (dict(rot=8, scaling=3, by=2.0), "original"),
                     (dict(rot=8, scaling=3, by=2.0, original=10.0, slow=4.0, fast=4.0), "slow")]:
        assert freq(**kw)[0] == g.GBMW_ERR_INVALID_ARG and word in g.gbmw_last_error(), (kw, g.gbmw_last_error())
    assert g._lib.gbmw_rotary_frequencies(8, 1e4, 0, 1.0, 0.0, 1.0, 32.0, None) == g.GBMW_ERR_INVALID_ARG


@no_device
def test_adamw_refuses():
    import paper_2307_02031_amd as g
    make, h = g._lib.gbmw_adamw_list_create, ct.c_void_p(None)

    def status(bits=8, n=2, **over):
        t = (g.gbmw_adamw_tensor * 2)()
        for i, x in enumerate(t):
            x.numel, x.grad_dtype, x.dtype, x.copy_dtype = 1000, g.GBMW_BF16, g.GBMW_F32, g.GBMW_BF16
            for k, name in enumerate(("grad", "param", "copy", "m", "v", "m_scale", "v_scale")):
                setattr(x, name, (i * 8 + k + 1) << 20)
        for name, x in over.items():
            setattr(t[1], name, x)
        return make(n, t, bits, ct.byref(h))

    for kw, word in [(dict(n=-1), "n=-1"), (dict(bits=16), "state_bits"), (dict(numel=-1), "numel"), (dict(grad_dtype=3), "grad_dtype"),
                     (dict(dtype=9), "dtype"), (dict(dtype=g.GBMW_F16), "copy"), (dict(copy_dtype=g.GBMW_F32), "copy"),
                     (dict(weight_decay=-1.0), "weight_decay"), (dict(weight_decay=math.nan), "weight_decay"), (dict(grad=None), "grad of tensor 1 is null"),
                     (dict(param=None), "param of tensor 1 is null"), (dict(m=None), "m of tensor 1"), (dict(v_scale=None), "v_scale of tensor 1"),
                     (dict(grad=(9 << 20) + 1), "aligned"), (dict(param=(10 << 20) + 2), "aligned"), (dict(m_scale=(14 << 20) + 2), "aligned"),
                     (dict(param=2 << 20), "overlaps"), (dict(param=(2 << 20) + 3996), "overlaps"), (dict(m=12 << 20, v=(12 << 20) + 999), "overlaps"),
                     (dict(grad=10 << 20), "overlaps")]:
        assert status(**kw) == g.GBMW_ERR_INVALID_ARG and word in g.gbmw_last_error(), (kw, g.gbmw_last_error())
        assert h.value is None
    assert make(1, None, 8, ct.byref(h)) == g.GBMW_ERR_INVALID_ARG and make(0, None, 8, None) == g.GBMW_ERR_INVALID_ARG
    # what touches, or is read twice, does not overlap; without a device the list itself cannot be made
    assert status(param=(2 << 20) + 4000) in (g.GBMW_ERR_DEVICE, g.GBMW_ERR_OOM)
    assert status(grad=1 << 20) in (g.GBMW_ERR_DEVICE, g.GBMW_ERR_OOM)
    o = g.gbmw_adamw_options(1e-3, 0.9, 0.99, 1e-8, 1.0, 1.0, 1, 0)
    assert g._lib.gbmw_adamw_step(None, ct.byref(o), None) == g.GBMW_ERR_INVALID_ARG
    g._lib.gbmw_adamw_list_destroy(None)


@no_device
def test_the_binding_refuses_what_is_not_on_the_gpu():
    import paper_2307_02031_amd as g
    x = torch.zeros(2, 3, 4, 8, dtype=torch.bfloat16)
    f = torch.zeros(2, dtype=torch.float64)
    for call in (lambda: g.gbmw_rms_norm_forward(x), lambda: g.gbmw_rms_norm_backward(x, x, None, x), lambda: g.gbmw_rotary_forward(x, x, f),
                 lambda: g.gbmw_rotary_backward(None, x, f), lambda: g.gbmw_adamw_list_create([x], [x], [x], [x])):
        with pytest.raises(g.GbmwError) as e:
            call()
        assert e.value.status == g.GBMW_ERR_INVALID_ARG and "not a tensor on the GPU" in str(e.value)
    with pytest.raises(g.GbmwError):
        g.gbmw_rotary_frequencies(8, scaling="other")
