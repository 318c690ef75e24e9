"""What the layer operators refuse, through the C entry points and without a device: every check is made on the host
before anything is enqueued."""
import ctypes as ct
import math

import pytest
import torch

# the addresses here are made up: where a GPU could be asked to read them, they are not handed out
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="checks the host side, without a device")


def _attention(g, **over):
    p = g.gbmw_attention_problem()
    for n in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv", "workspace"):
        setattr(p, n, 1 << 20)
    p.dtype, p.B, p.Hq, p.Hk, p.Lq, p.Lk, p.D, p.scale = g.GBMW_BF16, 2, 4, 2, 10, 12, 64, 0.125
    for n, L, H in (("q", 10, 4), ("k", 12, 2), ("v", 12, 2), ("out", 10, 4), ("dout", 10, 4), ("dq", 10, 4), ("dk", 12, 2), ("dv", 12, 2)):
        setattr(p, n + "_stride", (ct.c_int64 * 3)(L * H * 64, H * 64, 64))
    p.workspace_bytes = 1 << 20
    for n, x in over.items():
        setattr(p, n, (ct.c_int64 * 3)(*x) if n.endswith("_stride") else x)
    return p


@pytest.mark.parametrize("over,word", [
    (dict(dtype=7), "dtype"), (dict(B=-1), "negative"), (dict(Lq=-1), "negative"), (dict(Lk=-5), "negative"),
    (dict(Hq=0), "Hq"), (dict(Hk=0), "Hk"), (dict(Hq=5), "multiple"), (dict(D=0), "D="), (dict(D=129), "D="),
    (dict(Lq=2 ** 31 - 1), "too many"), (dict(Lk=2 ** 31 - 1), "too many"), (dict(B=2 ** 31 - 1, Lq=10 ** 6), "too many"),
    (dict(causal=2), "causal"), (dict(scale=-1.0), "scale"), (dict(scale=math.nan), "scale"), (dict(scale=math.inf), "scale"),
    (dict(q=None), "q is null"), (dict(k=None), "k is null"), (dict(v=None), "v is null"), (dict(out=None), "out is null"),
    (dict(lse=None), "lse"), (dict(lse=2), "lse"), (dict(q=(1 << 20) + 1), "q is not aligned"),
    (dict(len_q=2), "len_q"), (dict(len_k=6), "len_k"), (dict(k_stride=(1, -1, 1)), "stride"),
    (dict(q_stride=(1 << 41, 1, 1)), "stride")])
def test_attention_refuses(over, word):
    import paper_2307_02031_amd as g
    for call in (g._lib.gbmw_attention_forward, g._lib.gbmw_attention_backward):
        assert call(ct.byref(_attention(g, **over))) == g.GBMW_ERR_INVALID_ARG
        assert word in g.gbmw_last_error(), g.gbmw_last_error()


def test_attention_refuses_what_only_one_pass_uses():
    import paper_2307_02031_amd as g
    fwd, bwd = g._lib.gbmw_attention_forward, g._lib.gbmw_attention_backward
    assert fwd(None) == g.GBMW_ERR_INVALID_ARG and bwd(None) == g.GBMW_ERR_INVALID_ARG
    assert fwd(ct.byref(_attention(g, dtype=g.GBMW_F32))) == g.GBMW_ERR_UNSUPPORTED
    assert fwd(ct.byref(_attention(g, out_stride=(10 * 256, 256, 32)))) == g.GBMW_ERR_INVALID_ARG
    assert "overlap" in g.gbmw_last_error()
    for over, word in [(dict(dout=None), "dout"), (dict(dq=None), "dq"), (dict(dk=None), "dk"), (dict(dv=None), "dv"),
                       (dict(dk_stride=(0, 128, 64)), "overlap"), (dict(workspace=None), "workspace"),
                       (dict(workspace_bytes=8), "workspace"), (dict(workspace=(1 << 20) + 8), "workspace")]:
        assert bwd(ct.byref(_attention(g, **over))) == g.GBMW_ERR_INVALID_ARG
        assert word in g.gbmw_last_error()
    assert g._lib.gbmw_attention_workspace(ct.byref(_attention(g, D=200)), 1) == -1
    assert g._lib.gbmw_attention_workspace(ct.byref(_attention(g)), 1) >= 4 * 2 * 4 * 10
    # nothing to do needs no arrays and no device
    assert fwd(ct.byref(_attention(g, B=0, q=None, k=None, v=None, out=None, lse=None))) == g.GBMW_OK
    assert bwd(ct.byref(_attention(g, B=0))) == g.GBMW_OK


def _norm(g, **over):
    p = g.gbmw_layer_norm_problem()
    for n in ("x", "weight", "bias", "y", "mean", "rstd", "dx", "dweight", "dbias", "workspace"):
        setattr(p, n, 1 << 20)
    p.dy, p.y, p.dx = 2 << 20, 3 << 20, 4 << 20
    p.dtype, p.wdtype, p.rows, p.cols, p.eps = g.GBMW_BF16, g.GBMW_F32, 10, 64, 1e-5
    p.x_stride = p.y_stride = p.dx_stride = p.dy_stride = 64
    p.workspace_bytes = 1 << 20
    for n, x in over.items():
        setattr(p, n, x)
    return p


def test_norm_refuses():
    import paper_2307_02031_amd as g
    fwd, bwd = g._lib.gbmw_layer_norm_forward, g._lib.gbmw_layer_norm_backward
    both = [(dict(dtype=3), "dtype"), (dict(wdtype=g.GBMW_F16), "wdtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"),
            (dict(cols=0), "cols"), (dict(cols=32769), "cols"), (dict(x=None), "x is null"), (dict(x=(1 << 20) + 1), "x is not aligned"),
            (dict(x_stride=-1), "x: row stride"), (dict(mean=None), "mean"), (dict(rstd=None), "rstd"), (dict(weight=(1 << 20) + 2), "weight")]
    only = {0: [(dict(eps=-1.0), "eps"), (dict(eps=math.nan), "eps"), (dict(y=None), "y is null"), (dict(y_stride=63), "y: row stride"),
                  (dict(bias=(1 << 20) + 2), "bias"), (dict(y=1 << 20, x_stride=65), "y is x")],
            1: [(dict(dy=None), "dy"), (dict(dx=None), "dx"), (dict(dx_stride=3), "dx: row stride"), (dict(workspace=None), "workspace"),
                  (dict(workspace_bytes=64), "workspace"), (dict(dweight=(1 << 20) + 2), "dweight"), (dict(dx=2 << 20, dx_stride=70), "dx is dy")]}
    for i, call in enumerate((fwd, bwd)):
        assert call(None) == g.GBMW_ERR_INVALID_ARG
        for over, word in both + only[i]:
            assert call(ct.byref(_norm(g, **over))) == g.GBMW_ERR_INVALID_ARG, over
            assert word in g.gbmw_last_error(), (over, g.gbmw_last_error())
    assert fwd(ct.byref(_norm(g, rows=0, x=None, y=None, mean=None, rstd=None))) == g.GBMW_OK
    assert g._lib.gbmw_layer_norm_workspace(ct.byref(_norm(g, cols=0))) == -1


def test_clip_refuses():
    import paper_2307_02031_amd as g
    make, h = g._lib.gbmw_gradient_list_create, ct.c_void_p(None)

    def status(n=1, ins=(1 << 20,), outs=(1 << 20,), numel=(5,), it=g.GBMW_F32, ot=g.GBMW_F32, null=()):
        a, b, c = (ct.c_void_p * 1)(*ins), (ct.c_void_p * 1)(*outs), (ct.c_int64 * 1)(*numel)
        t, o = (ct.c_int32 * 1)(it), (ct.c_int32 * 1)(ot)
        return make(n, None if "in" in null else a, None if "out" in null else b, None if "numel" in null else c,
                    None if "types" in null else t, o, ct.byref(h))

    for kw, word in [(dict(n=-1), "n=-1"), (dict(null=("in",)), "null"), (dict(null=("numel",)), "null"), (dict(null=("types",)), "null"), (dict(it=9), "in_dtype"),
                     (dict(ot=g.GBMW_F16), "out_dtype"), (dict(numel=(-1,)), "numel"), (dict(ins=(None,)), "null"),
                     (dict(ins=((1 << 20) + 2,)), "aligned"), (dict(it=g.GBMW_F16), "in place")]:
        assert status(**kw) == g.GBMW_ERR_INVALID_ARG and word in g.gbmw_last_error(), (kw, g.gbmw_last_error())
        assert h.value is None
    assert make(0, None, None, None, None, None, None) == g.GBMW_ERR_INVALID_ARG
    assert g._lib.gbmw_clip_gradients(None, 1.0, 1.0, None, None) == g.GBMW_ERR_INVALID_ARG
    g._lib.gbmw_gradient_list_destroy(None)


def test_the_binding_refuses_what_is_not_on_the_gpu():
    import paper_2307_02031_amd as g
    x = torch.zeros(2, 3, 4, 8, dtype=torch.bfloat16)
    for call in (lambda: g.gbmw_attention_forward(x, x, x), lambda: g.gbmw_layer_norm_forward(x),
                 lambda: g.gbmw_gradient_list_create([x]), lambda: g.gbmw_attention_forward(None, x, x)):
        with pytest.raises(g.GbmwError) as e:
            call()
        assert e.value.status == g.GBMW_ERR_INVALID_ARG and "not a tensor on the GPU" in str(e.value)
