"""The workspace that is asked for is the one that a call needs, under either mask."""
import ctypes as ct

import pytest
import torch

# (B, Lq, Lk, Hq, Hk, D): few tiles of rows over many keys, where a causal mask has them shared by more workgroups
SHAPES = [(2, 1600, 6171, 4, 4, 64), (8, 2048, 2048, 4, 4, 64), (1, 1, 5000, 8, 2, 128), (1, 2100, 130, 2, 1, 40), (2, 70, 150, 2, 2, 80),
          (1, 4, 4, 1, 1, 64)]


def _need(g, q, k, backward, causal):
    """What the C entry point says for the call's own problem."""
    p = g.gbmw_attention_problem()
    p.dtype, (p.B, p.Lq, p.Hq, p.D), (p.Lk, p.Hk) = g._DTYPE[q.dtype], q.shape, k.shape[1:3]
    p.causal, p.scale = int(causal), 0.125
    return g._lib.gbmw_attention_workspace(ct.byref(p), int(backward))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_workspace_of_either_mask(dtype):
    import paper_2307_02031_amd as g
    differ = 0
    for B, Lq, Lk, Hq, Hk, D in SHAPES:
        q, k = torch.empty(B, Lq, Hq, D, dtype=dtype, device="meta"), torch.empty(B, Lk, Hk, D, dtype=dtype, device="meta")
        for backward in (False, True):
            full, causal = (_need(g, q, k, backward, c) for c in (False, True))
            differ += full != causal
            assert g.gbmw_attention_workspace(q, k, backward) == max(full, causal)
            assert g.gbmw_attention_workspace(q, k, backward, causal=True) == causal
            assert g.gbmw_attention_workspace(q, k, backward, causal=False) == full
    assert differ > 2
    with pytest.raises(g.GbmwError):
        g.gbmw_attention_workspace(torch.empty(1, 2, 3, 129, dtype=dtype), torch.empty(1, 2, 3, 129, dtype=dtype), True)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_calls_with_just_the_bytes_that_were_asked_for(causal):
    """The same bits as with memory of the call's own, and nothing written behind the last byte."""
    import paper_2307_02031_amd as g
    gen = torch.Generator().manual_seed(1)
    for B, Lq, Lk, Hq, Hk, D in SHAPES:
        print("workspace", (B, Lq, Lk, Hq, Hk, D), causal, flush=True)
        q, dout = (torch.randn(B, Lq, Hq, D, generator=gen).bfloat16().cuda() for _ in range(2))
        k, v = (torch.randn(B, Lk, Hk, D, generator=gen).bfloat16().cuda() for _ in range(2))

        def bytes_of(n):
            whole = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
            return whole[:n], whole[n:]

        out, lse = g.gbmw_attention_forward(q, k, v, causal=causal)
        grads = g.gbmw_attention_backward(dout, q, k, v, out, lse, causal=causal)
        # of the default query, then of the call's own mask
        for which in (dict(), dict(causal=causal)):
            fwd, after_f = bytes_of(g.gbmw_attention_workspace(q, k, False, **which))
            bwd, after_b = bytes_of(g.gbmw_attention_workspace(q, k, True, **which))
            got = g.gbmw_attention_forward(q, k, v, causal=causal, workspace=fwd)
            assert torch.equal(got[0], out) and torch.equal(got[1], lse)
            for a, b in zip(grads, g.gbmw_attention_backward(dout, q, k, v, out, lse, causal=causal, workspace=bwd)):
                assert torch.equal(a, b)
            assert bool((after_f == 0x5a).all()) and bool((after_b == 0x5a).all())
        few = g.gbmw_attention_workspace(q, k, True, causal=causal) - 4
        with pytest.raises(g.GbmwError):
            g.gbmw_attention_backward(dout, q, k, v, out, lse, causal=causal, workspace=bytes_of(few)[0])
