"""Rows that see no key have results of 0 and give no gradient, whatever they hold and whatever the keys hold that other
rows see."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
NAN, INF = float("nan"), float("inf")


def _inputs(B, Lq, Lk, Hq, Hk, D, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=gen).to(dtype).cuda()
    return new(B, Lq, Hq, D), new(B, Lk, Hk, D), new(B, Lk, Hk, D), new(B, Lq, Hq, D)


def _run(q, k, v, dout, **mask):
    import paper_2307_02031_amd as g
    print("empty rows", tuple(q.shape), tuple(k.shape), q.dtype, mask.get("causal"), flush=True)
    out, lse = g.gbmw_attention_forward(q, k, v, **mask)
    dq, dk, dv = g.gbmw_attention_backward(dout, q, k, v, out, lse, **mask)
    torch.cuda.synchronize()
    return out, lse, dq, dk, dv


# one workgroup of rows, rows of few tokens, shared keys, sizes that are loaded through registers, few rows and keys
SHAPES = [(2, 70, 150, 2, 2, 64), (2, 3, 90, 8, 2, 128), (2, 5, 4000, 4, 2, 80), (2, 40, 3000, 1, 1, 64), (2, 70, 150, 3, 1, 17), (2, 20, 1700, 1, 1, 100),
          (2, 6, 9, 2, 2, 64)]


@TYPES
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("B,Lq,Lk,Hq,Hk,D", SHAPES)
def test_rows_beyond_a_length_next_to_rows_of_nan(B, Lq, Lk, Hq, Hk, D, causal, dtype):
    """A NaN key and an infinite value reach the sample's own rows, not the padding behind them."""
    q, k, v, dout = _inputs(B, Lq, Lk, Hq, Hk, D, dtype, seed=Lq + Lk)
    nq = torch.tensor([Lq - 2, 0], dtype=torch.int32, device="cuda")
    for what, bad in ((k, NAN), (v, INF), (v, NAN)):
        old = what.clone()
        what[:, 0] = bad
        out, lse, dq, _, _ = _run(q, k, v, dout, causal=causal, len_q=nq)
        for b, n in enumerate(nq.tolist()):
            assert bool((out[b, n:] == 0).all()) and bool((dq[b, n:] == 0).all()) and bool(torch.isneginf(lse[b, :, n:]).all())
        assert not bool(torch.isfinite(out[0, Lq - 3]).any())      # the last row sees key 0 under either mask
        what.copy_(old)


@TYPES
@pytest.mark.parametrize("Lq,Lk,Hq,Hk,D", [(130, 70, 2, 2, 64), (300, 20, 2, 1, 80), (33, 5, 3, 3, 128), (70, 69, 6, 2, 40), (200, 131, 2, 2, 17),
                                           (2300, 200, 1, 1, 64), (12, 5, 2, 2, 64)])
def test_first_rows_of_a_causal_mask_that_see_nothing(Lq, Lk, Hq, Hk, D, dtype):
    """More queries than keys: the first rows' queries and gradients may be anything, and count for nothing."""
    q, k, v, dout = _inputs(1, Lq, Lk, Hq, Hk, D, dtype, seed=Lq)
    n = Lq - Lk
    q[:, :n], dout[:, :n] = 0, 0
    base = _run(q, k, v, dout, causal=True)
    assert all(bool(torch.isfinite(t).all()) for t in (base[0], *base[2:]))
    for bad in (NAN, INF, 6e4):      # 6e4: a float16 that would take all digits of a common factor
        q[:, :n], dout[:, :n] = bad, bad
        got = _run(q, k, v, dout, causal=True)
        assert bool((got[0][:, :n] == 0).all()) and bool((got[2][:, :n] == 0).all()) and bool(torch.isneginf(got[1][:, :, :n]).all())
        for a, b in zip(base, got):
            assert torch.equal(a, b)
    # nor do the keys' own values reach them
    v[:] = NAN
    out, lse, dq, _, _ = _run(q, k, v, dout, causal=True)
    assert bool((out[:, :n] == 0).all()) and bool((dq[:, :n] == 0).all()) and bool(torch.isneginf(lse[:, :, :n]).all())
