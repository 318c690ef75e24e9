"""Attention over many heads, dealt to the dies in every way there is, and head sizes between the others' steps."""
import pytest
import torch

from test_gpu_attention import _check, _inputs

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])


@TYPES
@pytest.mark.parametrize("B,Hq,Hk,D", [
    (11, 4, 4, 64),      # 44 heads: five a die, four of them at a time without a mask, and four heads that are left
    (83, 1, 1, 40),      # ten a die in lots of two; three are left
    (8, 8, 8, 80),       # eight a die in lots of four
    (6, 32, 16, 72),     # twelve a die in lots of four, heads that share
    (12, 8, 8, 32),      # twelve a die in lots of two
    (13, 8, 8, 128),     # thirteen a die, heads of whole lines
    (9, 5, 5, 17)])      # five a die and five that are left, rows that come through registers
def test_many_heads(B, Hq, Hk, D, dtype):
    """More than one tile of rows and of keys, samples of different lengths, rows without keys."""
    Lq, Lk = 150, 140
    q, k, v, dout = _inputs(B, Lq, Lk, Hq, Hk, D, dtype, seed=B * Hk)
    n = torch.arange(B, dtype=torch.int32, device="cuda")
    ragged = dict(len_q=Lq - 11 * n % 97, len_k=Lk - 17 * n % 131)
    _check(q, k, v, dout)
    _check(q, k, v, dout, causal=True)
    _check(q, k, v, dout, **ragged)
    _check(q, k, v, dout, causal=True, **ragged)


@TYPES
@pytest.mark.parametrize("D", [16, 24, 56, 88, 104, 112, 120])
def test_head_sizes_between(D, dtype):
    """Loaded straight to LDS, with pieces beyond the head's end."""
    _check(*_inputs(2, 70, 150, 4, 2, D, dtype, seed=D))
    _check(*_inputs(1, 130, 190, 2, 2, D, dtype, seed=D + 1), causal=True)
    _check(*_inputs(2, 3, 1500, 4, 2, D, dtype, seed=D + 2), causal=True)
