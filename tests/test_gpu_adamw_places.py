"""States in 8 bits of a list of more than 2^33 elements, which takes two launches: the last elements get what a short list of
theirs does, and random numbers are other ones beyond 2^32 elements, where the 32 bits of a place begin again."""
import pytest
import torch

from test_gpu_adamw_bits import F8, HOW, _codes, _hash

pytestmark = pytest.mark.gpu

SEED, STEP, LR = 99, 3, 1e-2


def _word(place):
    key = _hash((SEED + STEP * 0x9E3779B9) & 0xFFFFFFFF)
    high = place >> 32
    key = torch.where(high > 0, _hash((key + high * 0x9E3779B9) & 0xFFFFFFFF), key)
    return _hash((place & 0xFFFFFFFF) ^ key)


def test_places_beyond_32_bits_and_more_than_one_launch():
    import paper_2307_02031_amd as g
    first, n = 300, (1 << 33) + 1000       # the second tensor's places begin at 512: the middle of a run is at 2^32
    zeros = lambda k, dtype: torch.zeros(k, dtype=dtype, device="cuda")
    t = [dict(param=zeros(k, torch.bfloat16), grad=zeros(k, torch.bfloat16), m=zeros(k, torch.uint8).view(F8), v=zeros(k, torch.uint8).view(F8),
              m_scale=zeros(-(-k // 256), torch.float32), v_scale=zeros(-(-k // 256), torch.float32)) for k in (first, n)]
    big = t[1]
    windows = [slice(0, 1024), slice((1 << 32) - 2048, (1 << 32) + 2048), slice((1 << 33) - 1024, n)]
    # the same gradients in each: the places alone make the codes differ
    x = torch.randn(4096, generator=torch.Generator().manual_seed(1)).cuda().bfloat16()
    for w in windows:
        big["grad"][w] = x[:w.stop - w.start]
    make = lambda ts: g.gbmw_adamw_list_create(*([y[k] for y in ts] for k in ("param", "grad", "m", "v")),
                                               m_scales=[y["m_scale"] for y in ts], v_scales=[y["v_scale"] for y in ts])
    g.gbmw_adamw_step(make(t), LR, STEP, seed=SEED, **HOW)
    torch.cuda.synchronize()
    b1, b2 = HOW["beta1"], HOW["beta2"]
    got = []
    for w in windows:
        k = w.stop - w.start
        room = -(-k // 256) * 256
        grad = torch.nn.functional.pad(x[:k].float(), (0, room - k))
        word = _word(512 + w.start + torch.arange(room, device="cuda"))
        part = lambda z: (z.float() + 0.5) / 65536.0
        blocks = slice(w.start // 256, -(-w.stop // 256))
        for name, y, bits in (("m", grad * (1.0 - b1), word >> 16), ("v", torch.sqrt((grad * grad * (1.0 - b2)).double()).float(), word & 65535)):
            code, scale = _codes(y, part(bits), name == "v")
            assert torch.equal(big[name + "_scale"][blocks], scale), (name, w)
            assert torch.equal(big[name][w].view(torch.uint8), code[:k].view(torch.uint8)), (name, w)
        got.append(big["m"][w][:1024].view(torch.uint8))
        small = {a: zeros(k, y.dtype) if y.dtype != F8 else zeros(k, torch.uint8).view(F8) for a, y in big.items()}
        small.update(grad=x[:k].clone(), m_scale=zeros(room // 256, torch.float32), v_scale=zeros(room // 256, torch.float32))
        g.gbmw_adamw_step(make([small]), LR, STEP, **HOW)
        assert torch.equal(big["param"][w], small["param"]) and bool((small["param"] != 0).any())
    assert not torch.equal(got[0], got[2])
    # 0 between them
    for a, b in ((1024, 1 << 20), ((1 << 32) + 2048, (1 << 32) + (1 << 20))):
        assert bool((big["param"][a:b] == 0).all()) and bool((big["m"][a:b].view(torch.uint8) == 0).all())
    del t, big
    torch.cuda.empty_cache()
