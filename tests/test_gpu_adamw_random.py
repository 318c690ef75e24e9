"""Second moments in 8 bits of gradients that have become 0, beside one that stays and keeps the block's scale: by a seed they
fall by their rate on average, to the nearest they stay where they are."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


@pytest.mark.parametrize("seed", [1, 0xFFFFFFFF, 0])
def test_second_moments_fall(seed):
    import paper_2307_02031_amd as g
    blocks, steps, beta2 = 2000, 300, 0.999
    n = blocks * 256
    grad = torch.full((n,), 0.5, device="cuda")
    grad[::256] = 1.0
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(F8) for _ in range(2))
    ms, vs, p = torch.zeros(blocks, device="cuda"), torch.zeros(blocks, device="cuda"), torch.zeros(n, device="cuda")
    lst = g.gbmw_adamw_list_create([p], [grad], [m], [v], m_scales=[ms], v_scales=[vs])
    root = lambda: (v.float() * vs.repeat_interleave(256)).double().view(blocks, 256)[:, 1:]
    g.gbmw_adamw_step(lst, 1e-4, 1, beta2=beta2, seed=seed)
    first = root()
    grad.copy_((torch.arange(n, device="cuda") % 256 == 0).float())
    for step in range(2, steps + 2):
        g.gbmw_adamw_step(lst, 1e-4, step, beta2=beta2, seed=seed)
    fell = float(root().mean() / first.mean())
    if seed == 0:
        assert fell > 0.98
        return
    # each step multiplies by sqrt(beta2) and rounds to one of two neighbours at most an eighth of the value apart, right on
    # average: 1 / 16 of it at most is a step's standard deviation, and values are independent
    expect, deviation = beta2 ** (steps / 2), (steps / 256 / (blocks * 255)) ** 0.5
    assert abs(fell - expect) < 6 * deviation, (fell, expect)
