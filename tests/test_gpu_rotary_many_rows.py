"""More rows than a launch has waves for: a call makes several launches, and every row gets its own position."""
import pytest
import torch

pytestmark = pytest.mark.gpu

WAVES = (1 << 26) - 8      # of a launch


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "pairs"])
def test_a_second_launch(interleaved):
    import paper_2307_02031_amd as g
    H, L = 33, WAVES + 1000      # of 33 heads a wave has one token
    one = torch.randn(1, 1, H, 2, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    q = one.expand(1, L, H, 2)
    freq = torch.tensor([0.37], dtype=torch.float64, device="cuda")
    for call in (g.gbmw_rotary_forward, g.gbmw_rotary_backward):
        out = torch.zeros(1, L, H, 2, dtype=torch.bfloat16, device="cuda")      # 8.9 GB
        call(q, None, freq, interleaved=interleaved, q_out=out)
        for a, b in ((0, 100), (WAVES - 50, WAVES + 50), (L - 100, L)):
            positions = torch.arange(a, b, dtype=torch.int32, device="cuda")[None]
            assert torch.equal(out[:, a:b], call(q[:, a:b], None, freq, positions=positions, interleaved=interleaved)[0]), (a, b)
        del out
    torch.cuda.empty_cache()


def test_a_second_launch_of_waves_with_many_rows():
    """32 rows a wave, of which the last launch has few; values that are handed through, and lengths."""
    import paper_2307_02031_amd as g
    B, L = 4, (1 << 29) - 17     # 2^31 - 68 rows in all; a call takes up to 2^31 - 65
    one = torch.randn(B, 1, 2, 1, generator=torch.Generator().manual_seed(1)).half().cuda()
    out = torch.zeros(B, L, 2, 1, dtype=torch.float16, device="cuda")      # 8.6 GB
    n = torch.tensor([L, 10, L - 3, L - 7], dtype=torch.int32, device="cuda")
    g.gbmw_rotary_forward(one.expand(B, L, 2, 1), None, torch.zeros(0, dtype=torch.float64, device="cuda"), len_x=n, q_out=out)
    for b, m in enumerate(n.tolist()):
        for a, c in ((max(0, m - 500), m), (0, min(m, 500))):
            assert torch.equal(out[b, a:c], one[b].expand(c - a, 2, 1)), (b, a)
        assert bool((out[b, m:m + 500] == 0).all())
    del out
    torch.cuda.empty_cache()
