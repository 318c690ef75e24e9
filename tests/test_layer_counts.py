"""Sizes that the library's 32-bit counts cannot hold are refused, not cut down to their lower bits."""
import pytest
import torch

BIG = (1 << 32) + 5


def test_workspace_of_a_size_beyond_32_bits():
    import paper_2307_02031_amd as g
    q, k = (torch.empty(1, 4, 2, 8, dtype=torch.bfloat16, device="meta") for _ in range(2))
    assert g.gbmw_attention_workspace(q, k, True) > 0
    for a, b in ((q, k[:, :1].expand(1, BIG, 2, 8)), (q[:, :1].expand(1, BIG, 2, 8), k), (q[:, :, :1].expand(1, 4, BIG, 8), k),
                 (q, k[:, :1].expand(1, 1 << 31, 2, 8))):
        with pytest.raises(g.GbmwError) as e:
            g.gbmw_attention_workspace(a, b, True)
        assert e.value.status == g.GBMW_ERR_INVALID_ARG


@pytest.mark.gpu
def test_calls_of_a_size_beyond_32_bits():
    """Views of one row many times over: nothing of that size is in memory, and nothing is launched."""
    import paper_2307_02031_amd as g
    x = torch.randn(1, 4, 2, 8, device="cuda").bfloat16()
    many = x[:, :1].expand(1, BIG, 2, 8)
    heads = x[:, :, :1].expand(1, 4, BIG, 8)
    samples = x.expand(BIG, 4, 2, 8)
    for q, k in ((x, many), (many, x), (heads, x), (samples, samples)):
        with pytest.raises(g.GbmwError) as e:
            g.gbmw_attention_forward(q, k, k)
        assert e.value.status == g.GBMW_ERR_INVALID_ARG and "size" in str(e.value)
    row = torch.randn(1, device="cuda").expand(3, BIG)
    with pytest.raises(g.GbmwError) as e:
        g.gbmw_layer_norm_forward(row)
    assert e.value.status == g.GBMW_ERR_INVALID_ARG
