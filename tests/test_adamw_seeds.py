"""Seeds that do not fit 32 bits are refused, not cut: their lower bits may be 0, which rounds to the nearest."""
import pytest


@pytest.mark.parametrize("seed", [1 << 32, -1, 3 << 32, (1 << 32) + 5, -(1 << 32)])
def test_refused(seed):
    import paper_2307_02031_amd as g
    with pytest.raises(g.GbmwError) as e:
        g.gbmw_adamw_step(g.AdamWList(), 1e-3, 1, seed=seed)
    assert e.value.status == g.GBMW_ERR_INVALID_ARG and "seed" in str(e.value)
