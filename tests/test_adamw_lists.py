"""What a list's arguments may be, as far as that is seen without a device."""
import pytest
import torch


@pytest.mark.skipif(torch.cuda.is_available(), reason="shows that the library is reached by its failing without a device")
@pytest.mark.parametrize("how", [dict(), dict(m_scales=[], v_scales=[]), dict(m_scales={}.values(), v_scales={}.values(), weight_decay=[])])
def test_a_list_of_no_tensors(how):
    import paper_2307_02031_amd as g
    with pytest.raises(g.GbmwError) as e:
        g.gbmw_adamw_list_create([], [], [], [], **how)
    assert e.value.status in (g.GBMW_ERR_DEVICE, g.GBMW_ERR_OOM), e.value


def test_sizes_that_differ():
    import paper_2307_02031_amd as g
    for how, word in ((dict(weight_decay={1: 0.1}.values()), "1 weight_decay"), (dict(weight_decay=(x for x in (0.1, 0.2))), "2 weight_decay"),
                      (dict(m_scales=[torch.zeros(1)]), "1 m_scales")):
        with pytest.raises(g.GbmwError) as e:
            g.gbmw_adamw_list_create([], [], [], [], **how)
        assert e.value.status == g.GBMW_ERR_INVALID_ARG and word in str(e.value), e.value
