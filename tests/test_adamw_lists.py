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

