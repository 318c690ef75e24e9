"""Outputs of rotary positions over the other input, through the C entry points and without a device: heads that are still to be
read would be written."""
import ctypes as ct

import pytest
import torch

from test_more_refusals import _rotary


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the host side with made-up addresses, without a device")
@pytest.mark.parametrize("over,word", [(dict(q_out=5 << 20), "q_out is k"), (dict(k_out=4 << 20), "k_out is q"),
                                       (dict(k=4 << 20, q_out=4 << 20), "q_out is k"), (dict(q=5 << 20, k_out=5 << 20), "k_out is q")])
def test_an_output_over_the_other_input(over, word):
    import paper_2307_02031_amd as g
    for call in (g._lib.gbmw_rotary_forward, g._lib.gbmw_rotary_backward):
        assert call(ct.byref(_rotary(g, **over))) == g.GBMW_ERR_INVALID_ARG, over
        assert word in g.gbmw_last_error(), (over, g.gbmw_last_error())
        # without rows there is nothing to write
        assert call(ct.byref(_rotary(g, B=0, **over))) == g.GBMW_OK
