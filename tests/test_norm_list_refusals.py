"""A gradient list without outputs, through the C entry point and without a device."""
import ctypes as ct

import pytest
import torch


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the host side with made-up addresses, without a device")
def test_a_list_without_outputs():
    import paper_2307_02031_amd as g
    h = ct.c_void_p(None)
    one = lambda kind, x: (kind * 1)(x)

    def status(at=1 << 20, numel=5, dtype=g.GBMW_F16, out=None, out_dtype=None):
        return g._lib.gbmw_gradient_list_create(1, one(ct.c_void_p, at), out, one(ct.c_int64, numel), one(ct.c_int32, dtype), out_dtype,
                                                ct.byref(h))

    # without a device the list itself cannot be made
    assert status() in (g.GBMW_ERR_DEVICE, g.GBMW_ERR_OOM)
    assert status(out_dtype=one(ct.c_int32, 9)) in (g.GBMW_ERR_DEVICE, g.GBMW_ERR_OOM)      # not looked at
    for kw, word in [(dict(at=None), "null"), (dict(at=(1 << 20) + 1), "aligned"), (dict(dtype=9), "in_dtype"), (dict(numel=-1), "numel"),
                     (dict(out=one(ct.c_void_p, 1 << 20)), "null array")]:
        assert status(**kw) == g.GBMW_ERR_INVALID_ARG and word in g.gbmw_last_error(), (kw, g.gbmw_last_error())
        assert h.value is None
