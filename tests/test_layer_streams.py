"""The stream that the layer operators' calls run on, whichever way it is given."""
import contextlib

import pytest
import torch


def test_handle_zero_is_the_default_stream(monkeypatch):
    """Without a device: which stream is made current for a handle."""
    import paper_2307_02031_amd as g
    seen = []
    monkeypatch.setattr(torch.cuda, "stream", lambda s: seen.append(s) or contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: "default")
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: handle)

    class Other:     # another library's stream
        cuda_stream = 0

    call = g._on_stream(lambda: len(seen))
    assert [call(), call(stream=0), call(stream=Other()), call(stream=77)] == [0, 1, 2, 3]
    assert seen == ["default", "default", 77]


@pytest.mark.gpu
def test_every_way_to_name_a_stream():
    import paper_2307_02031_amd as g
    side = torch.cuda.Stream()
    now = g._on_stream(lambda: torch.cuda.current_stream().cuda_stream)
    main = torch.cuda.default_stream()
    for given, want in ((0, 0), (main, 0), (torch.cuda.current_stream(), 0), (side, side.cuda_stream), (side.cuda_stream,) * 2):
        assert now(stream=given) == want
        with torch.cuda.stream(side):
            assert now(stream=given) == want and now() == side.cuda_stream
    x = torch.randn(300, 640, device="cuda").bfloat16()
    base = g.gbmw_layer_norm_forward(x)
    for given in (0, main):
        # on the caller's own stream a call's inputs need no waiting for
        big = torch.randn(4096, 4096, device="cuda")
        y = (x.float() + 0.0 * (big @ big).sum()).bfloat16()
        for a, b in zip(base, g.gbmw_layer_norm_forward(y, stream=given)):
            assert torch.equal(a, b)
