"""Angles next to whole quarter turns, whose sine or cosine is small.  What an angle is off a quarter turn is taken in 64 bits
and rounded to 32 once; the series and the factor add a few roundings of 2^-24 relative: each result is off by at most 2^-21 of
itself, and by the angle's own error in 64 bits, 2^-51 of it (the frequency over 2 pi, and the product with the position)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "pairs"])
@pytest.mark.parametrize("position", [1, 3, 1000, -77])
def test_next_to_quarter_turns(position, interleaved):
    import paper_2307_02031_amd as g
    quarters, off = np.meshgrid(np.arange(0, 8), np.concatenate([s * 10.0 ** np.arange(-7, 0, 1.0) * 3 for s in (1, -1)]))
    freq = ((quarters * (np.pi / 2) + off) / position).ravel()
    n = len(freq)
    x = torch.zeros(1, 1, 1, 2 * n, device="cuda")
    x[..., slice(0, 2 * n, 2) if interleaved else slice(0, n)] = 1.0
    pos = torch.tensor([[position]], dtype=torch.int32, device="cuda")
    angle = np.longdouble(position) * freq.astype(np.longdouble)
    for call, sign in ((g.gbmw_rotary_forward, 1.0), (g.gbmw_rotary_backward, -1.0)):
        got = call(x, None, torch.from_numpy(freq).cuda(), positions=pos, interleaved=interleaved, factor=1.25)[0].cpu().double().view(-1).numpy()
        c, s = (got[0::2], got[1::2]) if interleaved else (got[:n], got[n:])
        for name, y, want in (("cos", c, np.cos(angle) * 1.25), ("sin", s, np.sin(angle) * 1.25 * sign)):
            bound = 2.0 ** -21 * np.abs(want) + 1.25 * 2.0 ** -51 * np.abs(angle)
            worst = np.argmax(np.abs(y - want) / bound)
            assert (np.abs(y - want) <= bound).all(), (name, float(angle[worst]), float(want[worst]), float(y[worst]))
