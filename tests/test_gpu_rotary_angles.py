"""Sines and cosines of rotary positions, read off the pairs (1, 0)."""
import numpy as np
import pytest
import torch

from paper_2006_09503_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", [1000, 1000000])
@pytest.mark.parametrize("inverse", [0, 1])
def test_sines_and_cosines_are_those_of_the_64_bit_angle(inverse, far):
    """A correctly rounded value is off by 1.5e-8 (root mean square over the circle); a function good to a unit and a last sum of about as much again:
    2.5e-8.  An angle that passed through 24 bits would make the sines 4e-8 by itself."""
    tokens, n = 4096, 32
    rng = np.random.default_rng(far)
    axis, freq = np.zeros(n, dtype=np.uint8), 1e4 ** (-np.arange(n) / n)
    pos = rng.integers(0, far, tokens).astype(np.int32)
    x = torch.zeros((tokens, 3 * 2 * n), device="cuda")
    x[:, :n] = 1.0
    P = torch.from_numpy(pos).cuda()
    B.check(B.lib().k2bw_rotary(0, 1, tokens, 1, 2 * n, n, 0, axis.ctypes.data, freq.ctypes.data, 1, P.data_ptr(), inverse, x.data_ptr(), None), "rotary")
    got = x[:, :2 * n].double().cpu().numpy()
    angle = pos[:, None].astype(np.float64) * freq
    turned = angle > 1.0         # (small angles have cosines near 1 and sines that are rounded to less)
    for v, want in ((got[:, :n], np.cos(angle)), (got[:, n:], np.sin(angle) * (-1.0 if inverse else 1.0))):
        off = (v - want)[turned]
        print(f"rms {np.sqrt((off * off).mean()):.3e}, largest {np.abs(off).max():.3e}")
        assert np.sqrt((off * off).mean()) < 2.5e-8 and np.abs(off).max() < 1.2e-7
