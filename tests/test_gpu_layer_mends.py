"""Calls around a layer's attention that gave wrong results, each against 64 bits."""
import numpy as np
import pytest
import torch

from test_gpu_rope import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_past_2_to_50(interleaved):
    """Angles whose quarter turns are too many to be counted in 64 bits to a fraction of one: what is left of them was up to 500, and results 10^18 times as large as their heads."""
    n = 48
    c = Call((1, 2, 1, n, 16, 16, "dense", "dense"), "f32", interleaved, False, True)
    at = np.array([[sign * ((1 << 46 + i // 3) + 12345 * i + 1) for i in range(n) for sign in (1, -1)][:n]], dtype=np.int64)
    assert at.max() > 1 << 52
    at[0, -4:] = (1 << 62) + 977, -(1 << 62) - 1, (1 << 63) - 1, -(1 << 63)
    freqs = np.array([1.0, 0.7, 3.0, 1e-3, 2.0 ** -10, 40.0, 2.0 ** 14, 1e-12])
    c.at, c.positions = at, torch.from_numpy(at).cuda()
    c.freqs64, c.freqs = freqs, torch.from_numpy(freqs).cuda()
    c.turn = (c.freqs, 1.0, interleaved, c.positions, c.off)
    c.check_forward(c.forward())
    c.check_backward(c.backward())
