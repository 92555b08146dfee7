"""Gradients of the gains of heads, sums over all rows and heads, against bounds that one lost term exceeds: many units to a workgroup, many workgroups, many parts to join."""
import numpy as np
import pytest

import layer_spread as S
from ends_harness import f64
from oracle import layer as L
from test_gpu_rope import CASES, EPS, Call

pytestmark = pytest.mark.gpu

MANY = [(2, 2, 1, 100003, 8, 8, "rows", "dense"), (1, 3, 2, 150001, 24, 10, "dense", "dense"), (1, 40, 40, 2100, 16, 16, "dense", "dense"), (1, 64, 8, 4100, 128, 128, "rows", "dense"),
        (1, 8, 8, 9001, 80, 20, "dense", "dense"), (1, 4, 2, 30011, 6, 4, "dense", "dense"), (1, 5, 3, 7003, 254, 250, "odd", "dense"), (1, 2, 1, 20001, 256, 256, "dense", "dense")]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES + MANY)
def test_gains_gradients_hold_every_term(case, dtype, interleaved):
    c = Call(case, dtype, interleaved, True, listed=case[3] % 2 == 1)
    b, hq, hk, n, dim, rotary = case[:6]
    dq_rot, dka, _, _, _, _, was, dgains = c.backward()
    chain = S.gains_chain(b * n, hq, hk, dim, "odd" not in case[6:])
    for name, d, x, gain, start, got in (("q", dq_rot, c.q, c.gains[0], was[0], dgains[0]), ("k", c.rows(dka), c.k, c.gains[1], was[1], dgains[1])):
        d, x, start = f64(d), f64(x), f64(start)
        dy, rstd = L.rotate(d, c.at, c.freqs64, 1.0, interleaved, back=True), L.head_norm(x, 1.0, EPS)[1]
        want = start + (dy * x * rstd).sum((0, 1, 2))
        tolerance = S.gains_tolerance(d, x, rstd, rotary, interleaved, 1.0, chain, start)(want)
        off = np.abs(f64(got) - want)
        assert (off <= tolerance).all(), (name, off.max(), tolerance[off.argmax()], off.argmax())
