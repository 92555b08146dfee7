"""Pins of oracle/layer.py: hand-worked values, torch's CPU fp64 functions with autograd, invariants of rotations."""
import math

import numpy as np
import torch

from oracle import layer as L


def test_rotations_by_hand():
    x = np.arange(1.0, 7.0).reshape(1, 1, 1, 6)
    quarter = np.array([math.pi / 2, 0.0])
    half = L.rotate(x, np.array([[1]]), quarter, 1.0, False)         # pairs (0, 2), (1, 3)
    assert np.allclose(half, [[[[-3, 2, 1, 4, 5, 6]]]], atol=1e-15)
    assert np.allclose(L.rotate(x, np.array([[1]]), quarter, 2.0, True), [[[[-4, 2, 6, 8, 5, 6]]]], atol=1e-14)
    assert np.allclose(L.rotate(half, np.array([[1]]), quarter, 1.0, False, back=True), x, atol=1e-15)
    assert L.frequencies(4, 100.0).tolist() == [1.0, 0.1]


def test_scores_depend_on_distances():
    rng = np.random.default_rng(1)
    q, k, f = rng.normal(size=(1, 1, 1, 16)), rng.normal(size=(1, 1, 1, 16)), L.frequencies(16)
    score = lambda p, r, inter: (L.rotate(q, np.array([[p]]), f, 1.0, inter) * L.rotate(k, np.array([[r]]), f, 1.0, inter)).sum()
    for inter in (False, True):
        assert abs(score(7, 3, inter) - score(1007, 1003, inter)) < 1e-11
        assert abs(score(0, 0, inter) - (q * k).sum()) < 1e-13


def test_against_autograd():
    rng = np.random.default_rng(2)
    x, gain, dy = rng.normal(size=(2, 3, 5, 8)), rng.normal(size=8), rng.normal(size=(2, 3, 5, 8))
    tx, tg = torch.tensor(x, requires_grad=True), torch.tensor(gain, requires_grad=True)
    y = torch.nn.functional.rms_norm(tx, (8,), tg, 1e-3)
    y.backward(torch.tensor(dy))
    assert np.allclose(L.head_norm(x, gain, 1e-3)[0], y.detach(), atol=1e-12)
    for a, b in zip(L.head_norm_grad(dy, x, gain, 1e-3), (tx.grad, tg.grad)):
        assert np.allclose(a, b, atol=1e-11)
    n, h, f = 6, 5, 7
    functions = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "gelu_tanh": lambda g: torch.nn.functional.gelu(g, approximate="tanh")}
    for act, function in functions.items():
        x, w_in, w_out, dy = (rng.normal(size=s) for s in ((n, h), (2 * f, h), (h, f), (n, h)))
        tx, ti, to = (torch.tensor(a, requires_grad=True) for a in (x, w_in, w_out))
        z = tx @ ti.T
        y = (function(z[:, :f]) * z[:, f:]) @ to.T
        y.backward(torch.tensor(dy))
        got, gate_up, hidden = L.gated_ffn(x, w_in, w_out, act)
        assert np.allclose(got, y.detach(), atol=1e-12)
        dx, di, do, dz, again = L.gated_ffn_grad(dy, x, w_in, w_out, act, gate_up)
        assert np.array_equal(again, hidden) and dz.shape == gate_up.shape
        for a, b in zip((dx, di, do), (tx.grad, ti.grad, to.grad)):
            assert np.allclose(a, b, atol=1e-11)
