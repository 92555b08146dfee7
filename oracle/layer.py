"""What a layer computes around its attention, in 64 bits from its definition (numpy): rotation of queries and keys by their positions, norms of their
heads, the gated feed-forward block; with their gradients.

Heads are [batch, heads, rows, head_dim], positions [batch, rows]; the block's rows are flat, [n, hidden]."""
import math

import numpy as np


def frequencies(rotary_dim, base=10000.0):
    return np.array([base ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)])


def pairs(rotary_dim, interleaved):
    """Indexes of the first and the second element of every pair."""
    i = np.arange(rotary_dim // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary_dim // 2)


def rotate(x, positions, freqs, magnitude, interleaved, back=False):
    first, second = pairs(2 * len(freqs), interleaved)
    angle = positions.astype(np.float64)[:, None, :, None] * freqs
    turn = magnitude * np.exp((-1j if back else 1j) * angle)
    z = (x[..., first] + 1j * x[..., second]) * turn
    out = np.array(x, dtype=np.float64)
    out[..., first], out[..., second] = z.real, z.imag
    return out


def head_norm(x, gain, eps):
    """Normed heads, and one over their root mean squares."""
    rstd = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    return x * rstd * gain, rstd


def head_norm_grad(dy, x, gain, eps):
    """dx, dgain"""
    _, rstd = head_norm(x, gain, eps)
    xhat, g = x * rstd, dy * gain
    return rstd * (g - xhat * (g * xhat).mean(-1, keepdims=True)), (dy * xhat).sum((0, 1, 2))


_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def _sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x < 0, e, 1) / (1 + e)


def activation(g, act):
    """act(g) and its derivative; act: "silu", "gelu" or "gelu_tanh".  1 + erf(x) is erfc(-x), and (1 + tanh(x)) / 2 the sigmoid of 2x: with the
    former, gates far below 0 would lose all digits of 64 bits, too."""
    if act == "silu":
        s = _sigmoid(g)
        return g * s, s + g * s * (1 - s)
    if act == "gelu":
        p = _erfc(-g / math.sqrt(2)) / 2
        return g * p, p + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    k = 2 * math.sqrt(2 / math.pi)
    s = _sigmoid(k * (g + 0.044715 * g ** 3))
    return g * s, s + g * s * (1 - s) * k * (1 + 3 * 0.044715 * g * g)


def gated_ffn(x, w_in, w_out, act):
    """y, [gate | up], h"""
    z = x @ w_in.T
    f = len(w_in) // 2
    h = activation(z[:, :f], act)[0] * z[:, f:]
    return h @ w_out.T, z, h


def gated_ffn_grad(dy, x, w_in, w_out, act, gate_up):
    """dx, dw_in, dw_out, [dgate | dup], h"""
    f = len(w_in) // 2
    g, u = gate_up[:, :f], gate_up[:, f:]
    a, slope = activation(g, act)
    dh = dy @ w_out
    dz = np.concatenate([dh * u * slope, dh * a], 1)
    return dz @ w_in, dz.T @ x, dy.T @ (a * u), dz, a * u
