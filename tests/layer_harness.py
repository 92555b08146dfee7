"""Inputs and tolerances of the tests of rotations, head norms and the gated feed-forward block.

As in ends_harness: U = 2^-24 is half a step of fp32 relative to the value, and a tolerance is the sum of the roundings that a formula allows."""
import numpy as np
import torch

from ends_harness import HALF, TYPES, U, f64, normal, within
from oracle import layer as L


def heads(rng, shape, dtype, layout, scale=1.0, fill=None):
    """[batch, heads, rows, head_dim] on the device: "dense"; "rows", parts of a projection's rows, with others beside them; "odd", one element off
    and rows one element apart; "wide", rows and heads four elements apart.  `fill`: value of everything."""
    b, h, n, d = shape
    if layout == "dense":
        out = torch.empty(shape, dtype=TYPES[dtype], device="cuda")
    elif layout == "rows":
        out = torch.full((b, n, h + 2, d), 777.0, dtype=TYPES[dtype], device="cuda")[:, :, 1:-1].transpose(1, 2)
    else:
        by = 1 if layout == "odd" else 4
        out = torch.full((b, h, n + 1, d + by), 777.0, dtype=TYPES[dtype], device="cuda")[:, :, 1:, by:]
    out.copy_(normal(rng, shape, dtype, scale)) if fill is None else out.fill_(fill)
    return out


def like(t, fill=float("nan")):
    """A tensor with the strides of t, its own memory filled."""
    size = 1 + sum((s - 1) * st for s, st in zip(t.shape, t.stride()))
    return torch.full((size,), fill, dtype=t.dtype, device="cuda").as_strided(t.shape, t.stride())


def pair_sizes(x, rotary, interleaved, magnitude):
    """For every element the magnitudes that its rotation adds: of both elements of its pair, or its own."""
    out = np.abs(x)
    first, second = L.pairs(rotary, interleaved)
    both = magnitude * (out[..., first] + out[..., second])
    out[..., first], out[..., second] = both, both
    return out


# cos and sin: the angle's rest in fp32 U, of at most 0.8; the series U each for its last addition and product, and what it leaves out, less than U; the product
# with the magnitude U: 5 U.  An element of a pair: two products and a sum more, 2 U each.
ROTATION = 8 * U
# a head's sum of squares: at most 16 squares in a lane, 6 additions over lanes: 24 U, half of that in its root; root, quotient and their products: 4 U
RSTD = 16 * U


def rounded(t, want, dtype):
    return t * (1 + HALF[dtype]) + HALF[dtype] * np.abs(want)


def check_forward(x, out, gain, eps, positions, freqs, magnitude, interleaved, dtype, what):
    x64, t = f64(x), ROTATION
    if gain is not None:
        x64, _ = L.head_norm(x64, f64(gain), eps)
        t += RSTD + 2 * U
    want = L.rotate(x64, positions, freqs, magnitude, interleaved)
    within(f64(out), want, rounded(t * pair_sizes(x64, 2 * len(freqs), interleaved, abs(magnitude)), want, dtype), what)


def check_backward(d, dx, x, gain, dgain, was, eps, positions, freqs, magnitude, interleaved, dtype, what):
    dy = L.rotate(f64(d), positions, freqs, magnitude, interleaved, back=True)
    size = pair_sizes(f64(d), 2 * len(freqs), interleaved, abs(magnitude))
    if gain is None:
        return within(f64(dx), dy, rounded(ROTATION * size, dy, dtype), what)
    x64, g64 = f64(x), f64(gain)
    want, wgain = L.head_norm_grad(dy, x64, g64, eps)
    _, rstd = L.head_norm(x64, g64, eps)
    xhat, g = np.abs(x64 * rstd), size * np.abs(g64)
    mean = lambda a: a.mean(-1, keepdims=True)
    # g: 9 U; xhat: 17 U; their products' mean: 24 U for its additions, 2 U; then a product, a difference and the product with rstd, 16 U and 3
    t = rstd * U * (32 * g + (9 + 17 + 26 + 17 + 16 + 4) * xhat * mean(g * xhat))
    within(f64(dx), want, rounded(t, want, dtype), what)
    n = x64.size // x64.shape[-1]
    start = f64(was)
    within(f64(dgain), start + wgain, (n + 40) * U * ((size * xhat).sum((0, 1, 2)) + np.abs(start)), what + " gain")


# ---- gated feed-forward block ----------------------------------------------------------------------------------------------------------

# What lies below the smallest fp32 and bf16 number that is not subnormal, 2^-126, may become 0: a sigmoid from an argument of -87.3 on, whose exponential passes the
# largest float at -88.8, and every product.
TINY = 2.0 ** -126


def act_errors(g, act):
    """Bounds for the errors of act(g) and act'(g) in fp32, from an exact g."""
    if act == "gelu":
        p = np.where(g == 0, 0.5, L.activation(g, act)[0] / np.where(g == 0, 1, g))
        pdf = np.exp(-g * g / 2) / np.sqrt(2 * np.pi)
        e_p = p * U * (16 + 4 * g * g) + TINY     # erfc to 8 units in its last place, of an argument that is 2 U off
        return np.abs(g) * e_p + 2 * U * np.abs(g * p), e_p + np.abs(g) * pdf * U * (8 + 2 * g * g) + 2 * U * (p + np.abs(g) * pdf)
    inside = np.ones_like(g) if act == "silu" else 2 * np.sqrt(2 / np.pi) * (1 + 0.134145 * g * g)
    arg = g if act == "silu" else 2 * np.sqrt(2 / np.pi) * g * (1 + 0.044715 * g * g)
    s = np.where(arg < 0, np.exp(-np.abs(arg)), 1) / (1 + np.exp(-np.abs(arg)))
    rest = s * (1 - s)
    # the sigmoid: its argument 6 U off, exponential and reciprocal 2 U each (2^-23)
    e_s = U * (6 * s + 7 * np.abs(arg) * rest) + TINY
    e_a = np.abs(g) * e_s + 2 * U * np.abs(g * s)
    return e_a, e_s + np.abs(g) * inside * (e_s * (1 - s) + s * (e_s + U)) + 8 * U * np.abs(g) * rest * inside + U * s


def ffn_forward_tolerances(x, w_in, w_out, act, dtype):
    """Bounds for y and [gate | up], from 64-bit operands."""
    k, f = (6 if dtype == "f32" else 1), len(w_in) // 2
    z = x @ w_in.T
    e_z = (k * x.shape[1] + 8) * U * (np.abs(x) @ np.abs(w_in).T)
    g, u = z[:, :f], z[:, f:]
    a, slope = L.activation(g, act)
    e_a = act_errors(g, act)[0] + 1.2 * e_z[:, :f]      # (no slope is above 1.13)
    h = a * u
    e_h = np.abs(u) * e_a + (np.abs(a) + e_a) * e_z[:, f:] + 2 * U * np.abs(h)
    e_h = e_h + (HALF["bf16"] if dtype == "bf16" else 2 * U) * (np.abs(h) + e_h)
    size = (np.abs(h) + e_h) @ np.abs(w_out).T
    return rounded(e_h @ np.abs(w_out).T + (k * f + 40) * U * size, h @ w_out.T, dtype), rounded(e_z, z, dtype)


def ffn_backward_tolerances(dy, x, w_in, w_out, act, gate_up, dtype):
    """Bounds for dx, dw_in and dw_out, sums alone."""
    k, f, half = (6 if dtype == "f32" else 1), len(w_in) // 2, HALF["bf16"] if dtype == "bf16" else 2 * U
    g, u = gate_up[:, :f], gate_up[:, f:]
    (a, slope), (e_a, e_slope) = L.activation(g, act), act_errors(g, act)
    dh, e_dh = np.abs(dy @ w_out), (k * dy.shape[1] + 8) * U * (np.abs(dy) @ np.abs(w_out))
    up = dh + e_dh
    e_dg = np.abs(u) * (e_dh * np.abs(slope) + up * e_slope) + 4 * U * up * np.abs(u * slope)
    e_du = e_dh * np.abs(a) + up * e_a + 2 * U * up * np.abs(a)
    dz = np.concatenate([dh * np.abs(u * slope), dh * np.abs(a)], 1)
    e_dz = np.concatenate([e_dg, e_du], 1)
    e_dz = e_dz + half * (dz + e_dz) + 4 * TINY
    dz = dz + e_dz
    h = np.abs(a * u)
    e_h = np.abs(u) * e_a + 2 * U * h
    e_h = e_h + half * (h + e_h) + 2 * TINY
    h = h + e_h
    n = len(x)
    ax, ay = np.abs(x), np.abs(dy)
    return (e_dz @ np.abs(w_in) + (k * 2 * f + 40) * U * (dz @ np.abs(w_in)), e_dz.T @ ax + (k * n + 40) * U * (dz.T @ ax),
            ay.T @ e_h + (k * n + 40) * U * (ay.T @ h))
