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
