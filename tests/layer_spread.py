"""How far the gated feed-forward block's results may be off as a whole, tile by tile, row by row and column by column: the bounds of layer_harness, sums of all roundings' largest sizes, hold for
every single element, and grow with the length of a sum so that a part of it could be missing.  Here roundings are counted as what they are in a sum of many, independent of one another.

A rounding to a step that is half of `half` relative to the value at most is off by half / sqrt 3 of it in the mean square at most (values at the low end of their power of two; 0.7 of that over all).
The mean square of an element's error is the sum of those of the roundings that it is made of, each times the square of what it is multiplied with; over N elements, the root of the
sum of squares is then 1 +- 4 / sqrt(N) times the expected one, but for one in 10^4, with N the elements or, if these are fewer, the terms of their sums, whose errors elements share.  What lies below 2^-126 plays no part
in the inputs that these bounds are for.

Sums of products in fp32, by matrix instructions of 32 terms, which round a running sum at most once for 8 of them; fp32 operands: six instructions instead of one.  A running sum's mean square is half of q, the sum of the terms' squares,
where they are of either sign, and a third of the result's square where they are of one: each rounding adds (q / 2 + S^2 / 3) U^2 / 3.  Sums of `most` terms at most, and the sums of these."""
import math

import torch

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
WHOLE = 1.3        # beside 1 + 4 / sqrt(N)
LONGEST = 12288    # terms of one fp32 sum
_FEW = 1e-300


def activation(g, act):
    """act(g), act'(g)"""
    if act == "gelu":
        p = torch.special.erfc(-g / math.sqrt(2)) / 2
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    k = 2 * math.sqrt(2 / math.pi)
    s = torch.sigmoid(g if act == "silu" else k * (g + 0.044715 * g ** 3))
    return g * s, s + g * s * (1 - s) * (1 if act == "silu" else k * (1 + 0.134145 * g * g))


def activation_spread(g, a, slope):
    """Mean squares of the errors of act(g) and act'(g) in fp32, relative to U: an exponential or error function of an argument that is 2 U |g| (1 + g^2 / 10) off, and eight roundings."""
    off = 2 * g.abs() * (1 + g * g / 10) + 8
    return (U * off) ** 2 * a * a, (U * off) ** 2 * (slope.abs() + 0.2) ** 2


def sums(a, b, dtype, most=LONGEST):
    """a @ b, and the mean square of its error in fp32."""
    k = a.shape[1]
    result, q = a @ b, (a * a) @ (b * b)
    if dtype == "f32" and k > most:
        turns = -(-k // most)
        roundings, one_sign = 6 * most / 8 + turns, 1 / turns
    else:
        roundings, one_sign = max(k / 8, 1) * (6 if dtype == "f32" else 1), 1.0
    # (what three planes of either operand leave out of a product: less than half of U)
    return result, U * U / 3 * (roundings * (q / 2 + one_sign * result * result / 3) + (q if dtype == "f32" else 0))


def rounded(v, value, half):
    return v + half * half / 3 * value * value


def forward(x, w_in, w_out, act, dtype):
    """{name: (value, mean square of its error, terms of its sums)} from 64-bit operands."""
    f, half = len(w_in) // 2, HALF["bf16"] if dtype == "bf16" else 2 * U
    z, v_z = sums(x, w_in.T.contiguous(), dtype)
    g, u = z[:, :f], z[:, f:]
    a, slope = activation(g, act)
    v_a = activation_spread(g, a, slope)[0]
    h = a * u
    v_h = rounded((u * slope) ** 2 * v_z[:, :f] + a * a * v_z[:, f:] + u * u * v_a, h, 2 * U)
    v_h = rounded(v_h, h, half)
    y, v_y = sums(h, w_out.T.contiguous(), dtype)
    v_y = rounded(v_y + v_h @ (w_out * w_out).T.contiguous(), y, HALF[dtype])
    return {"gate_up": (z, rounded(v_z, z, HALF[dtype]), x.shape[1]), "y": (y, v_y, f)}


def backward(dy, x, w_in, w_out, act, gate_up, dtype, half_w):
    """The same of dx, dw_in, dw_out (the latter two rounded to steps of which half_w is half)."""
    f, half = len(w_in) // 2, HALF["bf16"] if dtype == "bf16" else 2 * U
    g, u = gate_up[:, :f], gate_up[:, f:]
    a, slope = activation(g, act)
    v_a, v_slope = activation_spread(g, a, slope)
    dh, v_dh = sums(dy, w_out, dtype)
    dz = torch.cat([dh * u * slope, dh * a], 1)
    v_dz = torch.cat([(u * slope) ** 2 * v_dh + (dh * u) ** 2 * v_slope, a * a * v_dh + dh * dh * v_a], 1)
    v_dz = rounded(rounded(v_dz, dz, 2 * U), dz, half)
    h = a * u
    v_h = rounded(rounded(u * u * v_a, h, 2 * U), h, half)
    out = {}
    for name, (p, v_p, q, v_q, half_of) in {"dx": (dz, v_dz, w_in, None, HALF[dtype]), "dw_in": (dz.T.contiguous(), v_dz.T, x, None, half_w),
                                            "dw_out": (dy.T.contiguous(), None, h, v_h, half_w)}.items():
        r, v = sums(p, q, dtype)
        v = v + (v_p.contiguous() @ (q * q) if v_p is not None else (p * p) @ v_q)
        out[name] = (r, rounded(v, r, half_of), p.shape[1])
    return out


def _sum_blocks(t, side):
    rows, cols = (-(-s // side) for s in t.shape)
    t = torch.nn.functional.pad(t, (0, cols * side - t.shape[1], 0, rows * side - t.shape[0]))
    return t.view(rows, side, cols, side).sum((1, 3))


def near(got, expected, what, plus=None):
    """`got` against (value, mean square, terms) as a whole, in blocks of 32 x 32, rows and columns.  plus: (what was there, mean square of adding to it)."""
    want, v, terms = expected
    if plus is not None:
        want = want + plus
        v = v + U * U / 3 * (want * want + 1)
    error = (got.double() - want) ** 2
    assert torch.isfinite(error).all(), f"{what}: not finite"
    v, one = v + _FEW, torch.ones_like(want)
    kinds = {"all": lambda t: t.sum().view(1, 1), "block": lambda t: _sum_blocks(t, 32), "row": lambda t: t.sum(1, keepdim=True), "column": lambda t: t.sum(0, keepdim=True)}
    for kind, of in kinds.items():
        ratio = (of(error) / of(v)).sqrt() / (WHOLE * (1 + 4 / of(one).clamp(max=float(terms)).sqrt()))
        worst = int(ratio.argmax())
        at = (worst // ratio.shape[1], worst % ratio.shape[1])
        assert ratio[at] <= 1, f"{what}, {kind} {at}: {ratio[at].item():.3g} of what it may be off by, {of(error)[at].sqrt().item():.3g} of {of(want * want)[at].sqrt().item():.3g}"


def gains_tolerance(d, x, rstd, rotary, interleaved, magnitude, chain, start):
    """For every element of a gain: how far the sum over all rows and heads of dy * x * rstd, added to `start`, may be off.  d, x: [.., head_dim] gradients before they are turned back, and heads, rstd [.., 1], in numpy.

    A term is off by 26 U of the magnitudes that make it (layer_harness: rotation 8, rstd 16, products 2), one independent of the next, but for what all have in common: as much of the sum itself, and of what a sum of
    terms of either sign comes to.  Its additions: `chain` of them one behind the other, of running sums whose squares are at most those of all terms, and the result's.  Six times the root of the mean square."""
    import numpy as np
    from layer_harness import pair_sizes
    terms = pair_sizes(d, rotary, interleaved, abs(magnitude)) * np.abs(x * rstd)
    q = (terms ** 2).sum(tuple(range(d.ndim - 1)))

    def of(result):
        s2 = (np.abs(result) + np.abs(start)) ** 2
        return 6 * U * np.sqrt(26 ** 2 / 3 * q + chain / 3 * (q + s2)) + 26 * U * (np.abs(result - start) + 3 * np.sqrt(q)) + U * np.abs(result)
    return of


def gains_chain(rows, hq, hk, dim, aligned):
    """Additions one behind the other in a gain's gradient: three a unit of the workgroup's share, of which there are at least 256; the workgroup's groups of lanes; 2048 parts by 64 shares, and these."""
    items = dim // 8 if dim % 8 == 0 and aligned else dim // 2
    lanes = min(32, max(8, 1 << ((items if dim % 8 == 0 and aligned else -(-items // 4)) - 1).bit_length()))
    groups = 256 // lanes
    in_block = min(groups, 1 << (rows - 1).bit_length())
    units = -(-rows // in_block) * (hq + 2 * hk)
    return 3 * -(-units // 256) + groups + 32 + 64 + 1
