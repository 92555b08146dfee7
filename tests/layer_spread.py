"""How far the gated feed-forward block's results may be off as a whole, tile by tile, row by row and column by column: the bounds of layer_harness, sums of all roundings' largest sizes, hold for
every single element, and grow with the length of a sum so that a part of it could be missing.  Here roundings are counted as what they are in a sum of many, independent of one another.

A rounding to a step that is half of `half` relative to the value at most is off by half / sqrt 3 of it in the mean square at most (values at the low end of their power of two; 0.7 of that over all).
The mean square of an element's error is the sum V of those of the roundings that it is made of, each times the square of what it is multiplied with.  Over a block the sum of the squares of the errors e = M d, of operands'
errors d with a normal distribution and elements' own, has the mean tr(M M^T) (d of mean square 1), the sum of V over the block, and the variance 2 tr((M M^T)^2) = 2 sum of (m_k m_l)^2 over the columns of M, of which the
pairs of one column give w_k^2, w_k what error k adds to the mean, and the others, in directions that have nothing to do with one another, as much as independent elements would: the sum of V^2.  The root of the sum of squares is then
1 +- 4 / sqrt(N) times the expected one, but for one in 10^4, with N = (sum V)^2 / (sum V^2 + sum w^2).  (A row of dw_in of 65 tokens whose errors count like 5, one of them 40 % of the mean square, was 2.3 times the
expected one off: 1 + 4 / sqrt(5) = 2.8.)  What lies below 2^-126 plays no part in the inputs that these bounds are for.

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


def activation_spread(g, a, slope, act):
    """Mean squares of the errors of act(g) and act'(g) in fp32: an exponential and a reciprocal of 2 U each, or an error function of 8, of an argument that is 2 U |g| (1 + g^2 / 10) off, and eight roundings."""
    off = U * U / 3 * ((2 * g * (1 + g * g / 10)) ** 2 + 8 + (64 if act == "gelu" else 8))
    return off * a * a, off * (slope.abs() + 0.2) ** 2


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


def _blocks(t, rows, cols):
    """Sums over blocks of rows x cols; 0: all."""
    rows, cols = rows or t.shape[0], cols or t.shape[1]
    r, c = -(-t.shape[0] // rows), -(-t.shape[1] // cols)
    t = torch.nn.functional.pad(t, (0, c * cols - t.shape[1], 0, r * rows - t.shape[0]))
    return t.view(r, rows, c, cols).sum((1, 3))


def shared(v, q2):
    """Mean squares of the errors that p @ q has from p's, whose mean squares are v, and the sums of w^2 over the blocks that are looked at.  q2: squares of q."""
    def squares(rows, cols):
        q = _blocks(q2, 1, cols)
        return _blocks(v * v, rows, 1) @ (q * q)
    return v @ q2, squares


def forward(x, w_in, w_out, act, dtype):
    """{name: (value, mean square of its error, sums of w^2 or None)} from 64-bit operands."""
    f, half = len(w_in) // 2, HALF["bf16"] if dtype == "bf16" else 2 * U
    z, v_z = sums(x, w_in.T.contiguous(), dtype)
    g, u = z[:, :f], z[:, f:]
    a, slope = activation(g, act)
    v_a = activation_spread(g, a, slope, act)[0]
    h = a * u
    v_h = rounded((u * slope) ** 2 * v_z[:, :f] + a * a * v_z[:, f:] + u * u * v_a, h, 2 * U)
    v_h = rounded(v_h, h, half)
    y, v_y = sums(h, w_out.T.contiguous(), dtype)
    of_h, squares = shared(v_h, (w_out * w_out).T.contiguous())
    return {"gate_up": (z, rounded(v_z, z, HALF[dtype]), None), "y": (y, rounded(v_y + of_h, y, HALF[dtype]), squares)}


def backward(dy, x, w_in, w_out, act, gate_up, dtype, half_w):
    """The same of dx, dw_in, dw_out (the latter two rounded to steps of which half_w is half)."""
    f, half = len(w_in) // 2, HALF["bf16"] if dtype == "bf16" else 2 * U
    g, u = gate_up[:, :f], gate_up[:, f:]
    a, slope = activation(g, act)
    v_a, v_slope = activation_spread(g, a, slope, act)
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
        if v_p is not None:
            of, squares = shared(v_p.contiguous(), q * q)
        else:
            of, other = shared(v_q.T.contiguous(), (p * p).T.contiguous())
            of, squares = of.T, lambda rows, cols, other=other: other(cols, rows).T
        out[name] = (r, rounded(v + of, r, half_of), squares)
    return out


def near(got, expected, what, plus=None):
    """`got` against what forward or backward has for it: as a whole, in blocks of 32 x 32, rows and columns.  plus: what it was added to."""
    want, v, squares = expected
    if plus is not None:
        want = want + plus
        v = v + U * U / 3 * (want * want + 1)
    error = (got.double() - want) ** 2
    assert torch.isfinite(error).all(), f"{what}: not finite"
    v = v + _FEW
    for kind, rows, cols in (("all", 0, 0), ("block", 32, 32), ("row", 1, 0), ("column", 0, 1)):
        mean, square = _blocks(v, rows, cols), _blocks(v * v, rows, cols) + (squares(rows, cols) if squares else 0)
        ratio = (_blocks(error, rows, cols) / mean).sqrt() / (WHOLE * (1 + 4 * square.sqrt() / mean))
        worst = int(ratio.argmax())
        at = (worst // ratio.shape[1], worst % ratio.shape[1])
        assert ratio[at] <= 1, (f"{what}, {kind} {at}: {ratio[at].item():.3g} of what it may be off by, {_blocks(error, rows, cols)[at].sqrt().item():.3g} "
                                f"of {_blocks(want * want, rows, cols)[at].sqrt().item():.3g}")


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
