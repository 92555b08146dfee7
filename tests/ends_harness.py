"""Inputs, calls and tolerances of the tests of embedding, layer norm and token loss.

A tolerance is the sum of the roundings that the call's formula allows, element by element: U = 2^-24 is half a step of fp32, relative to the
value; sums of k fp32 terms in any order are off by at most (k - 1) U times the sum of their magnitudes (a little more, hence k); results are rounded
once to their type, off by half a step of it."""
import numpy as np
import torch

import paper_2406_03488_amd as s1f

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def f64(t):
    return t.detach().cpu().double().numpy()


def normal(rng, shape, dtype, scale=1.0, shift=0.0):
    return torch.from_numpy(rng.normal(shift, scale, shape).astype(np.float32)).to(TYPES[dtype])


def placed(t, layout, fill=None):
    """[batch, rows, hidden] on the device: "dense"; "view", rows in the middle of longer sequences; "odd", rows that start one element
    off and are one element apart; "seq", storage [rows, batch, hidden].  `fill`: value of everything, instead of t's."""
    b, n, h = t.shape
    if layout == "dense":
        out = torch.empty((b, n, h), dtype=t.dtype, device="cuda")
    elif layout == "view":
        out = torch.full((b, 2 * n + 3, h), 777.0, dtype=t.dtype, device="cuda")[:, n:2 * n]
    elif layout == "odd":
        out = torch.full((b, n + 1, h + 1), 777.0, dtype=t.dtype, device="cuda")[:, 1:, 1:]
    else:
        out = torch.full((n, b, h), 777.0, dtype=t.dtype, device="cuda").transpose(0, 1)
    out.copy_(t) if fill is None else out.fill_(fill)
    return out


def tokens_of(rng, batch, rows, vocab, blank, layout="dense"):
    """Low numbers often, high ones rarely; a share of `blank` of them is outside [0, vocab)."""
    t = np.minimum((np.exp(rng.random((batch, rows)) * np.log(vocab + 1)) - 1).astype(np.int64), vocab - 1)
    outside = rng.choice([-1, -100, vocab, vocab + 7, -2 ** 62, 2 ** 62, 2 ** 32], (batch, rows))
    t = torch.from_numpy(np.where(rng.random((batch, rows)) < blank, outside, t))
    if layout == "dense":
        return t.cuda()
    big = torch.zeros((batch, 2 * rows + 3), dtype=torch.int64, device="cuda")
    big[:, rows:2 * rows] = t.cuda()
    return big[:, rows:2 * rows]


def space(n, fill=0xFF):
    """A workspace whose bytes are NaN, and 256 bytes behind it that have to stay as they are."""
    buffer = torch.full((n + 256,), fill, dtype=torch.uint8, device="cuda")
    return buffer[:n], buffer


def untouched(buffer, n, fill=0xFF):
    return bool((buffer[n:] == fill).all())


def row_values(batch, rows):
    return torch.full((batch, rows), float("nan"), device="cuda")


def within(got, want, tolerance, what):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), f"{what}: not finite"
    over = np.abs(got - want) - tolerance
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, f"{what} at {at}: got {got[at]!r}, want {want[at]!r}, tolerance {np.broadcast_to(tolerance, over.shape)[at]!r}"


def loss_tolerances(x, w, targets, lse, dloss, dtype, rows):
    """Bounds for loss and lse [n], dx [n, h], dweight [v, h] from 64-bit operands.

    A score is a sum of h products (fp32 operands: six for each, what is left out at most 2^-24 of it): off by K U sum |x| |w|.
    lse: the largest score's error, its exponentials' (2^-22 each, v_exp_f32 and the product with log2 e on arguments that are off by
    2 U |z - most|), their sum's (over 16 columns of a lane, 4 lanes, 4 waves, then the vocabulary's tiles, rescaled: fewer than 64 + v / 128 terms) and the
    logarithm's.  dz: the exponential's error relative to it, U on the difference; rounded to the type of the rows (fp32: nothing, three planes hold it up to 2^-24)."""
    n, h = x.shape
    v = len(w)
    k = 8 + h * (6 if dtype == "f32" else 1)
    z = x[rows] @ w.T
    score = k * U * (np.abs(x[rows]) @ np.abs(w).T)
    most = z.max(1, initial=0.0)
    e_lse = np.zeros(n)
    spread = np.abs(z - lse[rows][:, None]) + np.abs(most - lse[rows])[:, None]
    p = np.exp(z - lse[rows][:, None])
    e_lse[rows] = (p * (score + 4 * U * spread)).sum(1) + score.max(1, initial=0.0) * 2 + (64 + v / 128) * U + 2.0 ** -21 + 4 * U * np.abs(lse[rows])
    e_loss = np.zeros(n)
    zt = np.take_along_axis(z, targets[rows][:, None], 1)[:, 0]
    e_loss[rows] = e_lse[rows] + np.take_along_axis(score, targets[rows][:, None], 1)[:, 0] + 2 * U * (np.abs(zt) + np.abs(lse[rows]))
    if dloss is None:
        return e_loss, e_lse
    g = np.abs(dloss[rows])[:, None]
    dz = np.exp(z - lse[rows][:, None])
    e_p = dz * (score + 4 * U * np.abs(z - lse[rows][:, None]) + 2.0 ** -21)
    dz[np.arange(len(rows)), targets[rows]] -= 1
    dz = np.abs(dz) * g
    half = HALF["bf16"] if dtype == "bf16" else 2 * U
    e_dz = (e_p + 2 * U) * g * (1 + half) + dz * (half + 2 * U)
    per = 6 if dtype == "f32" else 1
    e_dx = np.zeros((n, h))
    e_dx[rows] = e_dz @ np.abs(w) + (per * v + 24) * U * (dz @ np.abs(w))
    e_dw = e_dz.T @ np.abs(x[rows]) + (per * len(rows) + 8) * U * (dz.T @ np.abs(x[rows]))
    return e_loss, e_lse, e_dx, e_dw
