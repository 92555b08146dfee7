"""Layer norm and its gradient against 64 bits, at the sizes, values and layouts where it can go wrong."""
import numpy as np
import pytest
import torch

import paper_2406_03488_amd as s1f
from ends_harness import HALF, U, TYPES, f64, normal, placed, row_values, space, untouched, within
from oracle import ends as E

pytestmark = pytest.mark.gpu

# batch, rows, hidden, layout of x, layout of y: every width of the kernels, whole and not
CASES = [(1, 1, 1, "dense", "dense"), (1, 1, 64, "dense", "dense"), (2, 3, 7, "odd", "view"), (1, 5, 512, "view", "dense"), (1, 9, 511, "dense", "odd"),
         (3, 4, 520, "seq", "dense"), (1, 700, 256, "dense", "dense"), (2, 341, 515, "view", "view"), (1, 6, 2048, "dense", "seq"),
         (1, 5, 2049, "odd", "dense"), (1, 4, 2563, "dense", "dense"), (1, 3, 4096, "odd", "odd"), (1, 1100, 2560, "dense", "dense"),
         (1, 2, 4104, "dense", "dense"), (2, 2, 8192, "dense", "view"), (1, 3, 8191, "dense", "dense"), (1, 3, 8200, "dense", "dense"),
         (1, 2, 9001, "odd", "dense"), (1, 3, 16384, "dense", "dense"), (1, 2, 16383, "dense", "dense")]


def calls(x, gamma, beta, eps, dy, layout_y, start):
    """Forward, then backward with what it has left."""
    b, n, h = x.shape
    y = placed(dy, layout_y, float("nan"))
    mean, rstd = row_values(b, n), row_values(b, n)
    s1f.layer_norm_fwd(x, gamma, beta, eps, y, mean, rstd)
    dyd = placed(dy, layout_y)
    dx = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda").fill_(float("nan"))
    dg, db = start[0].clone(), start[1].clone()
    size = s1f.layer_norm_bwd_workspace_bytes(dyd, x)
    ws, buffer = space(size)
    s1f.layer_norm_bwd(dyd, x, gamma, mean, rstd, dx, dg, db, ws)
    assert untouched(buffer, size)
    return y, mean, rstd, dyd, dx, dg, db


def check(x, gamma, beta, eps, dyd, got, start, dtype):
    y, mean, rstd, dx, dg, db = got
    n, h = x.shape[0] * x.shape[1], x.shape[2]
    flat = lambda t: f64(t).reshape(n, h)
    x64, g64, b64, dy64 = flat(x), f64(gamma), f64(beta), flat(dyd)
    wy, wm, wr = E.layer_norm(x64, g64, b64, eps)
    # a thread sums up to 32 elements, then 64 lanes and up to 16 waves: fewer than 56 additions in a row, and the division
    off = 56 * U * np.abs(x64).mean(1)
    relative = 40 * U + (off * wr) ** 2
    within(f64(mean).reshape(n), wm, off, "mean")
    within(f64(rstd).reshape(n), wr, relative * wr, "rstd")
    xhat = (x64 - wm[:, None]) * wr[:, None]
    t = np.abs(g64) * ((off * wr)[:, None] + np.abs(xhat) * (relative[:, None] + 6 * U)) + 2 * U * np.abs(wy)
    within(flat(y), wy, t * (1 + HALF[dtype]) + HALF[dtype] * np.abs(wy), "y")
    # the backward's statistics are the forward's, as they are
    m64, r64 = f64(mean).reshape(n), f64(rstd).reshape(n)
    wdx, wdg, wdb = E.layer_norm_grad(dy64, x64, g64, m64, r64)
    xhat, g = (x64 - m64[:, None]) * r64[:, None], np.abs(dy64 * g64)
    mean_of = lambda a: a.mean(1)[:, None]
    t = r64[:, None] * U * (8 * g + 64 * mean_of(g) + 72 * np.abs(xhat) * mean_of(g * np.abs(xhat)))
    within(flat(dx), wdx, t * (1 + HALF[dtype]) + HALF[dtype] * np.abs(wdx), "dx")
    was = f64(start[0]), f64(start[1])
    within(f64(dg), was[0] + wdg, (n + 8) * U * (np.abs(dy64 * xhat).sum(0) + np.abs(was[0])), "dgamma")
    within(f64(db), was[1] + wdb, (n + 8) * U * (np.abs(dy64).sum(0) + np.abs(was[1])), "dbeta")


def vectors(rng, h, dtype):
    return normal(rng, (h,), dtype, 0.3, 1.0).cuda(), normal(rng, (h,), dtype, 0.3).cuda(), (normal(rng, (h,), "f32").cuda(), normal(rng, (h,), "f32").cuda())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_forward_and_gradient(case, dtype):
    b, n, h, layout_x, layout_y = case
    rng = np.random.default_rng(n * h)
    x = placed(normal(rng, (b, n, h), dtype, 1.5, 0.4), layout_x)
    gamma, beta, start = vectors(rng, h, dtype)
    y, mean, rstd, dyd, dx, dg, db = calls(x, gamma, beta, 1e-5, normal(rng, (b, n, h), dtype), layout_y, start)
    check(x, gamma, beta, np.float64(np.float32(1e-5)), dyd, (y, mean, rstd, dx, dg, db), start, dtype)
    if layout_y == "view":
        assert (y._base[:, :n] == 777.0).all() and (y._base[:, 2 * n:] == 777.0).all()


def test_mean_far_from_zero():
    """The squares' sum minus the square of the sum would have no digit left."""
    rng = np.random.default_rng(5)
    x = placed(normal(rng, (1, 40, 768), "f32", 1.0, 3000.0), "dense")
    gamma, beta, start = vectors(rng, 768, "f32")
    y, mean, rstd, dyd, dx, dg, db = calls(x, gamma, beta, 0.0, normal(rng, (1, 40, 768), "f32"), "dense", start)
    check(x, gamma, beta, 0.0, dyd, (y, mean, rstd, dx, dg, db), start, "f32")


@pytest.mark.parametrize("h", [64, 4096])
def test_constant_rows(h):
    """No variance: the result is beta, rstd 1 / sqrt(eps)."""
    x = torch.full((1, 6, h), 0.5, device="cuda")
    gamma, beta = torch.full((h,), 2.0, device="cuda"), torch.full((h,), 0.25, device="cuda")
    y, mean, rstd = torch.empty_like(x), row_values(1, 6), row_values(1, 6)
    s1f.layer_norm_fwd(x, gamma, beta, 2.0 ** -16, y, mean, rstd)
    assert (y == 0.25).all() and (mean == 0.5).all() and (rstd == 256.0).all()


@pytest.mark.parametrize("h", [100, 1024, 5000])
def test_rows_that_are_not_finite_stay_alone(h):
    rng = np.random.default_rng(h)
    x = normal(rng, (1, 9, h), "f32").cuda()
    dy = normal(rng, (1, 9, h), "f32")
    gamma, beta, start = vectors(rng, h, "f32")
    clean = calls(x, gamma, beta, 1e-5, dy, "dense", start)
    bad = x.clone()
    bad[0, 2, h // 2], bad[0, 6, 0] = float("nan"), float("inf")
    got = calls(bad, gamma, beta, 1e-5, dy, "dense", start)
    keep = [0, 1, 3, 4, 5, 7, 8]
    assert torch.equal(got[0][0, keep], clean[0][0, keep]) and torch.equal(got[4][0, keep], clean[4][0, keep])
    assert torch.isnan(got[0][0, [2, 6]]).all()


def test_gradient_is_the_same_every_time():
    rng = np.random.default_rng(6)
    x = normal(rng, (2, 1500, 520), "bf16").cuda()
    dy = normal(rng, (2, 1500, 520), "bf16")
    gamma, beta, start = vectors(rng, 520, "bf16")
    runs = [calls(x, gamma, beta, 1e-5, dy, "dense", start) for _ in range(3)]
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


def test_offsets_past_32_bits():
    x = torch.zeros((2, 3, 1024), dtype=torch.bfloat16, device="cuda")
    big = torch.empty((2 ** 31 + 8192,), dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((2, 3, 1024), (2 ** 31, 2048, 1))
    rng = np.random.default_rng(11)
    x.copy_(normal(rng, (2, 3, 1024), "bf16"))
    far.copy_(x)
    gamma, beta, start = vectors(rng, 1024, "bf16")
    dy = normal(rng, (2, 3, 1024), "bf16")
    near = calls(x, gamma, beta, 1e-5, dy, "dense", start)
    y, mean, rstd = torch.empty_like(x), row_values(2, 3), row_values(2, 3)
    s1f.layer_norm_fwd(far, gamma, beta, 1e-5, y, mean, rstd)
    assert torch.equal(y, near[0])
    dg, db = start[0].clone(), start[1].clone()
    dyd = dy.cuda()
    ws = torch.empty(s1f.layer_norm_bwd_workspace_bytes(dyd, far), dtype=torch.uint8, device="cuda")
    out = torch.empty((2 ** 31 + 8192,), dtype=torch.bfloat16, device="cuda").as_strided((2, 3, 1024), (2 ** 31, 2048, 1))
    s1f.layer_norm_bwd(dyd, far, gamma, mean, rstd, out, dg, db, ws)
    assert torch.equal(out, near[4]) and torch.equal(dg, near[5])
