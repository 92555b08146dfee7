"""Token loss and its gradient against 64 bits, at the sizes, targets and layouts where it can go wrong."""
import numpy as np
import pytest
import torch

import paper_2406_03488_amd as s1f
from ends_harness import HALF, U, TYPES, f64, loss_tolerances, normal, placed, row_values, space, tokens_of, untouched, within
from oracle import ends as E

pytestmark = pytest.mark.gpu

# batch, rows, hidden, vocab, share of rows without a target, layout of x, row stride of the weight beyond hidden
CASES = [(1, 1, 8, 1, 0.0, "dense", 0), (1, 1, 64, 2, 0.0, "dense", 0), (1, 2, 1, 3, 0.0, "dense", 0), (2, 5, 64, 129, 0.3, "view", 0),
         (1, 63, 72, 255, 0.0, "dense", 0), (1, 64, 128, 256, 0.0, "dense", 0), (3, 43, 100, 257, 0.2, "odd", 0), (1, 130, 192, 511, 0.1, "seq", 8),
         (2, 128, 64, 300, 0.0, "dense", 0), (1, 257, 256, 513, 0.0, "dense", 5), (2, 150, 200, 777, 0.5, "view", 0), (1, 255, 320, 1030, 0.0, "seq", 0),
         (1, 300, 33, 1000, 0.9, "odd", 3), (1, 70, 1288, 700, 0.0, "dense", 0), (1, 400, 520, 2100, 0.05, "dense", 0), (1, 200, 64, 600, 1.0, "dense", 0)]


def make(rng, b, n, h, v, blank, layout, more, dtype, scale=2.0):
    x = placed(normal(rng, (b, n, h), dtype), layout)
    w = torch.full((v, h + more), 777.0, dtype=TYPES[dtype], device="cuda")[:, :h]
    w.copy_(normal(rng, (v, h), dtype, scale / np.sqrt(h)))
    return x, w, tokens_of(rng, b, n, v, blank, "dense" if layout == "dense" else "view")


def forward(x, w, targets):
    b, n, _ = x.shape
    loss, lse = row_values(b, n), row_values(b, n)
    size = s1f.token_loss_fwd_workspace_bytes(x, w)
    ws, buffer = space(size)
    s1f.token_loss_fwd(x, w, targets, loss, lse, ws)
    assert untouched(buffer, size)
    return loss, lse


def backward(dloss, x, w, targets, lse, dw):
    dx = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda").fill_(float("nan"))
    size = s1f.token_loss_bwd_workspace_bytes(x, w)
    ws, buffer = space(size)
    s1f.token_loss_bwd(dloss, x, w, targets, lse, dx, dw, ws)
    assert untouched(buffer, size)
    return dx


def check(x, w, targets, dtype, dw, rng):
    """Forward and backward of one call; dw: accumulators, or bf16 to be overwritten."""
    b, n, h = x.shape
    loss, lse = forward(x, w, targets)
    x64, w64, t = f64(x).reshape(-1, h), f64(w), targets.cpu().numpy().reshape(-1)
    want_loss, want_lse = E.token_loss(x64, w64, t)
    rows = np.nonzero(E.known(t, len(w)))[0]
    dloss = torch.from_numpy(rng.normal(size=(b, n)).astype(np.float32)).cuda() / max(1, len(rows))
    lse64, d64 = f64(lse).reshape(-1), f64(dloss).reshape(-1)
    e_loss, e_lse, _, _ = loss_tolerances(x64, w64, t, want_lse, d64, dtype, rows)
    within(f64(loss).reshape(-1), want_loss, e_loss, "loss")
    within(lse64, want_lse, e_lse, "lse")
    was = f64(dw) if dw.dtype == torch.float32 else 0.0
    dx = backward(dloss, x, w, targets, lse, dw)
    want_dx, want_dw, _, _ = E.token_loss_grad(d64, x64, w64, t, lse64)     # from the lse that the call was given
    _, _, e_dx, e_dw = loss_tolerances(x64, w64, t, lse64, d64, dtype, rows)
    within(f64(dx).reshape(-1, h), want_dx, e_dx * (1 + HALF[dtype]) + HALF[dtype] * np.abs(want_dx), "dx")
    half = U if dw.dtype == torch.float32 else HALF["bf16"]
    within(f64(dw), was + want_dw, e_dw * (1 + half) + half * np.abs(was + want_dw), "dweight")
    return dx


@pytest.mark.parametrize("kind", ["f32", "bf16", "bf16 written"])
@pytest.mark.parametrize("case", CASES)
def test_loss_and_gradient(case, kind):
    b, n, h, v, blank, layout, more = case
    dtype = kind.split()[0]
    rng = np.random.default_rng(n * h + v)
    x, w, targets = make(rng, b, n, h, v, blank, layout, more, dtype)
    into = torch.full((v, h + more), 777.0, dtype=torch.bfloat16 if kind.endswith("written") else torch.float32, device="cuda")
    dw = into[:, :h]
    dw.copy_(normal(rng, (v, h), "f32", 0.1)) if kind != "bf16 written" else dw.fill_(float("nan"))
    dx = check(x, w, targets, dtype, dw, rng)
    assert (into[:, h:] == 777.0).all()
    if layout == "view":
        assert x._base is not None and (f64(dx) == f64(dx)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(dtype):
    """Scores of +-60: exponentials that only a running maximum keeps finite."""
    rng = np.random.default_rng(21)
    x, w, targets = make(rng, 1, 140, 64, 900, 0.1, "dense", 0, dtype, scale=60.0)
    check(x, w, targets, dtype, torch.zeros((900, 64), device="cuda"), rng)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [20, 300])
def test_rows_without_a_target_take_no_part(n, dtype):
    """Whatever they hold: infinities and NaN in x, lse and dloss."""
    rng = np.random.default_rng(n)
    x, w, targets = make(rng, 1, n, 72, 333, 0.0, "dense", 0, dtype)
    out = torch.from_numpy(rng.random((1, n)) < 0.4).cuda()
    targets[out] = torch.where(torch.rand(int(out.sum()), device="cuda") < 0.5, -1, 333)
    x[out] = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda").to(x.dtype).repeat(24)
    loss, lse = forward(x, w, targets)
    assert (loss[out] == 0).all() and (lse[out] == 0).all() and torch.isfinite(loss).all()
    lse[out] = float("nan")
    dloss = torch.rand((1, n), device="cuda")
    dloss[out] = float("inf")
    dw = torch.zeros((333, 72), device="cuda")
    dx = backward(dloss, x, w, targets, lse, dw)
    assert (dx[out] == 0).all() and torch.isfinite(dx).all() and torch.isfinite(dw).all()
    keep = ~out[0]
    few = backward(dloss[:, keep].contiguous(), x[:, keep].contiguous(), w, targets[:, keep].contiguous(), lse[:, keep].contiguous(),
                   more := torch.zeros_like(dw))
    assert torch.equal(few, dx[:, keep]) and torch.equal(more, dw)


def test_a_row_that_is_not_finite_stays_alone():
    rng = np.random.default_rng(2)
    x, w, targets = make(rng, 1, 150, 64, 300, 0.0, "dense", 0, "bf16")
    clean = forward(x, w, targets)
    x[0, 70] = float("nan")
    loss, lse = forward(x, w, targets)
    keep = torch.arange(150, device="cuda") != 70
    assert torch.isnan(loss[0, 70]) and torch.equal(loss[0, keep], clean[0][0, keep]) and torch.equal(lse[0, keep], clean[1][0, keep])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_vocabulary_than_a_piece(dtype):
    """Vocabularies that are walked in several pieces, the last one short, checked on the device in 64 bits."""
    rng = np.random.default_rng(4)
    b, n, h, v = (1, 450, 64, 700001) if dtype == "f32" else (1, 1100, 64, 600011)
    x, w, targets = make(rng, b, n, h, v, 0.1, "dense", 0, dtype)
    targets[0, :3] = torch.tensor([v - 1, v - 2, v // 2], device="cuda")
    loss, lse = forward(x, w, targets)
    known = (targets[0] >= 0) & (targets[0] < v)
    z = x[0, known].double() @ w.double().T
    want = torch.logsumexp(z, 1)
    t = targets[0, known]
    # scores of 64 products: 72 (bf16) and 6 * 72 (fp32) additions, each of magnitudes below 64 * 6 * 1.3 in sum; 2^-21 for exponentials; sums of 5000 tiles
    bound = (6 if dtype == "f32" else 1) * 72 * U * 60 + 2.0 ** -21 + 5600 * U
    assert (lse[0, known].double() - want).abs().max() <= bound
    assert (loss[0, known].double() - (want - z.gather(1, t[:, None])[:, 0])).abs().max() <= 2 * bound
    dloss = torch.rand((b, n), device="cuda") / n
    dw = torch.zeros((v, h), device="cuda")
    dx = backward(dloss, x, w, targets, lse, dw)
    z.sub_(lse[0, known].double()[:, None]).exp_()
    z[torch.arange(len(t), device="cuda"), t] -= 1
    z *= dloss[0, known].double()[:, None]
    for got, w64 in ((dx[0, known], z @ w.double()), (dw, z.T @ x[0, known].double())):
        # relative to the result's own size: bf16 dz is off by at most 2^-8 of itself, sums of both by far less; fp32 by the bound on scores
        off = (got.double() - w64).norm() / w64.norm()
        assert off <= (2.0 ** -7 if dtype == "bf16" else 2 * bound), off
    assert not dx[0, ~known].any()


def test_row_stride_past_32_bits():
    v, h, stride = 700, 64, 2 ** 22 - 8
    rng = np.random.default_rng(13)
    x, w, targets = make(rng, 1, 150, h, v, 0.1, "dense", 0, "bf16")
    far = torch.empty((v * stride,), dtype=torch.bfloat16, device="cuda").as_strided((v, h), (stride, 1))
    far.copy_(w)
    near, wide = forward(x, w, targets), forward(x, far, targets)
    assert torch.equal(near[0], wide[0])
    dloss = torch.rand((1, 150), device="cuda")
    dw, dw_far = torch.zeros((v, h), device="cuda"), torch.empty((v * stride,), device="cuda").as_strided((v, h), (stride, 1)).zero_()
    a, b = backward(dloss, x, w, targets, near[1], dw), backward(dloss, x, far, targets, near[1], dw_far)
    assert torch.equal(a, b) and torch.equal(dw, dw_far)


def test_gradient_is_the_same_every_time():
    rng = np.random.default_rng(6)
    x, w, targets = make(rng, 2, 400, 264, 3001, 0.2, "dense", 0, "bf16")
    _, lse = forward(x, w, targets)
    dloss = torch.rand((2, 400), device="cuda")
    runs = []
    for _ in range(3):
        dw = torch.zeros((3001, 264), device="cuda")
        runs.append((backward(dloss, x, w, targets, lse, dw), dw))
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))


# Products of more tiles than a round of workgroups holds (tests/test_host_ends.py: these are cut as they are there for): rows, hidden, vocabulary
CUTS = [(1040, 512, 16384), (2304, 8192, 2304), (700, 128, 130), (130, 2000, 9000), (2048, 72, 300), (2049, 72, 300), (9000, 64, 257)]


def check_in_norm(n, h, v, blank, dtype):
    """Checked on the device in 64 bits, norm-wise: bf16 results and dz are off by at most 2^-8 of themselves each; fp32 ones by the roundings of sums of as many terms as
    the longest one has, which in the worst case is k U of the terms' magnitudes, sqrt(k) or so times the norm of the result."""
    rng = np.random.default_rng(n + v)
    x, w, targets = make(rng, 1, n, h, v, blank, "dense", 0, dtype)
    loss, lse = forward(x, w, targets)
    known = (targets[0] >= 0) & (targets[0] < v)
    x64, w64, t = x[0, known].double(), w.double(), targets[0, known]
    z = x64 @ w64.T
    want = torch.logsumexp(z, 1)
    size = (x64.abs() @ w64.abs().T).max().item()
    bound = (6 * h if dtype == "f32" else h) * U * size + 2.0 ** -20 + v * U
    assert (lse[0, known].double() - want).abs().max() <= bound
    assert (loss[0, known].double() - (want - z.gather(1, t[:, None])[:, 0])).abs().max() <= 2 * bound
    dloss = torch.rand((1, n), device="cuda") / n
    dw = torch.zeros((v, h), device="cuda")
    dx = backward(dloss, x, w, targets, lse, dw)
    z.sub_(lse[0, known].double()[:, None]).exp_()
    z[torch.arange(len(t), device="cuda"), t] -= 1
    z *= dloss[0, known].double()[:, None]
    for got, w_ in ((dx[0, known], z @ w64), (dw, z.T @ x64)):
        off = (got.double() - w_).norm() / w_.norm()
        assert off <= (2.0 ** -7 if dtype == "bf16" else 4 * bound), off
    assert not dx[0, ~known].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,h,v", CUTS)
def test_cut_products(n, h, v, dtype):
    check_in_norm(n, h, v, 0.1, dtype)


# dx in parts whose number follows the rows that count, the last one over two pieces of the vocabulary (tests/test_host_ends.py): rows, hidden, vocabulary
PARTS = [(700, 264, 9001), (1500, 72, 2000), (700, 264, 180000)]


@pytest.mark.parametrize("blank", [0.5, 0.8, 0.99])
@pytest.mark.parametrize("n,h,v", PARTS)
def test_parts_of_fewer_rows(n, h, v, blank):
    for dtype in ("f32",) if v > 9001 else ("f32", "bf16"):
        check_in_norm(n, h, v, blank, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("h,more", [(72, 8), (200, 56), (8, 8), (100, 5)])
def test_what_lies_between_rows_is_not_read(h, more, dtype):
    """NaN between the rows of x and of the weight: whole stages of a product would read them."""
    rng = np.random.default_rng(h)
    b, n, v = 2, 70, 300
    x = torch.full((b, n + 1, h + more), float("nan"), dtype=TYPES[dtype], device="cuda")[:, :n, :h]
    w = torch.full((v, h + more), float("nan"), dtype=TYPES[dtype], device="cuda")[:, :h]
    x.copy_(normal(rng, (b, n, h), dtype))
    w.copy_(normal(rng, (v, h), dtype, 2 / np.sqrt(h)))
    dw = torch.full((v, h + more), float("nan"), device="cuda")[:, :h]
    dw.zero_()
    check(x, w, tokens_of(rng, b, n, v, 0.1), dtype, dw, rng)
