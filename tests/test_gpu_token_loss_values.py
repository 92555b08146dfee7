"""Token loss and its gradient where scores or operands lie at the edges of their types: masked tokens, whose score is the type's lowest value or near it."""
import numpy as np
import pytest
import torch

import paper_2406_03488_amd as s1f
from ends_harness import HALF, U, TYPES, f64, loss_tolerances, normal, row_values, space, untouched, within
from oracle import ends as E

LOWEST = torch.finfo(torch.float32).min
pytestmark = pytest.mark.gpu


def forward(x, w, targets):
    loss, lse = row_values(*x.shape[:2]), row_values(*x.shape[:2])
    size = s1f.token_loss_fwd_workspace_bytes(x, w)
    ws, buffer = space(size)
    s1f.token_loss_fwd(x, w, targets, loss, lse, ws)
    assert untouched(buffer, size)
    return loss, lse


def backward(dloss, x, w, targets, lse):
    dx, dw = torch.full_like(x, float("nan")), torch.zeros(w.shape, device="cuda")
    size = s1f.token_loss_bwd_workspace_bytes(x, w)
    ws, buffer = space(size)
    s1f.token_loss_bwd(dloss, x, w, targets, lse, dx, dw, ws)
    assert untouched(buffer, size)
    return dx, dw


# n, hidden, vocab, masked tokens: a whole tile of every size and a ragged end; the last few, behind which a tile is empty; all but one
MASKED = [(70, 64, 1030, [(256, 640), (1024, 1030)]), (300, 136, 2055, [(0, 512), (2048, 2055)]), (1040, 64, 16384, [(128, 16384)]), (5, 72, 300, [(0, 299)])]
# type, the last element of every row, that of masked tokens: scores of -3.39e38, of -2.55e38 out of moderate operands
MASKS = [("bf16", 1.0, torch.finfo(torch.bfloat16).min), ("bf16", 2.0 ** 60, -1.5 * 2.0 ** 67), ("f32", 2.0 ** 60, -1.5 * 2.0 ** 67)]


def masked_call(rng, n, h, v, spans, dtype, element, mask):
    """x, weight, the numbers of the tokens that are not masked; what is masked scores element * mask."""
    x, w = normal(rng, (1, n, h), dtype), normal(rng, (v, h), dtype, 2 / np.sqrt(h))
    x[..., -1] = element
    w[:, -1] = 0.0
    on = np.ones(v, dtype=bool)
    for i, j in spans:
        on[i:j] = False
        w[i:j], w[i:j, -1] = 0.0, mask
    return x.cuda(), w.cuda(), np.nonzero(on)[0]


def check_against_the_others(x, w, on, dtype, rng):
    """Masked tokens have weight zero: all is as over the vocabulary without them, and their gradients are zero."""
    n, h = x.shape[1:]
    at = rng.integers(0, len(on), n)
    targets = torch.from_numpy(on[at])[None].cuda()
    x64, w64, g = f64(x)[0], f64(w)[on], (rng.random(n) + 0.5).astype(np.float32)
    loss, lse = forward(x, w, targets)
    want_loss, want_lse = E.token_loss(x64, w64, at)
    e_loss, e_lse = loss_tolerances(x64, w64, at, want_lse, None, dtype, np.arange(n))
    within(f64(lse)[0], want_lse, e_lse, "lse")
    within(f64(loss)[0], want_loss, e_loss, "loss")
    dx, dw = backward(torch.from_numpy(g)[None].cuda(), x, w, targets, lse)
    lse64 = f64(lse)[0]
    want_dx, want_dw, _, _ = E.token_loss_grad(g.astype(np.float64), x64, w64, at, lse64)
    _, _, e_dx, e_dw = loss_tolerances(x64, w64, at, lse64, g.astype(np.float64), dtype, np.arange(n))
    within(f64(dx)[0], want_dx, e_dx * (1 + HALF[dtype]) + HALF[dtype] * np.abs(want_dx), "dx")
    got = f64(dw)
    within(got[on], want_dw, e_dw * (1 + U) + U * np.abs(want_dw), "dweight")
    got[on] = 0
    assert not got.any()


@pytest.mark.parametrize("dtype,element,mask", MASKS)
@pytest.mark.parametrize("case", MASKED)
def test_masked_tokens(case, dtype, element, mask):
    n, h, v, spans = case
    rng = np.random.default_rng(n + v)
    x, w, on = masked_call(rng, n, h, v, spans, dtype, element, mask)
    check_against_the_others(x, w, on, dtype, rng)


@pytest.mark.parametrize("dtype,element,mask", MASKS)
@pytest.mark.parametrize("n,v", [(3, 1), (40, 500)])
def test_every_token_masked(n, v, dtype, element, mask):
    """lse is the score that all tokens have: their number's logarithm is nothing beside it.  Then loss is 0 and every exponential 1."""
    x, w = torch.zeros((1, n, 64), dtype=TYPES[dtype], device="cuda"), torch.zeros((v, 64), dtype=TYPES[dtype], device="cuda")
    x[..., 5], w[:, 5] = element, mask
    targets = torch.arange(n, device="cuda")[None] % v
    loss, lse = forward(x, w, targets)
    score = x[0, 0, 5].double() * w[0, 5].double()
    assert (lse.double() == score).all() and (loss == 0).all()
    x[..., 6] = 1.0      # (gradients of elements that do not overflow)
    dloss = torch.ones((1, n), device="cuda")
    _, dw = backward(dloss, x, w, targets, lse)
    count = torch.bincount(targets[0], minlength=v)
    assert torch.equal(dw[:, 6], (n - count).float())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_score_far_above_the_others(dtype):
    """2.55e38: lse is that score, the others' exponentials are 0."""
    rng = np.random.default_rng(8)
    n, v = 130, 700
    x, w = torch.zeros((1, n, 64), dtype=TYPES[dtype]), normal(rng, (v, 64), dtype)
    x[0, :, 0], x[0, :, 3] = 2.0 ** 60, 1.0
    w[:, 0], w[300, 0] = 0.0, 1.5 * 2.0 ** 67
    x, w = x.cuda(), w.cuda()
    targets = torch.full((1, n), 300, device="cuda")
    targets[0, ::2] = 17
    loss, lse = forward(x, w, targets)
    most = 1.5 * 2.0 ** 127
    assert (lse == most).all() and (loss[0, 1::2] == 0).all() and (loss[0, ::2] == most).all()
    _, dw = backward(torch.ones((1, n), device="cuda"), x, w, targets, lse)
    want = torch.zeros(v, device="cuda")
    want[300], want[17] = n / 2, -n / 2
    assert torch.equal(dw[:, 3], want)


@pytest.mark.parametrize("element,mask", [(1.0, LOWEST), (1.0, -1.5 * 2.0 ** 127), (0.5, LOWEST), (1.25, LOWEST), (2.0 ** 100, LOWEST)])
@pytest.mark.parametrize("case", MASKED)
def test_masked_tokens_of_fp32(case, element, mask):
    """Masks past the largest bf16 number, of which the last two give scores of minus infinity: weight zero, and gradients of zero times a finite number."""
    n, h, v, spans = case
    rng = np.random.default_rng(n + v)
    x, w, on = masked_call(rng, n, h, v, spans, "f32", element, mask)
    check_against_the_others(x, w, on, "f32", rng)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", MASKED)
def test_masks_of_minus_infinity(case, dtype):
    """As above, but for the mask's own column of dx, in which zero times infinity is NaN."""
    n, h, v, spans = case
    rng = np.random.default_rng(n + v)
    x, w, on = masked_call(rng, n, h, v, spans, dtype, 1.0, float("-inf"))
    finite = w.clone()
    finite[:, -1] = 0.0
    finite[on, -1] = w[on, -1]
    targets = torch.from_numpy(on[rng.integers(0, len(on), n)])[None].cuda()
    loss, lse = forward(x, w, targets)
    x64, w64, at = f64(x)[0], f64(w)[on], np.searchsorted(on, targets[0].cpu().numpy())
    want_loss, want_lse = E.token_loss(x64, w64, at)
    e_loss, e_lse = loss_tolerances(x64, w64, at, want_lse, None, dtype, np.arange(n))
    within(f64(lse)[0], want_lse, e_lse, "lse")
    within(f64(loss)[0], want_loss, e_loss, "loss")
    g = torch.rand((1, n), device="cuda") + 0.5
    dx, dw = backward(g, x, w, targets, lse)
    assert torch.isnan(dx[..., -1]).all()
    lse64, g64 = f64(lse)[0], f64(g)[0]
    want_dx, want_dw, _, _ = E.token_loss_grad(g64, x64, w64, at, lse64)
    _, _, e_dx, e_dw = loss_tolerances(x64, w64, at, lse64, g64, dtype, np.arange(n))
    within(f64(dx)[0, :, :-1], want_dx[:, :-1], (e_dx * (1 + HALF[dtype]) + HALF[dtype] * np.abs(want_dx))[:, :-1], "dx")
    got = f64(dw)
    within(got[on], want_dw, e_dw * (1 + U) + U * np.abs(want_dw), "dweight")
    got[on] = 0
    assert not got.any()


@pytest.mark.parametrize("n,h,v", [(1, 1, 1), (70, 72, 300), (130, 67, 700), (300, 136, 2055), (1040, 64, 16384)])
def test_fp32_scores_that_are_not_finite_are_what_fp32_arithmetic_gives(n, h, v):
    """Infinities and NaN in rows and weights, and sums that pass the largest float, against the formula in fp32 on the CPU: what is NaN, infinite and finite is the same; rows
    without any are as without them."""
    rng = np.random.default_rng(n)
    x, w = normal(rng, (1, n, h), "f32"), normal(rng, (v, h), "f32", 2 / np.sqrt(h))
    targets = torch.from_numpy(rng.integers(0, v, (1, n)))
    x[0, :, 0] = x[0, :, 0].abs() + 0.1
    w[v // 2, 0] = float("-inf")                              # a score of minus infinity for every row
    kinds = [float("inf"), float("-inf"), float("nan"), 3e38, -3e38]
    for i, r in enumerate(range(0, n, 11)):
        x[0, r, (i * 7) % h] = kinds[i % 5]
    if v > 20:
        w[v - 1, h - 1], w[v - 2, h - 1] = 3e38, 3.4e38       # with rows whose last element is above 1: infinite
    z = x[0] @ w.T
    most = z.max(1).values
    lse = torch.where(most == float("-inf"), most, most + (z - most[:, None]).exp().sum(1).log())     # (of nothing but masked tokens: log 0)
    loss = lse - z.gather(1, targets[0][:, None])[:, 0]
    got_loss, got_lse = forward(x.cuda(), w.cuda(), targets.cuda())
    for got, want in ((got_loss, loss), (got_lse, lse)):
        got = got[0].cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
        there = torch.isfinite(want)
        assert torch.equal(got.sign()[torch.isinf(want)], want.sign()[torch.isinf(want)])
        # fp32 sums of h terms on both sides, of magnitudes that stay below 60, or one term and what is nothing beside it
        off = (got[there].double() - want[there].double()).abs() / want[there].double().abs().clamp(min=1.0)
        assert there.sum() == 0 or off.max() <= (16 * h + 64) * U * 60


@pytest.mark.parametrize("n,h,v", [(70, 72, 300), (300, 136, 2055)])
@pytest.mark.parametrize("power", [-116, -100, 60])
def test_fp32_gradients_of_small_and_large_size(n, h, v, power):
    """Gradients scale with dloss.  At 2^-116 numbers below 2^-126 are among them: dz is off by 2^-150, and by as much where its last plane ends; in dx that makes up to v 2^-149 |w| < 2^-139
    beside elements of 2^-116 |w| > 2^-119, in dweight n 2^-149 |x| < 2^-138 beside 2^-116."""
    rng = np.random.default_rng(power + 200)
    x, w = normal(rng, (1, n, h), "f32").cuda(), normal(rng, (v, h), "f32", 0.1).cuda()
    targets = torch.from_numpy(rng.integers(0, v, (1, n))).cuda()
    _, lse = forward(x, w, targets)
    g = torch.rand((1, n), device="cuda") + 0.5
    ones, many = backward(g, x, w, targets, lse), backward(g * 2.0 ** power, x, w, targets, lse)
    for a, b in zip(ones, many):
        off = (b.double() * 2.0 ** -power - a.double()).abs().amax()
        assert off <= (2.0 ** -20 * a.double().abs().amax() if power < -100 else 0), off
