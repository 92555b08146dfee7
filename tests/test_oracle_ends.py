"""Pins of oracle/ends.py: hand-worked values, torch's CPU fp64 functions with autograd, finite differences, invariants."""
import numpy as np
import torch

from oracle import ends as E


def test_two_tokens_by_hand():
    table = np.array([[1.0, 2.0], [3.0, -4.0]])
    tokens = np.array([1, -1, 0, 1, 2])
    assert E.embed(tokens, table, 0.5).tolist() == [[1.5, -2.0], [0, 0], [0.5, 1.0], [1.5, -2.0], [0, 0]]
    grad, size, count = E.embed_grad(tokens, np.array([[1.0, 1], [9, 9], [2, -2], [3, -5], [9, 9]]), 2.0, 2)
    assert grad.tolist() == [[4, -4], [8, -8]] and size.tolist() == [[4, 4], [8, 12]] and count.tolist() == [1, 2]
    y, mean, rstd = E.layer_norm(np.array([[1.0, 3.0]]), np.array([2.0, 1.0]), np.array([0.0, 5.0]), 0.0)
    assert y.tolist() == [[-2.0, 6.0]] and mean.tolist() == [2.0] and rstd.tolist() == [1.0]
    loss, lse = E.token_loss(np.array([[1.0], [7.0]]), np.array([[0.0], [np.log(3.0)]]), np.array([1, -1]))
    assert np.allclose(loss, [np.log(4 / 3), 0]) and np.allclose(lse, [np.log(4.0), 0])
    dx, dw, dz, rows = E.token_loss_grad(np.array([2.0, 5.0]), np.array([[1.0], [7.0]]), np.array([[0.0], [np.log(3.0)]]), np.array([1, -1]), lse)
    assert np.allclose(dz, [[0.5, -0.5]]) and rows.tolist() == [0] and np.allclose(dw, [[0.5], [-0.5]])
    assert np.allclose(dx, [[-0.5 * np.log(3.0)], [0]])


def test_against_autograd():
    rng = np.random.default_rng(7)
    n, h, v = 9, 12, 17
    x, w, gamma, beta, dy = (rng.normal(size=s) for s in ((n, h), (v, h), (h,), (h,), (n, h)))
    tokens = rng.integers(-2, v + 2, n)
    on = (tokens >= 0) & (tokens < v)
    tx, tw, tg, tb = (torch.tensor(a, requires_grad=True) for a in (x, w, gamma, beta))
    y = torch.nn.functional.layer_norm(tx, (h,), tg, tb, 1e-5)
    y.backward(torch.tensor(dy))
    got, mean, rstd = E.layer_norm(x, gamma, beta, 1e-5)
    assert np.allclose(got, y.detach(), atol=1e-12)
    for a, b in zip(E.layer_norm_grad(dy, x, gamma, mean, rstd), (tx.grad, tg.grad, tb.grad)):
        assert np.allclose(a, b, atol=1e-11)
    tx.grad = None
    target = torch.tensor(np.where(on, tokens, -100))
    loss = torch.nn.functional.cross_entropy(tx @ tw.T, target, ignore_index=-100, reduction="none")
    dloss = rng.normal(size=n)
    loss.backward(torch.tensor(dloss))
    got, lse = E.token_loss(x, w, tokens)
    assert np.allclose(got, loss.detach(), atol=1e-12)
    dx, dw, _, _ = E.token_loss_grad(dloss, x, w, tokens, lse)
    assert np.allclose(dx, tx.grad, atol=1e-12) and np.allclose(dw, tw.grad, atol=1e-12)
    tw.grad = None
    out = torch.nn.functional.embedding(torch.tensor(tokens[on]), tw) * 1.5
    out.backward(torch.tensor(dy[on]))
    assert np.allclose(E.embed(tokens, w, 1.5)[on], out.detach()) and not E.embed(tokens, w, 1.5)[~on].any()
    assert np.allclose(E.embed_grad(tokens, dy, 1.5, v)[0], tw.grad)


def test_differences():
    rng = np.random.default_rng(8)
    n, h, v, step = 3, 5, 7, 1e-6
    x, w, gamma, beta, dy, dloss = (rng.normal(size=s) for s in ((n, h), (v, h), (h,), (h,), (n, h), (n,)))
    targets = np.array([2, -1, 6])
    _, lse = E.token_loss(x, w, targets)
    dx, dw, _, _ = E.token_loss_grad(dloss, x, w, targets, lse)
    _, mean, rstd = E.layer_norm(x, gamma, beta, 1e-3)
    nx, ng, nb = E.layer_norm_grad(dy, x, gamma, mean, rstd)

    def slope(f, a, at):
        lo, hi = a.copy(), a.copy()
        lo[at] -= step
        hi[at] += step
        return (f(hi) - f(lo)) / (2 * step)

    for at in ((0, 1), (1, 3), (2, 4)):
        assert abs(slope(lambda a: dloss @ E.token_loss(a, w, targets)[0], x, at) - dx[at]) < 1e-8
        assert abs(slope(lambda a: (dy * E.layer_norm(a, gamma, beta, 1e-3)[0]).sum(), x, at) - nx[at]) < 1e-8
    for at in ((0, 0), (6, 2)):
        assert abs(slope(lambda a: dloss @ E.token_loss(x, a, targets)[0], w, at) - dw[at]) < 1e-8
    assert abs(slope(lambda a: (dy * E.layer_norm(x, a, beta, 1e-3)[0]).sum(), gamma, 2) - ng[2]) < 1e-8
    assert abs(slope(lambda a: (dy * E.layer_norm(x, gamma, a, 1e-3)[0]).sum(), beta, 2) - nb[2]) < 1e-8


def test_invariants():
    rng = np.random.default_rng(9)
    x, w = rng.normal(size=(6, 8)), rng.normal(size=(11, 8))
    targets = rng.integers(0, 11, 6)
    loss, lse = E.token_loss(x, w, targets)
    _, dw, dz, _ = E.token_loss_grad(np.ones(6), x, w, targets, lse)
    assert np.allclose(dz.sum(1), 0) and np.allclose(dw.sum(0), 0)           # a row's probabilities sum to its target's one
    assert (loss > 0).all() and np.allclose(E.token_loss(x, w + 3.0, targets)[0], loss)   # the same score more for all
    y, _, rstd = E.layer_norm(x, np.ones(8), np.zeros(8), 0.0)
    assert np.allclose(y.mean(1), 0) and np.allclose((y ** 2).mean(1), 1)
    assert np.allclose(E.layer_norm(5 * x + 3, np.ones(8), np.zeros(8), 0.0)[0], y)
    empty = E.token_loss(x, w, np.full(6, -1))
    assert not empty[0].any() and not empty[1].any()
