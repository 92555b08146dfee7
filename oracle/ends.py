"""Embedding, layer norm and token loss with their gradients, in 64 bits from their definitions (numpy).

Rows are flat here: tokens and targets [n], hidden states [n, hidden]."""
import numpy as np


def known(tokens, vocab):
    return (tokens >= 0) & (tokens < vocab)


def embed(tokens, table, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    for r, t in enumerate(tokens):
        if 0 <= t < len(table):
            out[r] = scale * table[t]
    return out


def embed_grad(tokens, dout, scale, vocab):
    """(gradient of the table, sum of the magnitudes that it is made of, number of rows of each token)"""
    grad, size, count = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1])), np.zeros(vocab)
    for r, t in enumerate(tokens):
        if 0 <= t < vocab:
            grad[t] += scale * dout[r]
            size[t] += np.abs(scale * dout[r])
            count[t] += 1
    return grad, size, count


def layer_norm(x, gamma, beta, eps):
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def layer_norm_grad(dy, x, gamma, mean, rstd):
    """dx, dgamma, dbeta for statistics as they are given"""
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1)[:, None] - xhat * (g * xhat).mean(1)[:, None])
    return dx, (dy * xhat).sum(0), dy.sum(0)


def token_loss(x, weight, targets):
    """loss, lse; zeros for rows without a target"""
    rows = np.nonzero(known(targets, len(weight)))[0]
    loss, lse = np.zeros(len(x)), np.zeros(len(x))
    z = x[rows] @ weight.T
    most = z.max(1, initial=-np.inf)
    lse[rows] = most + np.log(np.exp(z - most[:, None]).sum(1))
    loss[rows] = lse[rows] - z[np.arange(len(rows)), targets[rows]]
    return loss, lse


def token_loss_grad(dloss, x, weight, targets, lse):
    """dx, dweight, and dz of the rows that count with their numbers"""
    rows = np.nonzero(known(targets, len(weight)))[0]
    dz = np.exp(x[rows] @ weight.T - lse[rows][:, None])
    dz[np.arange(len(rows)), targets[rows]] -= 1
    dz *= dloss[rows][:, None]
    dx = np.zeros(x.shape)
    dx[rows] = dz @ weight
    return dx, dz.T @ x[rows], dz, rows
