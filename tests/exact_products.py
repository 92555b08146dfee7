"""Inputs of the token loss whose results are known element by element without a tolerance for sums, whatever the size of the call: for its products, in which a tile, a part, a step of
the contraction or a product of planes that is missing, doubled or misplaced changes some element by more than a rounding.

The backward takes lse as given.  Above all scores by far it makes every exponential 0, at 0 with scores of 0 every one 1, so that dz is chosen here:
  one    lse = 10^4: dz[r][v] = -g[r] for v = target[r], else 0.  dx[r] = -g[r] W[target[r]], dW[target[r]] = -g[r] x[r] (targets differ, or g is 0): one product per element, of
         operands that fill their bits, at places all over the contraction.
  all    W or x is 0, lse = 0: dz[r][v] = g[r] (1 - [v = target[r]]).  dx[r] = g[r] (sum of W - W[target[r]]), dW[v] = sum of g x - those of rows with target v: of small whole
         numbers, so that every sum is exact.
  some   x[r] = unit vector k(r), W[v] = -200 but 0 at k(v), lse = 0: scores 0 where k(r) = k(v), else -200, and their exponentials 1 or 0 (2^-288).  Whole numbers again.
And scores by themselves: x[r] = a[r] e_k(r), one token b[k] e_k for each k: the row's lse is that token's score, one product, beside which the others (0, by 64 or more below) are nothing.
"""
import numpy as np
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# One product of two fp32 operands as six of planes: what the three others would add is at most 2^-24 (1 + 2^-9) of it, and five additions round by 2^-23 each, were they cut off.
ONE_PRODUCT = (1 + 2.0 ** -9 + 5 * 2) * 2.0 ** -24

# rows, hidden, vocabulary.  Which instances of the kernels they run: test_host_token_loss_products.py
SHAPES = [(1040, 512, 16384), (2304, 8192, 2304), (700, 128, 130), (130, 2000, 9000), (300, 1280, 20011), (700, 264, 9001), (5, 64, 129), (3000, 72, 2000)]
# whole rounds of big tiles of dx, with a rest in parts behind them or without one
WHOLE = [(2049, 8192, 1000), (4096, 4096, 700)]
# fp32 calls of so many rows that dweight's sums over them are cut into parts: middle and big tiles, the last part short
LONG = [(24577, 136, 515), (24581, 2048, 4100)]
# several pieces of the vocabulary, the last one short
PIECES = {"f32": (700, 264, 180000), "bf16": (1100, 64, 600011)}


def full(rng, shape, dtype, low=1.0, high=2.0):
    """Numbers of either sign in [low, high) that fill the bits of their type."""
    v = rng.uniform(low, high, shape) * rng.choice([-1.0, 1.0], shape)
    return torch.from_numpy(v.astype(np.float32)).to(TYPES[dtype])


def whole(rng, shape, dtype):
    return torch.from_numpy(rng.integers(-3, 4, shape).astype(np.float32)).to(TYPES[dtype])


def targets_of(rng, n, v, blank):
    """Different ones as far as there are, spread over the vocabulary; a share of rows has none."""
    t = np.concatenate([rng.permutation(v) for _ in range(-(-n // v))])[:n]
    first = np.arange(n) < v
    return np.where(rng.random(n) < blank, -1, t), first


def backward_case(kind, n, h, v, dtype, blank=0.0, seed=0):
    """x [1, n, h], weight, targets, lse, dloss on the CPU, and (dx, dweight) in 64 bits."""
    rng = np.random.default_rng(seed + 31 * n + h + v)
    t, first = targets_of(rng, n, v, blank)
    on, at = torch.from_numpy(t >= 0), torch.from_numpy(np.maximum(t, 0))
    x, w = torch.zeros((n, h), dtype=TYPES[dtype]), torch.zeros((v, h), dtype=TYPES[dtype])
    dx, dw = torch.zeros((n, h), dtype=torch.float64), torch.zeros((v, h), dtype=torch.float64)
    if kind == "one":
        x, w = full(rng, (n, h), dtype), full(rng, (v, h), dtype)
        g = torch.where(torch.from_numpy(first) & on, full(rng, n, dtype).float(), 0.0)
        lse = torch.full((n,), 1e4)
        dx[on] = -g[on].double()[:, None] * w[at[on]].double()
        dw[at[on & (g != 0)]] = -(g.double()[:, None] * x.double())[on & (g != 0)]
    else:
        g = torch.from_numpy(rng.integers(1, 3, n).astype(np.float32))
        lse = torch.zeros(n)
        if kind == "all dx":
            w = whole(rng, (v, h), dtype)
            dx[on] = g[on].double()[:, None] * (w.double().sum(0) - w[at[on]].double())
        elif kind == "all dw":
            x = whole(rng, (n, h), dtype)
            gx = torch.where(on[:, None], g[:, None] * x.float(), 0.0).double()
            dw = (gx.sum(0)[None].expand(v, h)).clone().index_add_(0, at, -gx)
        else:
            assert kind == "some"
            kr, kv = torch.from_numpy(rng.integers(0, h, n)), torch.from_numpy(rng.integers(0, h, v))
            x[torch.arange(n), kr] = 1.0
            w.fill_(-200.0)
            w[torch.arange(v), kv] = 0.0
            # dz of a row: g for the tokens of its k, less g for its target
            of_k = torch.zeros((h, h), dtype=torch.float64).index_add_(0, kv, w.double())
            dx[on] = g[on].double()[:, None] * (of_k[kr[on]] - w[at[on]].double())
            sums = torch.zeros((h, h), dtype=torch.float64).index_add_(0, kr, torch.where(on[:, None], g[:, None] * x.float(), 0.0).double())
            dw = sums[kv].index_add_(0, at, -torch.where(on[:, None], g[:, None] * x.float(), 0.0).double())
    return x[None], w, torch.from_numpy(t)[None], lse[None], g[None], dx, dw


def scores_case(n, h, v, dtype, seed=0):
    """x, weight, targets, and lse in 64 bits (loss is 0)."""
    rng = np.random.default_rng(seed + 17 * n + h + v)
    kinds = min(h, v)
    places, token = rng.permutation(h)[:kinds], rng.permutation(v)[:kinds]
    of_row = rng.integers(0, kinds, n)
    a, b = full(rng, n, dtype, 8, 16).abs(), full(rng, kinds, dtype, 8, 16).abs()
    x, w = torch.zeros((n, h), dtype=TYPES[dtype]), torch.zeros((v, h), dtype=TYPES[dtype])
    x[torch.arange(n), torch.from_numpy(places[of_row])] = a
    w[torch.from_numpy(token), torch.from_numpy(places)] = b
    lse = a.double() * b.double()[torch.from_numpy(of_row)]
    return x[None], w, torch.from_numpy(token[of_row])[None], lse
