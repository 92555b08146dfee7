"""Embedding and its gradient against 64 bits, at the sizes, tokens and layouts where it can go wrong."""
import numpy as np
import pytest
import torch

import paper_2406_03488_amd as s1f
from ends_harness import HALF, U, TYPES, f64, normal, placed, space, tokens_of, untouched, within
from oracle import ends as E

pytestmark = pytest.mark.gpu

# batch, rows, hidden, vocab, share of tokens outside, layout
CASES = [(1, 1, 1, 1, 0.0, "dense"), (1, 1, 64, 5, 0.0, "dense"), (1, 1, 8, 5, 1.0, "dense"), (3, 7, 24, 11, 0.3, "view"),
         (2, 33, 515, 97, 0.1, "view"), (1, 64, 80, 3, 0.0, "odd"), (2, 65, 72, 40, 0.2, "seq"), (1, 129, 2056, 70, 0.0, "dense"),
         (1, 300, 257, 1000, 0.5, "odd"), (2, 500, 16, 2, 0.0, "dense"), (1, 1000, 40, 513, 1.0, "dense"), (3, 341, 64, 50021, 0.1, "seq")]


def forward(ids, table, scale, layout):
    b, n = ids.shape
    out = placed(torch.empty((b, n, table.shape[1]), dtype=table.dtype), layout, float("nan"))
    s1f.embed_fwd(ids, table, scale, out)
    return out


def backward(ids, dout, scale, acc):
    n = s1f.embed_bwd_workspace_bytes(ids, dout, acc)
    ws, buffer = space(n)
    s1f.embed_bwd(ids, dout, scale, acc, ws)
    assert untouched(buffer, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_forward_bit_for_bit(case, dtype):
    b, n, h, v, blank, layout = case
    rng = np.random.default_rng(n * h + v)
    table = normal(rng, (v, h), dtype).cuda()
    ids = tokens_of(rng, b, n, v, blank, layout)
    out = forward(ids, table, 1.7, layout)
    known = (ids >= 0) & (ids < v)
    want = torch.where(known[..., None], table[ids.clamp(0, v - 1)].float() * np.float32(1.7).item(), 0.0).to(TYPES[dtype])
    assert torch.equal(out, want)
    if layout == "view":
        assert (out._base[:, :n] == 777.0).all() and (out._base[:, 2 * n:] == 777.0).all()
    if layout == "odd":
        assert (out._base[:, 0] == 777.0).all() and (out._base[:, :, 0] == 777.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES + [(1, 12288, 24, 300, 0.1, "dense"), (1, 12289, 24, 300, 0.1, "dense"), (1, 16384, 24, 300, 0.1, "dense"), (1, 16385, 24, 300, 0.1, "dense"),
                                          (1, 8191, 40, 30, 0.0, "dense"), (1, 8193, 40, 30, 0.0, "odd"), (1, 33000, 2056, 7, 0.1, "dense"), (1, 65536, 8, 900, 0.1, "dense"), (1, 65537, 8, 900, 0.1, "dense"), (3, 40000, 8, 100003, 0.0, "seq"), (2, 9999, 17, 70000, 0.3, "view"),
                                          (1, 40000, 8, 1, 0.0, "dense"), (1, 17000, 8, 600000, 0.9, "dense"), (1, 20480, 8, 511, 1.0, "dense")])
def test_gradient(case, dtype):
    b, n, h, v, blank, layout = case
    rng = np.random.default_rng(n * h + v + 1)
    ids = tokens_of(rng, b, n, v, blank, layout)
    dout = placed(normal(rng, (b, n, h), dtype), layout)
    acc = normal(rng, (v, h), "f32").cuda()
    was = f64(acc)
    backward(ids, dout, 0.75, acc)
    grad, size, count = E.embed_grad(ids.cpu().numpy().reshape(-1), f64(dout).reshape(-1, h), 0.75, v)
    within(f64(acc), was + grad, (count[:, None] + 4) * U * (size + np.abs(was)), "dtable")
    assert (f64(acc)[count == 0] == was[count == 0]).all()


def test_gradient_is_the_same_every_time():
    rng = np.random.default_rng(3)
    for n, v in ((3000, 40), (30000, 5000)):
        ids, dout = tokens_of(rng, 1, n, v, 0.1), normal(rng, (1, n, 72), "f32").cuda()
        got = []
        for _ in range(3):
            acc = torch.zeros((v, 72), device="cuda")
            backward(ids, dout, 1.0, acc)
            got.append(acc)
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("n", [700, 20000])
def test_one_token_throughout(n):
    """One run through every chunk, and runs that end exactly on chunks' borders."""
    ids = torch.zeros((1, n), dtype=torch.int64, device="cuda")
    ids[0, 320:352], ids[0, 352:353] = 2, 3
    dout = torch.ones((1, n, 264), device="cuda")
    acc = torch.zeros((5, 264), device="cuda")
    backward(ids, dout, 2.0, acc)
    assert acc[:, 0].tolist() == [2.0 * (n - 33), 0, 64, 2, 0] and (acc == acc[:, :1]).all()


def test_rows_that_are_not_finite_stay_with_their_token():
    ids = torch.tensor([[4, -1, 7, 4, 2, 99]], device="cuda")
    dout = torch.ones((1, 6, 8), device="cuda")
    dout[0, 1], dout[0, 5], dout[0, 2] = float("nan"), float("inf"), float("nan")
    acc = torch.zeros((10, 8), device="cuda")
    backward(ids, dout, 1.0, acc)
    assert torch.isnan(acc[7]).all() and acc[[0, 1, 2, 4, 9], 0].tolist() == [0, 0, 1, 2, 0]
    table = torch.full((10, 8), float("nan"), device="cuda")
    table[4] = float("-inf")
    out = forward(ids, table, 1.0, "dense")
    assert (out[0, [1, 5]] == 0).all() and (out[0, 0] == float("-inf")).all() and torch.isnan(out[0, 2]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_past_32_bits(dtype):
    v, h = 280000, 8192                      # 2^31 elements lie below row 262144
    table = torch.zeros((v, h), dtype=TYPES[dtype], device="cuda")
    table[[3, 262144 + 3, v - 1]] = torch.tensor([[1.0], [2.0], [3.0]], device="cuda").to(TYPES[dtype])
    ids = torch.tensor([[3, 262147, v - 1, 262147]], device="cuda")
    out = forward(ids, table, 1.0, "dense")
    assert (out[0] == torch.tensor([[1.0], [2], [3], [2]], device="cuda")).all()
    del table
    acc = torch.zeros((v, h), device="cuda")
    backward(ids, out, 1.0, acc)
    assert acc[[3, 262147, v - 1]].unique(dim=1).flatten().tolist() == [1, 4, 3] and acc.sum().item() == 8 * h
