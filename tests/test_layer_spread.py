"""layer_spread passes what a kernel computes in fp32 or bf16, and rejects what has lost a stage, a part or a plane.  No device: the kernels' arithmetic in torch."""
import pytest
import torch

import layer_spread as S
from oracle import layer as L

N, H, F = 160, 192, 328


def operands(dtype, act="silu", n=N, h=H, f=F):
    gen = torch.Generator().manual_seed(n + h + f)
    normal = lambda *shape, scale=1.0: (torch.randn(shape, generator=gen) * scale).to(torch.bfloat16 if dtype == "bf16" else torch.float32).double()
    return normal(n, h), normal(n, h), normal(2 * f, h, scale=1.5 / h ** 0.5), normal(h, f, scale=f ** -0.5)


def to(t, dtype):
    return t.to(torch.bfloat16 if dtype == "bf16" else torch.float32).double()


def planes(t):
    p0 = t.float().bfloat16().float()
    p1 = (t.float() - p0).bfloat16().float()
    return [p.double() for p in (p0, p1, (t.float() - p0 - p1).bfloat16().float())]


SIX = [(2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0)]


def product(a, b, dtype, pairs=SIX):
    """What the kernels make of a @ b: stages of 64 terms, each of six pairs of planes, added in fp32."""
    total = torch.zeros(len(a), b.shape[1])
    pa, pb = (planes(a), planes(b)) if dtype == "f32" else ([a], [b])
    for k in range(0, a.shape[1], 32):
        for i, j in (pairs if dtype == "f32" else [(0, 0)]):
            total += (pa[i][:, k:k + 32] @ pb[j][k:k + 32]).float()
    return total.double()


def forward(x, w_in, w_out, act, dtype, pairs=SIX):
    z = product(x, w_in.T, dtype, pairs)
    f = len(w_in) // 2
    h = to((S.activation(z[:, :f], act)[0] * z[:, f:]).float().double(), dtype)
    return to(z, dtype), to(product(h, w_out.T, dtype, pairs), dtype), h


def backward(dy, x, w_in, w_out, act, gate_up, dtype, pairs=SIX):
    f = len(w_in) // 2
    g, u = gate_up[:, :f], gate_up[:, f:]
    a, slope = S.activation(g, act)
    dh = product(dy, w_out, dtype, pairs)
    dz, h = to(torch.cat([dh * u * slope, dh * a], 1), dtype), to(a * u, dtype)
    return {"dx": to(product(dz, w_in, dtype, pairs), dtype), "dw_in": product(dz.T, x, dtype, pairs), "dw_out": product(dy.T, h, dtype, pairs)}


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_and_errors_of_the_kernels_arithmetic(dtype, act):
    dy, x, w_in, w_out = operands(dtype)
    expected = S.forward(x, w_in, w_out, act, dtype)
    oracle = L.gated_ffn(x.numpy(), w_in.numpy(), w_out.numpy(), act)
    assert torch.allclose(expected["y"][0], torch.from_numpy(oracle[0]), rtol=1e-11, atol=1e-11) and torch.allclose(expected["gate_up"][0], torch.from_numpy(oracle[1]), rtol=1e-12, atol=1e-12)
    z, y, _ = forward(x, w_in, w_out, act, dtype)
    S.near(z, expected["gate_up"], "gate_up")
    S.near(y, expected["y"], "y")
    expected = S.backward(dy, x, w_in, w_out, act, z, dtype, S.U)
    oracle = L.gated_ffn_grad(dy.numpy(), x.numpy(), w_in.numpy(), w_out.numpy(), act, z.numpy())
    got = backward(dy, x, w_in, w_out, act, z, dtype)
    for i, name in enumerate(("dx", "dw_in", "dw_out")):
        assert torch.allclose(expected[name][0], torch.from_numpy(oracle[i]), rtol=1e-10, atol=1e-10)
        S.near(got[name], expected[name], name)


def rejected(got, expected):
    try:
        S.near(got, expected, "")
    except AssertionError:
        return True
    return False


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lost_and_doubled_stages_are_rejected(dtype):
    """64 terms of a sum left out, or taken twice, in one block of 32 x 32 of y, dx and the weights' gradients, sums as long as those of large calls."""
    dy, x, w_in, w_out = operands(dtype, n=96, h=64, f=11008)
    expected = S.forward(x, w_in, w_out, "silu", dtype)
    z, y, h = forward(x, w_in, w_out, "silu", dtype)
    assert not rejected(y, expected["y"])
    for sign in (1, -1):
        bad = y.clone()
        bad[32:64, :32] += sign * (h[32:64, 640:704] @ w_out[:32, 640:704].T)
        assert rejected(bad, expected["y"])
    expected = S.backward(dy, x, w_in, w_out, "silu", z, dtype, S.U)
    got = backward(dy, x, w_in, w_out, "silu", z, dtype)
    dh = dy @ w_out
    g, u = z[:, :11008], z[:, 11008:]
    a, slope = S.activation(g, "silu")
    dz = torch.cat([dh * u * slope, dh * a], 1)
    for name, lost in (("dx", dz[:32, 20032:20096] @ w_in[20032:20096, :32]), ("dw_in", dz[64:, :32].T @ x[64:, :32]), ("dw_out", dy[64:, :32].T @ h[64:, :32])):
        assert not rejected(got[name], expected[name])
        for sign in (1, -1):
            bad = got[name].clone()
            bad[:32, :32] += sign * lost
            assert rejected(bad, expected[name]), name
    # one term of 22016, of all of dx
    assert rejected(got["dx"] - dz[:, 77:78] @ w_in[77:78], expected["dx"])


@pytest.mark.parametrize("lost", [[(2, 0)], [(0, 2)], [(1, 1)], [(2, 0), (0, 2)], [(1, 1), (2, 0), (0, 2)]])
def test_lost_planes_are_rejected(lost):
    """fp32 products of fewer than six pairs of planes, the others as they are: sums of 1000 and 4000 terms."""
    pairs = [p for p in SIX if p not in lost]
    for n, h, f in ((70, 72, 1000), (70, 1000, 72), (2000, 72, 72), (70, 72, 4000)):
        dy, x, w_in, w_out = operands("f32", n=n, h=h, f=f)
        expected = S.forward(x, w_in, w_out, "silu", "f32")
        z, y, hid = forward(x, w_in, w_out, "silu", "f32")
        assert not rejected(y, expected["y"]) and not rejected(z, expected["gate_up"])
        assert rejected(product(x, w_in.T, "f32", pairs), expected["gate_up"]), ("gate_up", n, h, f)
        if f < 4000 or len(lost) > 1:
            assert rejected(product(hid, w_out.T, "f32", pairs), expected["y"]), ("y", n, h, f)
        expected = S.backward(dy, x, w_in, w_out, "silu", z, "f32", S.U)
        got, bad = backward(dy, x, w_in, w_out, "silu", z, "f32"), backward(dy, x, w_in, w_out, "silu", z, "f32", pairs)
        for name in got:
            assert not rejected(got[name], expected[name])
            if f < 4000 or len(lost) > 1:
                assert rejected(bad[name], expected[name]), (name, n, h, f)


def test_operands_rounded_to_bf16_are_rejected():
    dy, x, w_in, w_out = operands("f32")
    short = [t.bfloat16().double() for t in (dy, x, w_in, w_out)]
    assert rejected(forward(*short[1:], "silu", "f32")[1], S.forward(x, w_in, w_out, "silu", "f32")["y"])


def test_one_sum_of_many_rows_is_rejected():
    """131072 terms of one sign in one fp32 sum; in turns of 8192 they pass."""
    n = 131072
    gen = torch.Generator().manual_seed(4)
    a, b = torch.randn((12, n), generator=gen).abs().double(), torch.randn((n, 16), generator=gen).abs().double()
    expected = (*S.sums(a, b, "f32"), None)
    turns = torch.zeros(12, 16)
    for k in range(0, n, 8192):
        turns += product(a[:, k:k + 8192], b[k:k + 8192], "f32").float()
    assert not rejected(turns, expected) and rejected(product(a, b, "f32"), expected)


def test_lost_terms_of_gains_gradients_are_rejected():
    """One row's share of one head left out of 200006 rows of two heads; the kernel's order of additions passes."""
    import numpy as np
    from test_gpu_rope_gains import MANY
    b, hq, hk, n, dim, rotary = MANY[0][:6]
    rng = np.random.default_rng(3)
    d, x = rng.normal(size=(b, hq, n, dim)).astype(np.float32), rng.normal(size=(b, hq, n, dim)).astype(np.float32)
    at, freqs, start = np.arange(n)[None].repeat(b, 0), L.frequencies(rotary), rng.normal(size=dim)
    dy, rstd = L.rotate(d.astype(np.float64), at, freqs, 1.0, False, back=True), L.head_norm(x.astype(np.float64), 1.0, 1e-6)[1]
    terms = dy * x * rstd
    want = start + terms.sum((0, 1, 2))
    tolerance = S.gains_tolerance(d.astype(np.float64), x.astype(np.float64), rstd, rotary, False, 1.0, S.gains_chain(b * n, hq, hk, dim, True), start)(want)
    flat = (dy.astype(np.float32) * (x * rstd.astype(np.float32))).reshape(-1, dim)
    lanes = 256 * 32
    flat = np.concatenate([flat, np.zeros((-len(flat) % lanes, dim), np.float32)]).reshape(-1, lanes, dim)
    sums = np.add.accumulate(flat, 0, dtype=np.float32)[-1]
    got = start.astype(np.float32) + np.add.accumulate(sums.reshape(64, -1, dim), 1, dtype=np.float32)[:, -1].sum(0)
    assert (np.abs(got - want) <= tolerance).all()
    for lost in (terms[0, 1, 777], terms[1, 0, n - 1]):
        assert (np.abs(got - lost - want) > tolerance).any()
    assert S.gains_chain(200006, 2, 1, 8, True) < 600 and tolerance.max() < 0.05
