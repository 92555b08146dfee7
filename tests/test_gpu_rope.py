"""Rotations of queries and keys, with and without norms of heads, and their gradients against 64 bits, at the sizes, layouts and values where they can go wrong."""
import numpy as np
import pytest
import torch

import paper_2406_03488_amd as s1f
from ends_harness import f64, normal, space, untouched
from layer_harness import check_backward, check_forward, heads, like
from oracle import layer as L

pytestmark = pytest.mark.gpu
EPS = np.float64(np.float32(1e-6))

# batch, heads, kv_heads, rows, head_dim, rotary_dim, layout of projections, layout of q_rot and caches; every width of the kernels, whole and not
CASES = [(1, 4, 4, 1, 64, 64, "dense", "dense"), (1, 64, 8, 1, 128, 128, "rows", "dense"), (2, 3, 1, 17, 128, 64, "dense", "rows"),
         (1, 8, 2, 33, 80, 80, "rows", "dense"), (2, 4, 2, 37, 80, 20, "rows", "dense"), (1, 2, 2, 65, 96, 24, "dense", "dense"),
         (3, 2, 1, 5, 256, 256, "dense", "wide"), (1, 2, 1, 7, 256, 2, "odd", "dense"), (1, 3, 3, 31, 128, 128, "odd", "odd"),
         (1, 5, 1, 9, 2, 2, "dense", "dense"), (2, 2, 2, 3, 6, 4, "dense", "dense"), (1, 1, 1, 11, 254, 250, "dense", "dense"),
         (1, 4, 1, 700, 64, 32, "rows", "rows"), (1, 2, 2, 19, 128, 0, "dense", "dense"), (1, 4, 2, 13, 72, 40, "wide", "wide"),
         (1, 40, 8, 300, 128, 128, "rows", "dense"), (2, 6, 2, 21, 16, 16, "dense", "dense"), (1, 3, 1, 40, 200, 100, "dense", "dense"),
         (1, 7, 7, 4500, 64, 64, "dense", "dense"), (1, 2, 1, 2500, 256, 10, "odd", "odd")]


class Call:
    """Inputs of one case on the device, its outputs, and the rows that a call may write."""

    def __init__(self, case, dtype, interleaved, norm, listed, magnitude=1.0, values=True, far=1 << 20):
        b, hq, hk, n, d, rotary, layout, other = case
        rng = self.rng = np.random.default_rng(hq * n + d + rotary)
        self.case, self.dtype, self.interleaved, self.norm, self.magnitude, self.values = case, dtype, interleaved, norm, magnitude, values
        self.q, self.k, self.v = heads(rng, (b, hq, n, d), dtype, layout), heads(rng, (b, hk, n, d), dtype, layout), heads(rng, (b, hk, n, d), dtype, layout)
        self.off, self.capacity = n // 3 + 1, n + n // 3 + 4
        self.other = other
        self.freqs64 = L.frequencies(rotary) if rotary else np.zeros(0)
        self.freqs = torch.from_numpy(self.freqs64).cuda()
        if listed:
            at = rng.integers(-5, far, (b, n))
            big = torch.full((b, 2 * n + 1), 7, dtype=torch.int64, device="cuda")
            big[:, n:2 * n] = torch.from_numpy(at).cuda()
            self.at, self.positions = at, big[:, n:2 * n]
        else:
            self.positions = far - 3
            self.at = np.broadcast_to(np.arange(n) + self.positions, (b, n))
        self.gains = (normal(rng, (d,), dtype, 0.3, 1.0).cuda(), normal(rng, (d,), dtype, 0.3, 1.0).cuda()) if norm else (None, None)
        self.turn = (self.freqs, magnitude, interleaved, self.positions, self.off)

    def caches(self, fill):
        b, _, hk, n, d = self.case[:5]
        return [heads(self.rng, (b, hk, self.capacity, d), self.dtype, self.other, fill=fill) for _ in range(2)]

    def forward(self):
        q_rot = heads(self.rng, self.q.shape, self.dtype, self.other, fill=float("nan"))
        kc, vc = self.caches(333.0)
        v, vc = (self.v, vc) if self.values else (None, None)
        if self.norm:
            s1f.qk_norm_rope_fwd(self.q, self.k, v, *self.gains, 1e-6, *self.turn, q_rot, kc, vc)
        else:
            s1f.rope_fwd(self.q, self.k, v, *self.turn, q_rot, kc, vc)
        return q_rot, kc, vc

    def rows(self, t):
        return t[:, :, self.off:self.off + self.case[3]]

    def outside(self, t):
        return torch.cat([t[:, :, :self.off], t[:, :, self.off + self.case[3]:]], 2)

    def backward(self):
        b, hq, hk, n, d = self.case[:5]
        rng = np.random.default_rng(n + 1)
        dq_rot = heads(rng, self.q.shape, self.dtype, self.other)
        dka, dva = (heads(rng, (b, hk, self.capacity, d), "f32", self.other) for _ in range(2))
        dq, dk, dv = like(self.q), like(self.k), like(self.v)
        dva, dv = (dva, dv) if self.values else (None, None)
        kept = dka.clone()
        if self.norm:
            was = normal(rng, (d,), "f32").cuda(), normal(rng, (d,), "f32").cuda()
            dgains = was[0].clone(), was[1].clone()
            size = s1f.qk_norm_rope_bwd_workspace_bytes(dq_rot, dka)
            ws, buffer = space(size)
            s1f.qk_norm_rope_bwd(dq_rot, dka, dva, self.q, self.k, *self.gains, 1e-6, *self.turn, dq, dk, dv, *dgains, ws)
            assert untouched(buffer, size)
        else:
            was = dgains = (None, None)
            s1f.rope_bwd(dq_rot, dka, dva, *self.turn, dq, dk, dv)
        assert torch.equal(dka, kept)
        return dq_rot, dka, dva, dq, dk, dv, was, dgains

    def check_forward(self, out):
        q_rot, kc, vc = out
        rest = (EPS, self.at, self.freqs64, np.float64(np.float32(self.magnitude)), self.interleaved, self.dtype)
        check_forward(self.q, q_rot, self.gains[0], *rest, "q_rot")
        check_forward(self.k, self.rows(kc), self.gains[1], *rest, "k")
        assert (self.outside(kc) == 333.0).all()
        if self.values:
            assert torch.equal(self.rows(vc), self.v) and (self.outside(vc) == 333.0).all()

    def check_backward(self, out):
        dq_rot, dka, dva, dq, dk, dv, was, dgains = out
        rest = (EPS, self.at, self.freqs64, np.float64(np.float32(self.magnitude)), self.interleaved, self.dtype)
        check_backward(dq_rot, dq, self.q, self.gains[0], dgains[0], was[0], *rest, "dq")
        check_backward(self.rows(dka), dk, self.k, self.gains[1], dgains[1], was[1], *rest, "dk")
        if self.values:
            assert torch.equal(dv, self.rows(dva).to(dv.dtype))


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_forward_and_gradient(case, dtype, interleaved, norm):
    c = Call(case, dtype, interleaved, norm, listed=case[3] % 2 == 1)
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("case", [(2, 2, 1, 100003, 8, 8, "rows", "dense"), (1, 3, 2, 150001, 24, 10, "dense", "dense"), (1, 40, 40, 2100, 16, 16, "dense", "dense")])
def test_many_units_to_a_workgroup(case, norm):
    """More rows than there are workgroups: each walks blocks of them, with heads of every tensor."""
    c = Call(case, "bf16", False, norm, True)
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("norm", [False, True])
def test_magnitude_and_no_values(norm):
    c = Call((2, 4, 2, 29, 128, 96, "rows", "dense"), "f32", False, norm, True, magnitude=1.25, values=False)
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("far", [1, 4096, 1 << 24, 1 << 30])
def test_far_positions(far):
    """Angles of 2^30 radians: a product in 32 bits would be off by many turns."""
    c = Call((1, 2, 1, 64, 64, 64, "dense", "dense"), "f32", False, False, True, far=far)
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("interleaved", [False, True])
def test_every_quarter_turn(interleaved):
    """Angles next to multiples of a quarter turn, on both sides of each."""
    n = 4096
    freqs = np.array([np.pi / 4, np.pi / 2, np.pi / 2 + 2.0 ** -40, 1e-9, 3.0, 0.0, np.pi, 1.0])
    c = Call((1, 1, 1, n, 16, 16, "dense", "dense"), "f32", interleaved, False, False)
    c.freqs64, c.freqs = freqs, torch.from_numpy(freqs).cuda()
    c.positions, c.at = -n // 2, (np.arange(n) - n // 2)[None]
    c.turn = (c.freqs, 1.0, interleaved, c.positions, c.off)
    c.check_forward(c.forward())


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(dtype, norm):
    """q_rot is q, the caches' rows are k and v, dq is dq_rot."""
    c = Call((2, 4, 2, 25, 128, 64, "rows", "dense"), dtype, False, norm, True)
    want = c.forward()
    q, k, v = (like(t).copy_(t) for t in (c.q, c.k, c.v))
    turn = (*c.turn[:4], 0)
    if norm:
        s1f.qk_norm_rope_fwd(q, k, v, *c.gains, 1e-6, *turn, q, k, v)
    else:
        s1f.rope_fwd(q, k, v, *turn, q, k, v)
    assert torch.equal(q, want[0]) and torch.equal(k, c.rows(want[1])) and torch.equal(v, c.v)
    dq_rot = like(c.q).copy_(heads(c.rng, c.q.shape, dtype, "rows"))
    dka, dva = (heads(c.rng, (2, 2, 40, 128), "f32", "dense") for _ in range(2))
    dgains = []
    for dq in (like(c.q), dq_rot):
        dk, dv = like(c.k), like(c.v)
        if norm:
            dgains.append(torch.zeros(2, 128, device="cuda"))
            ws, _ = space(s1f.qk_norm_rope_bwd_workspace_bytes(dq_rot, dka))
            s1f.qk_norm_rope_bwd(dq_rot, dka, dva, c.q, c.k, *c.gains, 1e-6, *c.turn, dq, dk, dv, *dgains[-1], ws)
        else:
            s1f.rope_bwd(dq_rot, dka, dva, *c.turn, dq, dk, dv)
        if dq is not dq_rot:
            want = dq
    assert torch.equal(want, dq_rot) and (not norm or torch.equal(*dgains))


@pytest.mark.parametrize("interleaved", [False, True])
def test_what_is_not_finite_stays_in_its_pair(interleaved):
    c = Call((1, 3, 2, 40, 128, 64, "dense", "dense"), "f32", interleaved, False, False)
    clean = c.forward()
    first, second = L.pairs(64, interleaved)
    c.q[0, 1, 7, first[5]], c.q[0, 2, 9, 100], c.k[0, 1, 3, second[0]] = float("inf"), float("nan"), float("-inf")
    got = c.forward()
    mask = torch.ones_like(clean[0], dtype=torch.bool)
    mask[0, 1, 7, [first[5], second[5]]] = False
    mask[0, 2, 9, 100] = False
    assert torch.equal(got[0][mask], clean[0][mask]) and not torch.isfinite(got[0][~mask]).any()
    bad = c.rows(got[1])[0, 1, 3]
    rest = [i for i in range(128) if i not in (first[0], second[0])]
    assert torch.equal(bad[rest], c.rows(clean[1])[0, 1, 3][rest]) and not torch.isfinite(bad[[first[0], second[0]]]).any()


def test_heads_that_are_zero_or_not_finite():
    """A head of zeros has the norm 1 / sqrt(eps); one that holds a NaN is lost alone."""
    c = Call((1, 4, 2, 33, 80, 32, "dense", "dense"), "f32", False, True, False)
    clean = c.forward(), c.backward()
    c.q[0, 1, 5], c.q[0, 2, 6, 3] = 0.0, float("nan")
    got = c.forward(), c.backward()
    assert (got[0][0][0, 1, 5] == 0).all() and torch.isnan(got[0][0][0, 2, 6]).all()
    mask = torch.ones(4, 33, dtype=torch.bool)
    mask[1, 5] = mask[2, 6] = False
    assert torch.equal(got[0][0][0][mask], clean[0][0][0][mask]) and torch.equal(got[1][3][0][mask], clean[1][3][0][mask])
    assert torch.isfinite(got[1][3][0, 1, 5]).all() and torch.isnan(got[1][7][0]).all() and torch.isfinite(got[1][7][1]).all()


@pytest.mark.parametrize("case", [(1, 5, 3, 7, 128, 0, "dense", "dense"), (1, 3, 1, 33, 80, 0, "dense", "dense"), (1, 3, 1, 5, 6, 0, "dense", "dense")])
def test_infinite_gradients(case):
    """An infinity in the last head of the last row is one share of its column of the gain's gradient."""
    c = Call(case, "f32", False, True, False)
    dq_rot, dka, _, _, _, _, was, _ = c.backward()
    dq_rot[0, -1, -1, 1] = c.rows(dka)[0, -1, -1, 2] = float("inf")
    dgains = [w.clone() for w in was]
    ws, _ = space(s1f.qk_norm_rope_bwd_workspace_bytes(dq_rot, dka))
    s1f.qk_norm_rope_bwd(dq_rot, dka, None, c.q, c.k, *c.gains, 1e-6, *c.turn, torch.empty_like(c.q), torch.empty_like(c.k), None, *dgains, ws)
    for got, x, col in ((dgains[0], c.q, 1), (dgains[1], c.k, 2)):
        assert got[col].item() == float("inf") * np.sign(x[0, -1, -1, col].item()) and torch.isfinite(got).sum() == len(got) - 1


def test_gradients_of_gains_are_the_same_every_time():
    c = Call((2, 8, 2, 900, 128, 128, "rows", "dense"), "bf16", False, True, False)
    runs = [c.backward() for _ in range(3)]
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r[3:6] + r[7], runs[0][3:6] + runs[0][7]))


def test_gradient_against_differences():
    """The norm and the rotation as one function: d(sum w * out) along random directions."""
    c = Call((1, 2, 1, 6, 32, 16, "dense", "dense"), "f32", True, True, False, far=50)
    dq_rot, dka, _, dq, dk, _, was, dgains = c.backward()

    def value(q, k, gq, gk):
        total = (L.rotate(L.head_norm(q, gq, EPS)[0], c.at, c.freqs64, 1.0, True) * f64(dq_rot)).sum()
        return total + (L.rotate(L.head_norm(k, gk, EPS)[0], c.at, c.freqs64, 1.0, True) * f64(c.rows(dka))).sum()
    args = [f64(t) for t in (c.q, c.k, *c.gains)]
    grads = [f64(dq), f64(dk), f64(dgains[0]) - f64(was[0]), f64(dgains[1]) - f64(was[1])]
    for i, g in enumerate(grads):
        way = c.rng.normal(size=g.shape)
        step = [a + 1e-5 * way if j == i else a for j, a in enumerate(args)], [a - 1e-5 * way if j == i else a for j, a in enumerate(args)]
        slope = (value(*step[0]) - value(*step[1])) / 2e-5
        # fp32 values of about 1 each, sums of fewer than 400; the difference itself leaves 1e-9
        assert abs(slope - (g * way).sum()) <= 1e-4 * (1 + np.abs(g * way).sum())


def test_offsets_past_32_bits():
    """Heads and caches further apart than 2^31 elements, and a far segment of a long cache."""
    c = Call((2, 2, 2, 3, 128, 128, "dense", "dense"), "bf16", False, True, False)
    near = c.forward()
    big = torch.empty(2 ** 31 + 2 ** 20, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((2, 2, 3, 128), (2 ** 31, 2 ** 18, 128, 1))
    far.copy_(c.q)
    q_rot = torch.empty_like(near[0])
    kc = torch.empty((2, 2, 2 ** 22 + 8, 128), dtype=torch.bfloat16, device="cuda")
    at = 2 ** 22
    s1f.qk_norm_rope_fwd(far, c.k, c.v, *c.gains, 1e-6, *c.turn[:4], at, q_rot, kc, torch.empty_like(kc))
    assert torch.equal(q_rot, near[0]) and torch.equal(kc[:, :, at:at + 3], c.rows(near[1]))


def test_takes_the_place_of_append_and_emit():
    """Without a rotation the calls are kv_append and kv_grad_emit."""
    c = Call((2, 4, 2, 50, 64, 0, "dense", "dense"), "bf16", False, False, False)
    q_rot, kc, vc = c.forward()
    kc2, vc2 = torch.full_like(kc, 333.0), torch.full_like(vc, 333.0)
    s1f.kv_append(c.k, c.v, c.off, kc2, vc2)
    assert torch.equal(kc, kc2) and torch.equal(vc, vc2) and torch.equal(q_rot, c.q)
    _, dka, dva, _, dk, dv, _, _ = c.backward()
    dk2, dv2 = torch.empty_like(dk), torch.empty_like(dv)
    s1f.kv_grad_emit(dka, dva, c.off, dk2, dv2)
    assert torch.equal(dk, dk2) and torch.equal(dv, dv2)
