"""Calls around a layer's attention that gave wrong results: against 64 bits, or against the calls that gave right ones."""
import numpy as np
import pytest
import torch

import paper_2406_03488_amd as s1f
import layer_spread as S
from layer_harness import like
from test_gpu_ffn import ACTS, Block
from test_gpu_rope import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_past_2_to_50(interleaved):
    """Angles whose quarter turns are too many to be counted in 64 bits to a fraction of one: what is left of them was up to 500, and results 10^18 times as large as their heads."""
    n = 48
    c = Call((1, 2, 1, n, 16, 16, "dense", "dense"), "f32", interleaved, False, True)
    at = np.array([[sign * ((1 << 46 + i // 3) + 12345 * i + 1) for i in range(n) for sign in (1, -1)][:n]], dtype=np.int64)
    assert at.max() > 1 << 52
    at[0, -4:] = (1 << 62) + 977, -(1 << 62) - 1, (1 << 63) - 1, -(1 << 63)
    freqs = np.array([1.0, 0.7, 3.0, 1e-3, 2.0 ** -10, 40.0, 2.0 ** 14, 1e-12])
    c.at, c.positions = at, torch.from_numpy(at).cuda()
    c.freqs64, c.freqs = freqs, torch.from_numpy(freqs).cuda()
    c.turn = (c.freqs, 1.0, interleaved, c.positions, c.off)
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(1, 9, 64, 96, "dense", "dense", "silu"), (1, 300, 640, 1000, "dense", "dense", "silu"), (2, 150, 136, 1001, "view", "view", "gelu_tanh"),
                                  (1, 2100, 512, 264, "dense", "dense", "gelu")])
def test_block_in_the_place_of_its_rows(case, dtype):
    """y may be x, and dx x or dy; the weights' gradients read both."""
    c = Block(case, dtype)
    y, gate_up = c.forward()
    kind = "f32" if dtype == "f32" else "bf16"
    zeros = [torch.zeros_like(w, dtype=torch.float32) for w in (c.w_in, c.w_out)]
    want = c.backward(gate_up, kind, zeros)
    space_of = lambda f, *rows: torch.empty(f(*rows, c.w_in, c.w_out), dtype=torch.uint8, device="cuda")
    x = like(c.x).copy_(c.x)
    s1f.gated_ffn_fwd(x, c.w_in, c.w_out, ACTS[c.act], x, None, space_of(s1f.gated_ffn_fwd_workspace_bytes, x))
    assert torch.equal(x, y)
    for place in ("x", "dy"):
        x, dy = like(c.x).copy_(c.x), like(c.x).copy_(c.dy)
        dx, dw = (x if place == "x" else dy), [torch.zeros_like(t) for t in want[1:]]
        s1f.gated_ffn_bwd(dy, x, c.w_in, c.w_out, ACTS[c.act], gate_up, dx, *dw, space_of(s1f.gated_ffn_bwd_workspace_bytes, dy, x))
        assert torch.equal(dx, want[0]) and all(torch.equal(a, b) for a, b in zip(dw, want[1:])), place


def test_long_fp32_sums_between_the_projections():
    """y's sums of 65536 terms and dx's of 131072, in as many tiles as there are compute units: in one sum each y is 4.3e-6 of its norm off."""
    n, h, f = 16384, 1024, 65536
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    normal = lambda *shape, scale=1.0: torch.empty(shape, device="cuda").normal_(0, scale, generator=gen)
    x, dy, w_in, w_out = normal(1, n, h), normal(1, n, h), normal(2 * f, h, scale=h ** -0.5), normal(h, f, scale=f ** -0.5)
    y, dx, gate_up = torch.empty_like(x), torch.empty_like(x), torch.empty((1, n, 2 * f), device="cuda")
    ws = torch.empty(s1f.gated_ffn_bwd_workspace_bytes(dy, x, w_in, w_out), dtype=torch.uint8, device="cuda")
    assert s1f.gated_ffn_fwd_workspace_bytes(x, w_in, w_out) <= len(ws)
    s1f.gated_ffn_fwd(x, w_in, w_out, s1f.SILU, y, gate_up, ws)
    dw = torch.zeros_like(w_in), torch.zeros_like(w_out)
    s1f.gated_ffn_bwd(dy, x, w_in, w_out, s1f.SILU, gate_up, dx, *dw, ws)
    rows = torch.randint(0, n, (128,), device="cuda", generator=gen)
    xs, ys, wi, wo = (t.double() for t in (x[0, rows], dy[0, rows], w_in, w_out))
    S.near(y[0, rows], S.forward(xs, wi, wo, "silu", "f32")["y"], "y")
    S.near(dx[0, rows], S.backward(ys, xs, wi, wo, "silu", gate_up[0, rows].double(), "f32", S.U)["dx"], "dx")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [12, 517])
def test_block_in_part_of_the_place_of_its_inputs(n, dtype):
    """y some rows behind x, dx some rows behind x or dy, or in gate_up."""
    c = Block((1, n, 128, 264, "dense", "dense", "silu"), dtype)
    y, gate_up = c.forward()
    start = c.start()
    want = c.backward(gate_up, "f32", start)
    ws = torch.empty(max(s1f.gated_ffn_fwd_workspace_bytes(c.x, c.w_in, c.w_out), s1f.gated_ffn_bwd_workspace_bytes(c.dy, c.x, c.w_in, c.w_out)), dtype=torch.uint8, device="cuda")

    def shifted(t):
        rows = torch.zeros((1, n + 5, 128), dtype=t.dtype, device="cuda")
        rows[:, :n] = t
        return rows[:, :n], rows[:, 5:]
    x, to = shifted(c.x)
    s1f.gated_ffn_fwd(x, c.w_in, c.w_out, s1f.SILU, to, None, ws)
    assert torch.equal(to, y)
    for place in ("x", "dy", "gate_up"):
        x, dy, kept = c.x, c.dy, gate_up.clone()
        if place == "x":
            x, dx = shifted(x)
        elif place == "dy":
            dy, dx = shifted(dy)
        else:
            dx = kept.view(-1)[:n * 128].view(1, n, 128)
        dw = [t.clone() for t in start]
        s1f.gated_ffn_bwd(dy, x, c.w_in, c.w_out, s1f.SILU, kept, dx, *dw, ws)
        assert torch.equal(dx, want[0]) and all(torch.equal(a, b) for a, b in zip(dw, want[1:])), place


def test_turns_in_a_graph():
    """fp32 sums in turns, captured and replayed with new inputs: the first turn writes, whatever the replay before has left."""
    n, h, f = 65, 8192, 26000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    normal = lambda *shape, scale=1.0: torch.empty(shape, device="cuda").normal_(0, scale, generator=gen)
    x, dy, w_in, w_out = normal(1, n, h), normal(1, n, h), normal(2 * f, h, scale=h ** -0.5), normal(h, f, scale=f ** -0.5)
    y, dx, gate_up, dw = torch.empty_like(x), torch.empty_like(x), torch.empty((1, n, 2 * f), device="cuda"), [torch.zeros_like(w_in), torch.zeros_like(w_out)]
    ws = torch.empty(s1f.gated_ffn_bwd_workspace_bytes(dy, x, w_in, w_out), dtype=torch.uint8, device="cuda")
    ws_fwd = torch.empty(s1f.gated_ffn_fwd_workspace_bytes(x, w_in, w_out), dtype=torch.uint8, device="cuda")

    def run():
        s1f.gated_ffn_fwd(x, w_in, w_out, s1f.SILU, y, gate_up, ws_fwd)
        s1f.gated_ffn_bwd(dy, x, w_in, w_out, s1f.SILU, gate_up, dx, *dw, ws)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        x.normal_(0, 1, generator=gen)
        run()
        want = y.clone(), dx.clone()
        y.fill_(float("nan")), dx.fill_(float("nan"))
        graph.replay()
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1])
        torch.cuda.synchronize()
