"""The gated feed-forward block and its gradient as a whole, by blocks of 32 x 32, by rows and by columns, in every kind of tile and cut: a lost stage, part or plane of products shows (test_layer_spread.py),
which the bounds for single elements of test_gpu_ffn.py are too wide for."""
import pytest
import torch

import layer_spread as S
import paper_2406_03488_amd as s1f
from ends_harness import TYPES, space, untouched
from test_gpu_ffn import ACTS
from test_host_layer_launches import SHAPES

pytestmark = pytest.mark.gpu

# (test_host_layer_launches.py: these take tiles of every size for every product, their rests in quarters or in parts; dW in turns)
CASES = [(*shape, dtype) for shape, dtypes in SHAPES for dtype in dtypes]
# the kernel of few rows, of up to 16, 32 and 64
CASES += [(n, h, f, dtype) for n, h, f in ((1, 1032, 2500), (16, 520, 1400), (13, 4096, 11008), (30, 520, 1400), (57, 520, 1400), (64, 193, 331)) for dtype in (0, 1)]
# fp32 sums of y and dx in turns, in tiles of every size, in parts and not; turns that do not end a stage
TURNS = [(65, 8192, 26000), (300, 2048, 26001), (2000, 640, 33333), (8200, 1100, 14001), (4400, 4096, 13000), (16384, 1024, 13000)]
CASES += [(*shape, 0) for shape in TURNS]
CASES += [(512, 4096, 11008, 0), (512, 4096, 11008, 1), (1000, 2048, 5632, 1), (4099, 4096, 11008, 0)]


@pytest.mark.parametrize("n,h,f,dtype", CASES)
def test_block_and_gradient_as_a_whole(n, h, f, dtype):
    dtype = ("f32", "bf16")[dtype]
    act = ("silu", "gelu_tanh", "gelu")[(n + h + f) % 3]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n + h + f)
    normal = lambda *shape, scale=1.0: torch.empty(shape, device="cuda", dtype=TYPES[dtype]).normal_(0, scale, generator=gen)
    x, dy, w_in, w_out = normal(1, n, h), normal(1, n, h), normal(2 * f, h, scale=1.5 * h ** -0.5), normal(h, f, scale=f ** -0.5)
    y, dx, gate_up = torch.full_like(x, float("nan")), torch.full_like(x, float("nan")), torch.full((1, n, 2 * f), float("nan"), device="cuda", dtype=x.dtype)
    size = s1f.gated_ffn_fwd_workspace_bytes(x, w_in, w_out)
    ws, buffer = space(size)
    s1f.gated_ffn_fwd(x, w_in, w_out, ACTS[act], y, gate_up, ws)
    assert untouched(buffer, size)
    x64, dy64, wi, wo, gu = (t.double() for t in (x[0], dy[0], w_in, w_out, gate_up[0]))
    expected = S.forward(x64, wi, wo, act, dtype)
    S.near(gate_up[0], expected["gate_up"], "gate_up")
    S.near(y[0], expected["y"], "y")
    del expected
    size = s1f.gated_ffn_bwd_workspace_bytes(dy, x, w_in, w_out)
    ws, buffer = space(size)
    start = [torch.empty(w.shape, device="cuda").normal_(0, 1, generator=gen) for w in (w_in, w_out)]
    for into in ("f32", "bf16") if dtype == "bf16" else ("f32",):
        dw = [t.clone() for t in start] if into == "f32" else [torch.full_like(w, float("nan")) for w in (w_in, w_out)]
        s1f.gated_ffn_bwd(dy, x, w_in, w_out, ACTS[act], gate_up, dx.fill_(float("nan")), *dw, ws)
        assert untouched(buffer, size)
        expected = S.backward(dy64, x64, wi, wo, act, gu, dtype, S.HALF[into])
        S.near(dx[0], expected["dx"], "dx")
        for name, got, was in zip(("dw_in", "dw_out"), dw, start):
            S.near(got, expected[name], name, was.double() if into == "f32" else None)


def test_sums_of_weights_gradients_over_many_rows():
    """fp32, 131072 rows of values of one sign: sums of up to 12288 terms, and their sums; one sum of all would be four times as far off, or more."""
    n, h, f = 131072, 40, 24
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    normal = lambda *shape: torch.empty(shape, device="cuda").normal_(0, 1, generator=gen)
    x, dy, gate_up = normal(1, n, h).abs_(), normal(1, n, h).abs_(), 1 + 0.2 * normal(1, n, 2 * f)
    w_in, w_out = normal(2 * f, h), normal(h, f).abs_()
    dx, dw = torch.empty_like(x), [torch.zeros_like(w_in), torch.zeros_like(w_out)]
    ws = space(s1f.gated_ffn_bwd_workspace_bytes(dy, x, w_in, w_out))[0]
    s1f.gated_ffn_bwd(dy, x, w_in, w_out, s1f.SILU, gate_up, dx, *dw, ws)
    expected = S.backward(*(t.double() for t in (dy[0], x[0], w_in, w_out)), "silu", gate_up[0].double(), "f32", S.U)
    for name, got in (("dx", dx[0]), ("dw_in", dw[0]), ("dw_out", dw[1])):
        S.near(got, expected[name], name)
