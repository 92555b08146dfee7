"""The token loss's products element by element, in calls of every instance of its kernels and every way they are cut (exact_products.py): whole numbers have to be
equal, single products of full operands right to the roundings of one."""
import pytest
import torch

import paper_2406_03488_amd as s1f
from ends_harness import row_values, space, untouched
from exact_products import LONG, ONE_PRODUCT, PIECES, SHAPES, TYPES, WHOLE, backward_case, scores_case

pytestmark = pytest.mark.gpu


def check(kind, n, h, v, dtype, into, blank=0.0, seed=0):
    """into: type of dweight.  fp32: added to what is there."""
    x, w, t, lse, g, dx, dw = (a.cuda() for a in backward_case(kind, n, h, v, dtype, blank, seed))
    got_dx = torch.full_like(x, float("nan"))
    start = torch.zeros((v, h), device="cuda") if kind == "one" else torch.arange(v, device="cuda").remainder(7).float()[:, None].expand(v, h).contiguous()
    got_dw = start.clone() if into == "f32" else torch.full((v, h), float("nan"), dtype=TYPES[into], device="cuda")
    size = s1f.token_loss_bwd_workspace_bytes(x, w)
    ws, buffer = space(size)
    s1f.token_loss_bwd(g, x, w, t, lse, got_dx, got_dw, ws)
    assert untouched(buffer, size)
    want_dw = dw + start.double() if into == "f32" else dw
    for what, got, want in (("dx", got_dx[0], dx), ("dweight", got_dw, want_dw)):
        if kind == "one" and dtype == "f32":
            off = (got.double() - want).abs() - ONE_PRODUCT * want.abs()
            bad = ~(off <= 0)
        else:
            bad = got != want.to(torch.float32).to(got.dtype)      # (exact in fp32: rounded once)
        assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} elements are wrong, the first at {torch.nonzero(bad)[0].tolist()}"


KINDS = ["one", "all dx", "all dw", "some"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("types", ["f32 f32", "bf16 f32", "bf16 bf16"])
@pytest.mark.parametrize("n,h,v", SHAPES + WHOLE)
def test_gradient(n, h, v, types, kind):
    check(kind, n, h, v, *types.split())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("types", ["f32 f32", "bf16 f32", "bf16 bf16"])
def test_gradient_over_several_pieces(types, kind):
    dtype, into = types.split()
    check(kind, *PIECES[dtype], dtype, into)


@pytest.mark.parametrize("kind", ["one", "all dx", "some"])
@pytest.mark.parametrize("types", ["f32 f32", "bf16 bf16"])
@pytest.mark.parametrize("blank", [0.5, 0.95, 1.0])
@pytest.mark.parametrize("n,h,v", WHOLE + [(1040, 512, 16384), (2304, 8192, 2304), (700, 264, 9001)])
def test_gradient_of_fewer_rows(n, h, v, blank, types, kind):
    """Most rows out, behind whole rounds of tiles and where all are in parts."""
    check(kind, n, h, v, *types.split(), blank=blank, seed=1)


@pytest.mark.parametrize("kind", ["one", "all dw", "some"])
@pytest.mark.parametrize("blank", [0.0, 0.5, 0.95, 1.0])
@pytest.mark.parametrize("n,h,v", LONG)
def test_gradient_of_many_rows(n, h, v, blank, kind):
    """dweight's sums in parts of about 8192 rows that count."""
    check(kind, n, h, v, "f32", "f32", blank=blank, seed=2)


@pytest.mark.parametrize("kind", ["all dx", "all dw", "some"])
@pytest.mark.parametrize("v", [171, 200, 255, 300])
def test_gradient_of_as_many_rows_as_there_may_be(v, kind):
    """A piece of the vocabulary has 256 tokens then, or all that there are."""
    check(kind, 1 << 20, 8, v, "f32", "f32", blank=0.3, seed=4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_calls_at_once(dtype):
    """On two streams, each with a workspace of its own, and captured into one graph as two branches of it that are replayed with other targets."""
    n, h, v = 9000, 72, 700
    calls = []
    for seed in (5, 6):
        x, w, t, lse, g, *_ = (a.cuda() for a in backward_case("some", n, h, v, dtype, 0.2, seed))
        ws = torch.empty(max(s1f.token_loss_bwd_workspace_bytes(x, w), s1f.token_loss_fwd_workspace_bytes(x, w)), dtype=torch.uint8, device="cuda")
        calls.append((x, w, t, lse, g, torch.empty_like(x), torch.zeros((v, h), device="cuda"), row_values(1, n), row_values(1, n), ws))

    def run(x, w, t, lse, g, dx, dw, loss, made, ws):
        dw.zero_()
        s1f.token_loss_fwd(x, w, t, loss, made, ws)
        s1f.token_loss_bwd(g, x, w, t, lse, dx, dw, ws)

    outputs = lambda: [a.clone() for c in calls for a in c[5:9]]
    sides = [torch.cuda.Stream() for _ in calls]

    def both():
        here = torch.cuda.current_stream()
        for side, c in zip(sides, calls):
            side.wait_stream(here)
            with torch.cuda.stream(side):
                run(*c)
        for side in sides:
            here.wait_stream(side)

    for c in calls:
        run(*c)
    want = outputs()
    both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for turn in range(3):
        for c in calls:
            c[2].copy_(torch.where(torch.rand(c[2].shape, device="cuda") < 0.3 * turn, -1, torch.randint(0, v, c[2].shape, device="cuda")))
            run(*c)
        want = outputs()
        for c in calls:
            for a in c[5:9]:
                a.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want)), turn


def test_long_sums_keep_their_bits():
    """dweight of 49152 fp32 rows over 300 tokens, relative to its norm: 1.5e-6 off with the library's products of 32-bit scores.  One sum over all rows, six products for each, was 2.6e-6 off.  Roundings
    are of either sign and follow the size of the sum so far: in six parts their squares are a sixth, 1.1e-6."""
    rng = torch.Generator(device="cuda").manual_seed(3)
    n, h, v = 49152, 64, 300
    x, w = torch.randn((1, n, h), device="cuda", generator=rng), torch.randn((v, h), device="cuda", generator=rng) * (2 / h ** 0.5)
    t = torch.randint(0, v, (1, n), device="cuda", generator=rng)
    z = x[0].double() @ w.double().T
    lse = torch.logsumexp(z, 1)[None].float()
    g = (torch.rand((1, n), device="cuda", generator=rng) + 0.5) / n
    dz = (z - lse[0].double()[:, None]).exp()
    dz[torch.arange(n, device="cuda"), t[0]] -= 1
    want = (dz * g[0].double()[:, None]).T @ x[0].double()
    dx, dw = torch.empty_like(x), torch.zeros((v, h), device="cuda")
    s1f.token_loss_bwd(g, x, w, t, lse, dx, dw, space(s1f.token_loss_bwd_workspace_bytes(x, w))[0])
    assert (dw.double() - want).norm() <= 1.5e-6 * want.norm()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,h,v", SHAPES + WHOLE)
def test_scores(n, h, v, dtype):
    x, w, t, want = (a.cuda() for a in scores_case(n, h, v, dtype))
    loss, lse = row_values(1, n), row_values(1, n)
    size = s1f.token_loss_fwd_workspace_bytes(x, w)
    ws, buffer = space(size)
    s1f.token_loss_fwd(x, w, t, loss, lse, ws)
    assert untouched(buffer, size)
    assert (loss == 0).all()
    assert ((lse[0].double() - want).abs() <= (ONE_PRODUCT if dtype == "f32" else 0) * want).all()
