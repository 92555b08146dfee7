"""Which instances of the token loss's kernels the shapes of exact_products.py run, and what its expected values tell apart.  No device."""
import os
import re
import subprocess
import sys

import numpy as np
import pytest

from exact_products import LONG, ONE_PRODUCT, PIECES, SHAPES, WHOLE, backward_case, scores_case
from oracle import ends as E
from test_host_fp32_planes import SIX, product

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
import paper_2406_03488_amd as s1f
from paper_2406_03488_amd.binding import Rows
lib = s1f.load_library()
p, big = 4096, 1 << 45   # (no address is looked at)
for n, h, v, dtype, written in eval(sys.argv[2]):
    d = ctypes.byref(Rows(1, h, dtype, 0, n, 0, h, 0, h))
    assert lib.s1f_token_loss_fwd(d, p, p, h, v, p, 0, p, p, p, big, None) == 0
    assert lib.s1f_token_loss_bwd(d, p, p, p, h, v, p, 0, p, p, p, h, written, p, big, None) == 0
"""


def launches(tmp_path, shapes):
    """[(kernel's name and template arguments, workgroups)] of a forward and a backward of each (rows, hidden, vocabulary, dtype, type of dweight)."""
    so, record = str(tmp_path / "recording.so"), str(tmp_path / "record")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-o", so, os.path.join(ROOT, "tests", "recording_runtime.c")], check=True)
    run = subprocess.run([sys.executable, "-c", DRIVER, so, repr(shapes)], env=dict(os.environ, RECORD=record, PYTHONPATH=ROOT), capture_output=True, text=True, cwd=ROOT)
    assert run.returncode == 0, run.stderr
    lines = [line.split() for line in open(record) if line.startswith("launch") and "loss_" in line]
    return [(name.split("loss_", 1)[1], int(grid)) for _, name, grid, *_ in lines]


def products_of(tmp_path, shapes):
    return {name for name, _ in launches(tmp_path, shapes) if name.startswith(("scores", "dx_kernel", "dw_kernel"))}


def instances(names, what):
    """{(rows of a tile, columns, last template argument if it is a truth value)}"""
    return {re.search(r"Li(\d+)ELi(\d+)ELi\dELi\dE(?:Lb([01])E)?", x).groups() for x in names if x.startswith(what)}


def test_every_instance_is_run(tmp_path):
    """By shapes that the GPU tests check element by element: all sizes of tiles of each product, both types, both directions, dweight added (1) and written (0)."""
    for dtype, code in (("f32", 0), ("bf16", 1)):
        done = products_of(tmp_path, [(*s, code, written) for s in SHAPES + WHOLE + [PIECES[dtype]] for written in ((0, 1) if code else (0,))])
        tiles = [("256", "256"), ("128", "128")]
        assert instances(done, "scores") == {(*t, forward) for t in tiles + [("64", "128")] for forward in "01"}
        assert instances(done, "dx_kernel") == {(*t, None) for t in tiles}
        assert instances(done, "dw_kernel") == {(*t, add) for t in tiles for add in ("01" if code else "1")}


@pytest.mark.parametrize("code", [0, 1])
def test_whole_rounds_of_dx(tmp_path, code):
    """256 big tiles that nothing cuts: behind them a rest in parts, or none."""
    dx = [grid for s in WHOLE for name, grid in launches(tmp_path, [(*s, code, 0)]) if name.startswith("dx_kernel")]
    assert dx[0] > 256 and (dx[0] - 256) % 32 == 0 and dx[1] == 256


@pytest.mark.parametrize("shape,tile", zip(LONG, (128, 256)))
def test_long_sums_are_cut(tmp_path, shape, tile):
    """dweight of 12288 fp32 rows and more: as many workgroups for a tile as there are parts, and a join; of fewer, and of bf16 rows, one for a tile."""
    n, h, v = shape
    done = [(name, grid) for name, grid in launches(tmp_path, [(*shape, 0, 0)]) if name.startswith("dw")]
    assert len(done) == 2 and f"Li{tile}ELi{tile}" in done[0][0] and done[1][0].startswith("dw_join")
    assert done[0][1] == -(-v // tile) * -(-h // tile) * ((n + 4096) // 8192) and done[1][1] == -(-v * (h // 4) // 256)
    assert not any(name.startswith("dw_join") for name, _ in launches(tmp_path, [(12287, h, v, 0, 0), (n, h, v, 1, 0), (n, h, v, 1, 1)]))


@pytest.mark.parametrize("dtype,code", [("f32", 0), ("bf16", 1)])
def test_pieces(tmp_path, dtype, code):
    n = sum(name.startswith("dx_kernel") for name, _ in launches(tmp_path, [(*PIECES[dtype], code, 0)]))
    assert n == 2


@pytest.mark.parametrize("kind", ["one", "all dx", "all dw", "some"])
@pytest.mark.parametrize("n,h,v,blank", [(40, 12, 30, 0.0), (33, 7, 90, 0.4)])
def test_expected_gradients(kind, n, h, v, blank):
    """Against the oracle.  (Exponentials that are 2^-288 and less are 0 in fp32.)"""
    x, w, t, lse, g, dx, dw = backward_case(kind, n, h, v, "f32", blank)
    want_dx, want_dw, _, rows = E.token_loss_grad(g[0].double().numpy(), x[0].double().numpy(), w.double().numpy(), t[0].numpy(), lse[0].double().numpy())
    assert len(rows) == int((t >= 0).sum()) and (blank == 0 or len(rows) < n)
    assert np.abs(dx.numpy() - want_dx).max() <= 1e-12 * np.abs(want_dx).max() and np.abs(dw.numpy() - want_dw).max() <= 1e-12 * max(1.0, np.abs(want_dw).max())
    if kind != "one":
        assert all((t == t.round()).all() and t.abs().max() < 2 ** 24 for t in (dx, dw))


@pytest.mark.parametrize("n,h,v", [(40, 12, 30), (20, 64, 33)])
def test_expected_scores(n, h, v):
    x, w, t, lse = scores_case(n, h, v, "f32")
    loss, want = E.token_loss(x[0].double().numpy(), w.double().numpy(), t[0].numpy())
    assert np.abs(lse.numpy() - want).max() <= 1e-12 * want.max() and loss.max() <= 1e-12


def test_sums_stay_whole_in_fp32():
    """Whatever the order: fewer than 2^24 / 400 terms of at most 400, or 2^24 / 6 of at most 6."""
    for n, h, v in SHAPES + WHOLE + LONG + list(PIECES.values()):
        assert 6 * max(n, v) < 2 ** 24 and 400 * max(v / h * 2 + 200, n / h * 2 + 200) < 2 ** 24


@pytest.mark.parametrize("n,h,v", [s for s in SHAPES if s[1] <= 2000])
def test_a_product_of_planes_that_is_missing_shows(n, h, v):
    """In the scores, in dx and in dweight, at the tolerance that the GPU tests have for one product; with all six nothing does."""
    x, w, t, lse, g, dx, dw = backward_case("one", n, h, v, "f32")
    on = np.nonzero(g[0].numpy())[0][:512]
    at = t[0].numpy()[on]
    xs, ws, ts, _ = scores_case(n, h, v, "f32")
    hot = xs[0].abs().argmax(1).numpy()
    calls = [(xs[0].numpy()[np.arange(n), hot], ws.numpy()[ts[0].numpy(), hot]), (-g[0].numpy()[on][:, None], w.numpy()[at]), (-g[0].numpy()[on][:, None], x[0].numpy()[on])]
    for a, b in calls:
        want = a.astype(np.float64) * b
        relative = lambda products: np.abs(product(a, b, products) / want - 1).max()
        assert relative(SIX) <= ONE_PRODUCT
        if a.size * b.size >= 1000:
            for out in SIX:
                assert relative([p for p in SIX if p != out]) > 2 * ONE_PRODUCT, out
                assert relative(SIX + [out]) > 2 * ONE_PRODUCT, out
