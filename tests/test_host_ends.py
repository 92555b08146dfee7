"""What the calls of embedding, layer norm and token loss refuse: the C entry points before anything is launched, and their Python forms before the
library is called.  No device."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

import paper_2406_03488_amd as s1f
from paper_2406_03488_amd import binding
from paper_2406_03488_amd.binding import Rows

P, ODD, OFF = 4096, 4097, 4104     # addresses: aligned, not even, on 8 bytes (none is looked at)
BIG = 1 << 50


def rows(**kw):
    base = dict(batch=2, hidden=64, dtype=1, reserved=0, rows=5, x_stride_b=320, x_stride_s=64, y_stride_b=320, y_stride_s=64)
    base.update(kw)
    return Rows(**base)


def embed_fwd(d, ids=P, table=P, stride=64, vocab=10, out=P):
    return s1f.load_library().s1f_embed_fwd(ctypes.byref(d) if d else None, ids, 5, table, stride, vocab, 1.0, out, None)


def embed_bwd(d, ids=P, dout=P, vocab=10, acc=P, stride=64, ws=P, n=BIG):
    return s1f.load_library().s1f_embed_bwd(ctypes.byref(d) if d else None, ids, 5, dout, vocab, 1.0, acc, stride, ws, n, None)


def norm_fwd(d, x=P, gamma=P, beta=P, eps=1e-5, y=P, mean=P, rstd=P):
    return s1f.load_library().s1f_layer_norm_fwd(ctypes.byref(d) if d else None, x, gamma, beta, eps, y, mean, rstd, None)


def norm_bwd(d, dy=P, x=P, gamma=P, mean=P, rstd=P, dx=P, dg=P, db=P, ws=P, n=BIG):
    return s1f.load_library().s1f_layer_norm_bwd(ctypes.byref(d) if d else None, dy, x, gamma, mean, rstd, dx, dg, db, ws, n, None)


def loss_fwd(d, x=P, weight=P, stride=64, vocab=10, targets=P, loss=P, lse=P, ws=P, n=BIG):
    return s1f.load_library().s1f_token_loss_fwd(ctypes.byref(d) if d else None, x, weight, stride, vocab, targets, 5, loss, lse, ws, n, None)


def loss_bwd(d, dloss=P, x=P, weight=P, stride=64, vocab=10, targets=P, lse=P, dx=P, dw=P, into=64, code=0, ws=P, n=BIG):
    return s1f.load_library().s1f_token_loss_bwd(ctypes.byref(d) if d else None, dloss, x, weight, stride, vocab, targets, 5, lse, dx, dw, into, code,
                                                 ws, n, None)


CALLS = {embed_fwd: "y", embed_bwd: "y", norm_fwd: "xy", norm_bwd: "xy", loss_fwd: "x", loss_bwd: "x"}


@pytest.mark.parametrize("call", CALLS)
def test_descriptors_refused(call):
    assert call(None) == 1
    for bad in (dict(batch=0), dict(batch=-1), dict(hidden=0), dict(reserved=1)):
        assert call(rows(**bad)) == 1, bad
    for bad in (dict(dtype=2), dict(dtype=-1), dict(hidden=16385), dict(rows=(1 << 21) + 1), dict(batch=1 << 20, rows=1 << 20),
                dict(batch=1 << 30, rows=1 << 34)):
        h = bad.get("hidden", 64)
        d = rows(**{"x_stride_s": h, "y_stride_s": h, "x_stride_b": 1 << 40, "y_stride_b": 1 << 40, **bad})
        kw = {} if call in (norm_fwd, norm_bwd) else {"stride": h}
        assert call(d, **kw) == 2, bad
    for bad in (0, -1, -(1 << 40)):
        assert call(rows(rows=bad)) == 3
    for side in CALLS[call]:
        for bad in ({f"{side}_stride_s": 63}, {f"{side}_stride_s": -64}, {f"{side}_stride_b": 63}):
            assert call(rows(**bad)) == 1, bad


@pytest.mark.parametrize("call", CALLS)
def test_pointers_and_sizes_refused(call):
    """Whatever is checked last would be launched here, where there is no device: every call has to end before."""
    names = {embed_fwd: ("ids", "table", "out"), embed_bwd: ("ids", "dout", "acc", "ws"), norm_fwd: ("x", "gamma", "beta", "y", "mean", "rstd"),
             norm_bwd: ("dy", "x", "gamma", "mean", "rstd", "dx", "dg", "db", "ws"), loss_fwd: ("x", "weight", "targets", "loss", "lse", "ws"),
             loss_bwd: ("dloss", "x", "weight", "targets", "lse", "dx", "dw", "ws")}[call]
    for name in names:
        assert call(rows(), **{name: None}) == 1, name
        assert call(rows(), **{name: ODD}) == 1, name
    if "ws" in names:
        assert call(rows(), ws=OFF) == 1 and call(rows(), n=255) == 1 and call(rows(), n=0) == 1
    if call in (embed_fwd, loss_fwd, loss_bwd):
        assert call(rows(), stride=63) == 1
    if call not in (norm_fwd, norm_bwd):
        assert call(rows(), vocab=0) == 1 and call(rows(), vocab=-5) == 1
        assert call(rows(), vocab=(1 << 26) + 1) == 2
    if call is norm_fwd:
        assert call(rows(), eps=-1e-9) == 1 and call(rows(), eps=float("nan")) == 1
    if call in (loss_fwd, loss_bwd):
        assert call(rows(), weight=OFF) == 1
        assert call(rows(), vocab=(1 << 24) + 1) == 2 and call(rows(), stride=1 << 22) == 2
        assert call(rows(batch=1, rows=(1 << 20) + 1)) == 2
        assert call(rows(batch=1, rows=1 << 20, hidden=8200, x_stride_s=8200), stride=8200) == 2
    if call is loss_bwd:
        assert call(rows(), into=63) == 1 and call(rows(), code=2) == 2 and call(rows(dtype=0), code=1) == 2


def test_workspace_sizes():
    lib = s1f.load_library()
    ask = lambda f, d, *a: f(ctypes.byref(d) if d else None, *a)
    queries = [(lib.s1f_embed_bwd_workspace_bytes, (10,)), (lib.s1f_layer_norm_bwd_workspace_bytes, ()),
               (lib.s1f_token_loss_fwd_workspace_bytes, (10, 64)), (lib.s1f_token_loss_bwd_workspace_bytes, (10, 64))]
    for f, a in queries:
        assert ask(f, rows(), *a) > 0
        assert ask(f, None, *a) == 0 and ask(f, rows(rows=0), *a) == 0 and ask(f, rows(hidden=0), *a) == 0 and ask(f, rows(dtype=5), *a) == 0
    # scores never exist as a whole: a piece of them is at most 1 GiB, however many there are
    d = rows(batch=1, rows=1 << 17, hidden=1024, x_stride_s=1024, x_stride_b=0)
    fwd, bwd = ask(lib.s1f_token_loss_fwd_workspace_bytes, d, 200000, 1024), ask(lib.s1f_token_loss_bwd_workspace_bytes, d, 200000, 1024)
    assert fwd < 4 << 30 and bwd < 12 << 30


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or 0


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "_stream_ptr", lambda: 0)
    monkeypatch.setattr(binding, "_check_device", lambda *t: None)
    monkeypatch.setattr(binding, "_native", lambda: binding._PythonForms)
    return lib


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def f32(*shape):
    return torch.zeros(shape)


def ids(*shape):
    return torch.zeros(shape, dtype=torch.int64)


def good():
    """Arguments of every call, by name; all of them fit."""
    x, ws = bf16(2, 5, 16), torch.zeros(64, dtype=torch.uint8)
    return {"embed_fwd": [ids(2, 5), bf16(9, 16), 1.0, x], "embed_bwd": [ids(2, 5), x, 1.0, f32(9, 16), ws],
            "layer_norm_fwd": [x, bf16(16), bf16(16), 1e-5, bf16(2, 5, 16), f32(2, 5), f32(2, 5)],
            "layer_norm_bwd": [bf16(2, 5, 16), x, bf16(16), f32(2, 5), f32(2, 5), bf16(2, 5, 16), f32(16), f32(16), ws],
            "token_loss_fwd": [x, bf16(9, 16), ids(2, 5), f32(2, 5), f32(2, 5), ws],
            "token_loss_bwd": [f32(2, 5), x, bf16(9, 16), ids(2, 5), f32(2, 5), bf16(2, 5, 16), f32(9, 16), ws]}


def test_good_calls_reach_the_library(library):
    for name, args in good().items():
        getattr(s1f, name)(*args)
        assert library.calls.pop() == "s1f_" + name and not library.calls


BAD = [("embed_fwd", 0, ids(2, 4)), ("embed_fwd", 0, ids(5)), ("embed_fwd", 0, ids(2, 10)[:, ::2]), ("embed_fwd", 0, ids(2, 5).int()),
       ("embed_fwd", 1, bf16(9, 8)), ("embed_fwd", 1, f32(9, 16)), ("embed_fwd", 1, bf16(16, 9).t()), ("embed_fwd", 3, bf16(2, 5, 32)[..., ::2]),
       ("embed_fwd", 3, bf16(5, 16)), ("embed_fwd", 3, bf16(2, 5, 16).half()), ("embed_bwd", 3, bf16(9, 16)), ("embed_bwd", 3, f32(9, 8)),
       ("embed_bwd", 0, ids(3, 5)), ("embed_bwd", 4, torch.zeros(128, dtype=torch.uint8)[::2]),
       ("layer_norm_fwd", 1, f32(16)), ("layer_norm_fwd", 2, bf16(15)), ("layer_norm_fwd", 2, bf16(32)[::2]), ("layer_norm_fwd", 4, bf16(2, 6, 16)),
       ("layer_norm_fwd", 4, f32(2, 5, 16)), ("layer_norm_fwd", 5, f32(2, 6)), ("layer_norm_fwd", 5, bf16(2, 5)), ("layer_norm_fwd", 6, f32(5, 2).t()),
       ("layer_norm_bwd", 0, bf16(1, 5, 16)), ("layer_norm_bwd", 5, bf16(2, 5, 32)[..., :16]), ("layer_norm_bwd", 5, f32(2, 5, 16)),
       ("layer_norm_bwd", 6, bf16(16)), ("layer_norm_bwd", 7, f32(17)), ("layer_norm_bwd", 3, f32(10)),
       ("token_loss_fwd", 1, f32(9, 16)), ("token_loss_fwd", 1, bf16(9, 17)), ("token_loss_fwd", 2, ids(2, 6)), ("token_loss_fwd", 2, f32(2, 5)),
       ("token_loss_fwd", 3, bf16(2, 5)), ("token_loss_fwd", 4, f32(5, 2)), ("token_loss_bwd", 0, bf16(2, 5)), ("token_loss_bwd", 4, f32(2, 4)),
       ("token_loss_bwd", 5, bf16(2, 6, 16)), ("token_loss_bwd", 5, bf16(2, 10, 16)[:, ::2]), ("token_loss_bwd", 6, f32(8, 16)),
       ("token_loss_bwd", 6, f32(9, 16).half()), ("token_loss_bwd", 6, f32(16, 9).t())]


@pytest.mark.parametrize("name,at,bad", BAD)
def test_tensors_that_do_not_fit_are_refused(library, name, at, bad):
    args = good()[name]
    args[at] = bad
    with pytest.raises((TypeError, ValueError)):
        getattr(s1f, name)(*args)
    assert library.calls == []


def test_strides_of_single_rows_and_batches_do_not_matter(library):
    """torch gives a dimension of one element any stride."""
    x = torch.zeros((1, 1, 16), dtype=torch.bfloat16).as_strided((1, 1, 16), (3, 5, 1))
    s1f.layer_norm_fwd(x, bf16(16), bf16(16), 1e-5, bf16(1, 1, 16), f32(1, 1), f32(1, 1))
    s1f.layer_norm_bwd(bf16(1, 1, 16), x, bf16(16), f32(1, 1), f32(1, 1), bf16(1, 1, 16), f32(16), f32(16), torch.zeros(64))
    assert library.calls == ["s1f_layer_norm_fwd", "s1f_layer_norm_bwd"]


def test_tensors_outside_device_memory_are_refused(monkeypatch):
    monkeypatch.setattr(binding, "_native", lambda: binding._PythonForms)
    for name, args in good().items():
        with pytest.raises(ValueError):
            getattr(s1f, name)(*args)


DRIVER = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
import paper_2406_03488_amd as s1f
from paper_2406_03488_amd.binding import Rows
lib = s1f.load_library()
p, big = 4096, 1 << 45   # (no address is looked at)
for n, h, v, dtype in eval(sys.argv[2]):
    d = ctypes.byref(Rows(1, h, dtype, 0, n, 0, h, 0, h))
    assert lib.s1f_token_loss_fwd(d, p, p, h, v, p, 0, p, p, p, big, None) == 0
    assert lib.s1f_token_loss_bwd(d, p, p, p, h, v, p, 0, p, p, p, h, 0, p, big, None) == 0
    assert lib.s1f_embed_bwd(d, p, 0, p, v, 1.0, p, h, p, big, None) == 0
"""
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def launches(tmp_path, shapes):
    so = str(tmp_path / "recording.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-o", so, os.path.join(ROOT, "tests", "recording_runtime.c")], check=True)
    record = str(tmp_path / "record")
    run = subprocess.run([sys.executable, "-c", DRIVER, so, repr(shapes)], env=dict(os.environ, RECORD=record, PYTHONPATH=ROOT), capture_output=True, text=True,
                         cwd=ROOT)
    assert run.returncode == 0, run.stderr
    lines = [line.split() for line in open(record)]
    told = {name: int(rest[1]) for what, name, *rest in lines if what == "attribute"}
    done = [(name, int(rest[0]), int(rest[2])) for what, name, *rest in lines if what == "launch"]
    assert all(lds <= 64 * 1024 or told.get(name, 0) >= lds for name, _, lds in done)
    assert all(lds <= 160 * 1024 for _, _, lds in done)
    return done


def test_products_are_cut_as_the_gpu_tests_presume(tmp_path):
    """tests/test_gpu_token_loss.py checks these shapes: big tiles with their rest in quarters, all sizes of tiles, dx in parts behind whole tiles."""
    of = lambda shape, dtype=1: [(name.split("loss_")[1], grid) for name, grid, _ in launches(tmp_path, [(*shape, dtype)]) if "loss_" in name]
    first = of((1040, 512, 16384))
    scores = [(name, grid) for name, grid in first if name.startswith("scores")]
    assert [grid for _, grid in scores] == [256, 256] * 2                     # 320 big tiles: a round of them, 64 in quarters, in both directions
    assert "Li256ELi256" in scores[0][0] and "Li128ELi128" in scores[1][0]
    second = of((2304, 8192, 2304))
    dx = [grid for name, grid in second if name.startswith("dx_kernel")]
    assert dx[0] > 256 and (dx[0] - 256) % 32 == 0 and dx[0] > 256 + 32       # 288 big tiles: 32 of them in parts
    dw = [(name, grid) for name, grid in second if name.startswith("dw_kernel")]
    assert [grid for _, grid in dw] == [256, 128] and "Li128ELi128" in dw[1][0]
    assert any("scores" in name and "Li128ELi128" in name for name, _ in second)
    for shape, dtypes in (((700, 264, 9001), (0, 1)), ((1500, 72, 2000), (0, 1)), ((700, 264, 180000), (0,))):
        for dtype in dtypes:                                                  # no whole tiles, more workgroups than tiles: each in parts
            parts = [(grid, 128 if "Li128ELi128" in name else 256) for name, grid in of(shape, dtype) if name.startswith("dx_kernel")]
            assert len(parts) == (2 if shape[2] > 9001 else 1)
            tiles = -(-shape[0] // parts[0][1]) * -(-shape[1] // parts[0][1])
            assert all(grid % tiles == 0 and 2 * tiles <= grid <= 1024 for grid, _ in parts), (shape, dtype, parts)
    assert any("scores" in name and "Li64ELi128" in name for name, _ in of((130, 2000, 9000)) + of((700, 128, 130)) + of((5, 64, 129)))


def test_sorting_paths(tmp_path):
    """Few rows are ranked, more take two or three passes over their tokens' digits."""
    names = lambda n, v: [name for name, *_ in launches(tmp_path, [(n, 64, v, 0)]) if "embed_" in name]
    assert sum("rank" in x for x in names(12288, 600)) == 1 and not any("place" in x for x in names(12288, 600))
    assert sum("place" in x for x in names(12289, 600)) == 2 and sum("place" in x for x in names(12289, 300)) == 1
    assert sum("place" in x for x in names(20000, 600000)) == 3


LARGEST = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
import paper_2406_03488_amd as s1f
from paper_2406_03488_amd.binding import Rows
lib = s1f.load_library()
p, big = 4096, 1 << 60   # (no address is looked at)
for n, h, v, dtype in eval(sys.argv[2]):
    d = ctypes.byref(Rows(1, h, dtype, 0, n, 0, h, 0, h))
    if v <= 1 << 24 and n <= 1 << 20:
        assert lib.s1f_token_loss_fwd(d, p, p, h, v, p, 0, p, p, p, big, None) == 0
        assert lib.s1f_token_loss_bwd(d, p, p, p, h, v, p, 0, p, p, p, h, 0, p, big, None) == 0
    assert lib.s1f_embed_fwd(d, p, 0, p, h, v, 1.0, p, None) == 0 and lib.s1f_embed_bwd(d, p, 0, p, v, 1.0, p, h, p, big, None) == 0
    assert lib.s1f_layer_norm_fwd(d, p, p, p, 1e-5, p, p, p, None) == 0 and lib.s1f_layer_norm_bwd(d, p, p, p, p, p, p, p, p, p, big, None) == 0
"""


def test_the_largest_calls_fit_a_launch(tmp_path, monkeypatch):
    """The runtime takes launches of 2^32 threads and more, and runs fewer workgroups."""
    monkeypatch.setattr(sys.modules[__name__], "DRIVER", LARGEST)
    shapes = [(1 << 21, 16384, 1 << 26), (1 << 20, 8192, 300), (1 << 19, 16384, 1 << 17), (1, 16384, 1 << 24), (64, 1, 1 << 24), (1 << 20, 64, 1 << 16), (1 << 20, 1, 1)]
    done = launches(tmp_path, [(*s, dtype) for s in shapes for dtype in (0, 1)])
    assert len(done) > 100 and all(0 < grid <= (1 << 31) - 1 for _, grid, _ in done)
    assert all(grid * threads < 1 << 32 for _, grid, threads in threads_of(tmp_path))


def threads_of(tmp_path):
    return [(line.split()[1], int(line.split()[2]), int(line.split()[3])) for line in open(tmp_path / "record") if line.startswith("launch")]


@pytest.mark.parametrize("n,v", [(1 << 20, 200), (1 << 20, 171), (1 << 20, 255), (700000, 255), (1 << 20, 300), (699050, 255), (3000, 200), (2048, 200)])
def test_no_more_of_the_weight_is_packed_than_there_is(tmp_path, n, v):
    """fp32 calls whose rows leave room for fewer than 256 tokens a piece: a launch that packs the weight has a workgroup (or a
    quarter of one) for each of its rows."""
    h = 2048
    done = launches(tmp_path, [(n, h, v, 0)])
    grids = [(name, grid) for name, grid, _ in done if "loss_prepare" in name or ("loss_pack" in name and name.split("loss_pack_kernel")[1].split("EE")[0].endswith("Lb0"))]
    assert grids
    for name, grid in grids:
        threads, rows = (1024, (n + 7) // 8) if "loss_prepare" in name else (256, 0)
        assert grid <= rows + -(-v * (h // 8) // threads), (name, grid)
