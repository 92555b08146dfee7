"""How the calls around a layer's attention are launched, with a recording runtime in place of a device: cuts of the products that the GPU tests presume, shares of the
rotations, and the largest calls."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
import paper_2406_03488_amd as s1f
from paper_2406_03488_amd.binding import Heads, Rows
lib = s1f.load_library()
p, big = 4096, 1 << 60   # (no address is looked at)
for what, *shape in eval(sys.argv[2]):
    if what == "ffn":
        n, h, f, dtype = shape
        d = ctypes.byref(Rows(1, h, dtype, 0, n, 0, h, 0, h))
        assert lib.s1f_gated_ffn_fwd(d, p, p, h, p, f, f, 0, p, p, p, big, None) == 0
        assert lib.s1f_gated_ffn_bwd(d, p, p, p, h, p, f, f, 0, p, p, p, h, p, f, 0, p, big, None) == 0
    else:
        n, hq, hk, dim, rotary, dtype, interleaved = shape
        row = 1 << 26
        d = ctypes.byref(Heads(1, hq, hk, dim, dtype, rotary, interleaved, 0, n, *[0, row * dim, dim] * 4, n))
        turn = (p, 1.0, None, 0, 0, 0)
        assert lib.s1f_rope_fwd(d, p, p, p, *turn, p, p, p, None) == 0
        assert lib.s1f_rope_bwd(d, p, p, p, *turn, p, p, p, None) == 0
        assert lib.s1f_qk_norm_rope_fwd(d, p, p, p, p, p, 1e-6, *turn, p, p, p, None) == 0
        assert lib.s1f_qk_norm_rope_bwd(d, p, p, p, p, p, p, p, 1e-6, *turn, p, p, p, p, p + 4096, p, big, None) == 0
"""


def launches(tmp_path, calls):
    """(kernel, workgroups, threads, LDS) of every launch."""
    so, record = str(tmp_path / "recording.so"), str(tmp_path / "record")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-o", so, os.path.join(ROOT, "tests", "recording_runtime.c")], check=True)
    run = subprocess.run([sys.executable, "-c", DRIVER, so, repr(calls)], env=dict(os.environ, RECORD=record, PYTHONPATH=ROOT), capture_output=True, text=True, cwd=ROOT)
    assert run.returncode == 0, run.stderr
    lines = [line.split() for line in open(record)]
    told = {name: int(rest[1]) for what, name, *rest in lines if what == "attribute"}
    done = [(name, *(int(x) for x in rest)) for what, name, *rest in lines if what == "launch"]
    assert all(lds <= 64 * 1024 or told.get(name, 0) >= lds for name, _, _, lds in done) and all(lds <= 160 * 1024 for *_, lds in done)
    return done


def of(done, part):
    return [(name, grid) for name, grid, *_ in done if part in name]


SHAPES = [((72, 4360, 2180), (0, 1)), ((4360, 72, 2184), (0, 1)), ((4361, 4360, 68), (0, 1)), ((30000, 40, 24), (0, 1)), ((300, 640, 1000), (0, 1)), ((515, 96, 2052), (0, 1)),
          ((130, 128, 4), (0, 1)), ((700, 72, 264), (0, 1)), ((129, 200, 332), (0, 1)), ((4100, 4100, 1500), (0,)), ((4500, 4500, 1000), (0,)), ((8200, 1100, 2100), (0, 1)), ((600, 1100, 8200), (1,)),
          ((4100, 4100, 6000), (1,)), ((4099, 4096, 11008), (1,))]


def test_products_are_cut_as_the_gpu_tests_presume(tmp_path):
    """tests/test_gpu_ffn.py checks these shapes: tiles of every size for every product, their rests in quarters or in parts, few rows, dW in turns."""
    kinds = set()
    for shape, dtypes in SHAPES:
        for dtype in dtypes:
            done = launches(tmp_path, [("ffn", *shape, dtype)])
            for (name, *_), (behind, *_) in zip(done, done[1:] + [("", 0, 0, 0)]):
                side = "big" if "Li256ELi256" in name else "middle" if "Li128ELi128" in name else "low" if "Li64ELi128" in name else ""
                kernel = next(k for k in ("up", "dh", "product", "join", "few", "pack") if f"ffn_{k}_kernel" in name)
                if kernel == "product":
                    kernel = {"Lb0ELb0E": "y", "Lb0ELb1E": "dx", "Lb1ELb1E": "dw"}[name.split("ELNS")[0][-7:] + "E"]
                    if "join" in behind:
                        kernel += " in parts"
                kinds.add((kernel, side, dtype))
    for dtype in (0, 1):
        for kernel in ("up", "dh", "y", "dx"):
            for side in ("big", "middle", "low"):
                assert (kernel, side, dtype) in kinds, (kernel, side, dtype)
        assert {("dw", "big", dtype), ("dw", "middle", dtype), ("dw in parts", "middle", dtype), ("dw in parts", "big", dtype), ("pack", "", dtype)} <= kinds
        for kernel in ("y in parts", "dx in parts"):
            assert {(kernel, "low", dtype), (kernel, "big", dtype)} <= kinds and ((kernel, "middle", 0) in kinds or (kernel, "middle", 1) in kinds), (kernel, dtype)
    few = launches(tmp_path, [("ffn", 16, 520, 1400, 1), ("ffn", 64, 520, 1400, 0)])
    assert len(of(few, "ffn_few")) == 4 and not of(few, "ffn_up")
    assert not of(launches(tmp_path, [("ffn", 17, 4096, 11008, 1), ("ffn", 65, 64, 64, 0)]), "ffn_few")
    # fp32 sums of a weight's gradient from 12288 rows on in turns of about 8192
    dw = lambda n: [name for name, _ in of(launches(tmp_path, [("ffn", n, 64, 64, 0)]), "ffn_product") if "Lb1ELb1E" in name]
    assert len(dw(12287)) == 2 and len(dw(12288)) == 4 and len(dw(49152)) == 12


def test_the_largest_calls_fit_a_launch(tmp_path):
    """The runtime takes launches of 2^32 threads and more, and runs fewer workgroups."""
    calls = [("ffn", 1 << 20, 8192, 4096, t) for t in (0, 1)] + [("ffn", 1 << 19, 16384, 8192, t) for t in (0, 1)] + [("ffn", 1, 4096, 1 << 17, t) for t in (0, 1)]
    calls += [("ffn", 1 << 15, 4096, 1 << 17, t) for t in (0, 1)] + [("ffn", 1 << 20, 1, 1, t) for t in (0, 1)] + [("ffn", 1, 16384, 1, t) for t in (0, 1)]
    calls += [("rope", 1 << 26, 16, 8, d, r, t, i) for d, r in ((256, 256), (2, 2), (64, 20), (6, 2)) for t in (0, 1) for i in (0, 1)]
    calls += [("rope", 1, 1 << 16, 1 << 16, d, r, t, i) for d, r in ((256, 2), (2, 0), (128, 128)) for t in (0, 1) for i in (0, 1)]
    calls += [("rope", 1 << 13, 1 << 16, 1 << 16, 8, 8, 1, 0)]
    done = launches(tmp_path, calls)
    assert len(done) > 150
    for name, grid, threads, _ in done:
        assert 0 < grid <= (1 << 31) - 1 and grid * threads < 1 << 32, (name, grid)


@pytest.mark.parametrize("dim,rotary,lanes", [(128, 128, "Li4ELi16ELi1E"), (64, 64, "Li4ELi8ELi1E"), (256, 256, "Li4ELi32ELi1E"), (80, 20, "Li4ELi16ELi1E"), (6, 4, "Li1ELi8ELi4E"),
                                              (254, 250, "Li1ELi32ELi4E"), (90, 90, "Li1ELi16ELi4E")])
def test_rows_are_dealt_out(tmp_path, dim, rotary, lanes):
    """Lanes of a row, and the gradient's workgroups: no more than the workspace has room for."""
    done = launches(tmp_path, [("rope", 3000, 32, 8, dim, rotary, t, i) for t in (0, 1) for i in (0, 1)])
    kernels = [(name, grid) for name, grid, *_ in done if "rope_kernel" in name]
    assert len(kernels) == 16 and any(lanes in name for name, _ in kernels)
    gains = [grid for name, grid in kernels if name.endswith("Lb1ELb1EEEvNS0_8RopeArgsE")]
    assert len(gains) == 4 and all(1 <= g <= 2048 for g in gains)
    assert [grid for name, grid, *_ in done if "rope_join" in name] == [-(-2 * dim // 16)] * 4
