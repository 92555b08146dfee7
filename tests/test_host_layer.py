"""What the calls around a layer's attention refuse: the C entry points before anything is launched, and their Python forms before the library is
called; frequencies of the rotations.  No device."""
import ctypes
import math

import pytest
import torch

import paper_2406_03488_amd as s1f
from oracle import layer as L
from paper_2406_03488_amd import binding
from paper_2406_03488_amd.binding import Heads, Rows

P, ODD, OFF = 4096, 4097, 4104     # addresses: aligned, not even, on 8 bytes (none is looked at)
BIG = 1 << 50
STRIDES = ("q", "kv", "rot", "cache")


def heads(**kw):
    base = dict(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=1, rotary_dim=32, interleaved=0, reserved=0, rows=5, cache_capacity=9)
    for side in STRIDES:
        base.update({f"{side}_stride_b": 1 << 20, f"{side}_stride_h": 1 << 12, f"{side}_stride_s": 64})
    base.update(kw)
    return Heads(**base)


def ref(d):
    return ctypes.byref(d) if d else None


def rope_fwd(d, q=P, k=P, v=P, freqs=P, magnitude=1.0, positions=P, off=0, q_rot=P, kc=P, vc=P):
    return s1f.load_library().s1f_rope_fwd(ref(d), q, k, v, freqs, magnitude, positions, 5, 0, off, q_rot, kc, vc, None)


def rope_bwd(d, q_rot=P, kc=P, vc=P, freqs=P, magnitude=1.0, positions=P, off=0, q=P, k=P, v=P):
    return s1f.load_library().s1f_rope_bwd(ref(d), q_rot, kc, vc, freqs, magnitude, positions, 5, 0, off, q, k, v, None)


def norm_fwd(d, q=P, k=P, v=P, q_gain=P, k_gain=P, eps=1e-6, freqs=P, magnitude=1.0, positions=P, off=0, q_rot=P, kc=P, vc=P):
    return s1f.load_library().s1f_qk_norm_rope_fwd(ref(d), q, k, v, q_gain, k_gain, eps, freqs, magnitude, positions, 5, 0, off, q_rot, kc, vc, None)


def norm_bwd(d, q_rot=P, kc=P, vc=P, x=P, y=P, q_gain=P, k_gain=P, eps=1e-6, freqs=P, magnitude=1.0, positions=P, off=0, q=P, k=P, v=P, dq_gain=P, dk_gain=2 * P,
             ws=P, n=BIG):
    return s1f.load_library().s1f_qk_norm_rope_bwd(ref(d), q_rot, kc, vc, x, y, q_gain, k_gain, eps, freqs, magnitude, positions, 5, 0, off, q, k, v, dq_gain,
                                                   dk_gain, ws, n, None)


ROTATIONS = (rope_fwd, rope_bwd, norm_fwd, norm_bwd)


@pytest.mark.parametrize("call", ROTATIONS)
def test_descriptors_refused(call):
    assert call(None) == 1
    for bad in (dict(batch=0), dict(batch=-1), dict(n_q_heads=0), dict(n_kv_heads=0), dict(reserved=1), dict(interleaved=2), dict(interleaved=-1),
                dict(rotary_dim=-2), dict(rotary_dim=31), dict(rotary_dim=66)):
        assert call(heads(**bad)) == 1, bad
    for bad in (dict(dtype=2), dict(dtype=-1), dict(head_dim=0), dict(head_dim=63), dict(head_dim=-64), dict(head_dim=258), dict(n_q_heads=(1 << 16) + 1),
                dict(n_kv_heads=(1 << 16) + 1), dict(rows=(1 << 26) + 1, cache_capacity=1 << 27), dict(batch=1 << 14, rows=1 << 13, cache_capacity=1 << 14),
                dict(batch=1 << 30, rows=1 << 34)):
        assert call(heads(**{**{f"{s}_stride_s": 300 for s in STRIDES}, **bad})) == 2, bad
    for bad in (dict(rows=0), dict(rows=-1), dict(rows=10), dict(cache_capacity=4), dict(cache_capacity=-1)):
        assert call(heads(**bad)) == 3, bad
    for off in (-1, 5, 1 << 40, (1 << 63) - 1, -(1 << 63)):
        assert call(heads(), off=off) == 3, off
    for side in STRIDES:
        for which in "bhs":
            for bad in (63, 0, -64):
                assert call(heads(**{f"{side}_stride_{which}": bad})) == 1, (side, which, bad)
    # one row, but of a cache of more
    assert call(heads(rows=1, cache_stride_s=0)) == 1


@pytest.mark.parametrize("call", ROTATIONS)
def test_pointers_refused(call):
    names = {rope_fwd: ("q", "k", "q_rot", "kc"), rope_bwd: ("q", "k", "q_rot", "kc"), norm_fwd: ("q", "k", "q_rot", "kc", "q_gain", "k_gain"),
             norm_bwd: ("q", "k", "q_rot", "kc", "x", "y", "q_gain", "k_gain", "dq_gain", "dk_gain", "ws")}[call]
    for name in names:
        assert call(heads(), **{name: None}) == 1, name
        assert call(heads(), **{name: ODD}) == 1, name
    for name in ("v", "vc"):                                      # both or neither
        assert call(heads(), **{name: None}) == 1 and call(heads(), **{name: ODD}) == 1, name
    for name in ("freqs", "positions"):
        assert call(heads(), **{name: 4100}) == 1, name
    assert call(heads(), freqs=None) == 1
    for bad in (math.inf, -math.inf, math.nan):
        assert call(heads(), magnitude=bad) == 1
    if call in (norm_fwd, norm_bwd):
        assert call(heads(), eps=-1e-9) == 1 and call(heads(), eps=math.nan) == 1
    if call is norm_bwd:
        for at in (P, P + 4 * 63, P - 4 * 63):                    # gains' gradients in one place
            assert call(heads(), dk_gain=at) == 1
        assert call(heads(), ws=OFF) == 1 and call(heads(), n=s1f.load_library().s1f_qk_norm_rope_bwd_workspace_bytes(ref(heads())) - 1) == 1


def test_workspace_of_the_norms_gradient():
    ask = s1f.load_library().s1f_qk_norm_rope_bwd_workspace_bytes
    assert 0 < ask(ref(heads())) < 1 << 23
    for bad in (None, heads(rows=0), heads(batch=0), heads(dtype=7), heads(head_dim=300)):
        assert ask(ref(bad)) == 0
    acc = torch.zeros(2, 2, 9, 64)
    assert s1f.qk_norm_rope_bwd_workspace_bytes(torch.zeros(2, 4, 5, 64, dtype=torch.bfloat16), acc) == ask(ref(heads()))


def test_frequencies():
    freqs, magnitude = s1f.rope_frequencies(128, 5e5)
    assert magnitude == 1.0 and max(abs(a / b - 1) for a, b in zip(freqs, L.frequencies(128, 5e5))) < 1e-14
    linear, magnitude = s1f.rope_frequencies(64, scaling=s1f.ROPE_LINEAR, factor=4.0)
    assert magnitude == 1.0 and max(abs(4 * a / b - 1) for a, b in zip(linear, L.frequencies(64))) < 1e-14
    base, magnitude = s1f.rope_frequencies(64, scaling=s1f.ROPE_BASE, factor=8.0)
    plain = L.frequencies(64)
    assert magnitude == 1.0 and base[0] == 1.0 and abs(8 * base[-1] / plain[-1] - 1) < 1e-13 and all(a <= b for a, b in zip(base, plain))
    parts, magnitude = s1f.rope_frequencies(128, scaling=s1f.ROPE_PARTS, factor=16.0, trained_rows=4096, slow_turns=1.0, fast_turns=32.0)
    assert magnitude == ctypes.c_float(0.1 * math.log(16) + 1).value
    for i, (got, f) in enumerate(zip(parts, L.frequencies(128))):
        turns = 4096 * f / (2 * math.pi)
        share = 1.0 if turns >= 32 else 0.0 if turns <= 1 else (turns - 1) / 31
        assert abs(got / (f * share + f / 16 * (1 - share)) - 1) < 1e-13, i
    assert s1f.rope_frequencies(2) == ([1.0], 1.0)


def test_frequencies_refused():
    good = dict(rotary_dim=64, base=1e4, scaling=s1f.ROPE_PARTS, factor=2.0, trained_rows=4096, slow_turns=1.0, fast_turns=32.0)
    s1f.rope_frequencies(**good)
    for bad in (dict(rotary_dim=0), dict(rotary_dim=-4), dict(rotary_dim=7), dict(base=0.0), dict(base=-1.0), dict(base=math.inf), dict(base=math.nan),
                dict(scaling=4), dict(scaling=-1), dict(factor=0.0), dict(factor=-2.0), dict(factor=0.5), dict(factor=math.nan), dict(factor=math.inf),
                dict(trained_rows=0), dict(slow_turns=-1.0), dict(slow_turns=32.0), dict(fast_turns=math.inf), dict(fast_turns=math.nan),
                dict(scaling=s1f.ROPE_BASE, rotary_dim=2)):
        with pytest.raises(s1f.S1FError):
            s1f.rope_frequencies(**{**good, **bad})
    lib = s1f.load_library()
    out, magnitude = (ctypes.c_double * 32)(), ctypes.c_float()
    assert lib.s1f_rope_frequencies(64, 1e4, 0, 1.0, 0, 0.0, 0.0, None, ctypes.byref(magnitude)) == 1
    assert lib.s1f_rope_frequencies(64, 1e4, 0, 1.0, 0, 0.0, 0.0, out, None) == 1


# ---- gated feed-forward block ----------------------------------------------------------------------------------------------------------

def rows(**kw):
    base = dict(batch=2, hidden=64, dtype=1, reserved=0, rows=5, x_stride_b=320, x_stride_s=64, y_stride_b=320, y_stride_s=64)
    base.update(kw)
    return Rows(**base)


def ffn_fwd(d, x=P, w_in=P, in_stride=64, w_out=P, out_stride=96, inner=96, act=0, y=P, gate_up=P, ws=P, n=BIG):
    return s1f.load_library().s1f_gated_ffn_fwd(ref(d), x, w_in, in_stride, w_out, out_stride, inner, act, y, gate_up, ws, n, None)


def ffn_bwd(d, dy=P, x=P, w_in=P, in_stride=64, w_out=P, out_stride=96, inner=96, act=0, gate_up=P, dx=P, dw_in=P, dw_in_stride=64, dw_out=P, dw_out_stride=96, code=0,
            ws=P, n=BIG):
    return s1f.load_library().s1f_gated_ffn_bwd(ref(d), dy, x, w_in, in_stride, w_out, out_stride, inner, act, gate_up, dx, dw_in, dw_in_stride, dw_out, dw_out_stride,
                                                code, ws, n, None)


@pytest.mark.parametrize("call", [ffn_fwd, ffn_bwd])
def test_ffn_refused(call):
    assert call(None) == 1
    for bad in (dict(batch=0), dict(batch=-1), dict(hidden=0), dict(reserved=1), dict(x_stride_s=63), dict(y_stride_s=63), dict(x_stride_b=63), dict(y_stride_b=-320)):
        assert call(rows(**bad)) == 1, bad
    for bad in (dict(dtype=2), dict(dtype=-1), dict(hidden=16385, x_stride_s=1 << 15, y_stride_s=1 << 15, x_stride_b=1 << 20, y_stride_b=1 << 20),
                dict(batch=1, rows=(1 << 20) + 1), dict(batch=1 << 30, rows=1 << 34)):
        assert call(rows(**bad), in_stride=1 << 15) == 2, bad
    for bad in (0, -1, -(1 << 40)):
        assert call(rows(rows=bad)) == 3
    for bad in (dict(inner=0), dict(inner=-96), dict(in_stride=63), dict(out_stride=95), dict(act=-1), dict(act=3)):
        assert call(rows(), **bad) == 1, bad
    for bad in (dict(inner=(1 << 17) + 1, out_stride=1 << 18), dict(in_stride=1 << 22), dict(out_stride=1 << 22), dict(inner=1 << 17, out_stride=1 << 17, in_stride=4097)):
        assert call(rows(), **bad, **({"dw_out_stride": 1 << 18} if call is ffn_bwd else {})) == 2, bad
    big = dict(batch=1, rows=1 << 20)
    assert call(rows(**big, hidden=8200, x_stride_s=8200, y_stride_s=8200), in_stride=8200) == 2
    assert call(rows(**big), inner=4097, out_stride=4097, **({"dw_out_stride": 4097} if call is ffn_bwd else {})) == 2
    names = ("x", "w_in", "w_out", "y", "ws") if call is ffn_fwd else ("dy", "x", "w_in", "w_out", "gate_up", "dx", "dw_in", "dw_out", "ws")
    for name in names:
        assert call(rows(), **{name: None}) == 1 and call(rows(), **{name: ODD}) == 1, name
    for name in ("w_in", "w_out", "ws"):
        assert call(rows(), **{name: OFF}) == 1, name
    assert call(rows(), gate_up=ODD) == 1 and call(rows(), n=255) == 1 and call(rows(), n=0) == 1
    if call is ffn_bwd:
        assert call(rows(), code=2) == 2 and call(rows(dtype=0), code=1) == 2 and call(rows(), dw_in_stride=63) == 1 and call(rows(), dw_out_stride=95) == 1


def test_ffn_workspaces():
    lib = s1f.load_library()
    for f in (lib.s1f_gated_ffn_fwd_workspace_bytes, lib.s1f_gated_ffn_bwd_workspace_bytes):
        assert f(ref(rows()), 96, 64, 96) > 0
        for bad in (None, rows(rows=0), rows(hidden=0), rows(dtype=5)):
            assert f(ref(bad), 96, 64, 96) == 0
        assert f(ref(rows()), 0, 64, 96) == 0 and f(ref(rows()), 96, 63, 96) == 0 and f(ref(rows()), 96, 64, 95) == 0
    # a forward of bf16 rows keeps what is between its products, not the weights
    d = rows(batch=1, rows=4096, hidden=4096, x_stride_s=4096, y_stride_s=4096)
    assert lib.s1f_gated_ffn_fwd_workspace_bytes(ref(d), 11008, 4096, 11008) < 2 * 4096 * (4096 + 11008) + (64 << 20)


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


def good():
    """Arguments of every call, by name; all of them fit."""
    f, at, ws = torch.zeros(8, dtype=torch.float64), torch.zeros(2, 5, dtype=torch.int64), torch.zeros(64, dtype=torch.uint8)
    q, k, v, kc, vc = bf16(2, 4, 5, 16), bf16(2, 2, 5, 16), bf16(2, 2, 5, 16), bf16(2, 2, 9, 16), bf16(2, 2, 9, 16)
    ka, va = f32(2, 2, 9, 16), f32(2, 2, 9, 16)
    gains = [bf16(16), bf16(16)]
    return {"rope_fwd": [q, k, v, f, 1.0, False, at, 3, bf16(2, 4, 5, 16), kc, vc], "rope_bwd": [bf16(2, 4, 5, 16), ka, va, f, 1.0, False, at, 3, q, k, v],
            "qk_norm_rope_fwd": [q, k, v, *gains, 1e-6, f, 1.0, False, at, 3, bf16(2, 4, 5, 16), kc, vc],
            "gated_ffn_fwd": [bf16(2, 5, 16), bf16(48, 16), bf16(16, 24), s1f.SILU, bf16(2, 5, 16), bf16(2, 5, 48), ws],
            "gated_ffn_bwd": [bf16(2, 5, 16), bf16(2, 5, 16), bf16(48, 16), bf16(16, 24), s1f.GELU, bf16(2, 5, 48), bf16(2, 5, 16), f32(48, 16), f32(16, 24), ws],
            "qk_norm_rope_bwd": [bf16(2, 4, 5, 16), ka, va, bf16(2, 4, 5, 16), bf16(2, 2, 5, 16), *gains, 1e-6, f, 1.0, False, at, 3, q, k, v, f32(16),
                                 f32(16), ws]}


def test_good_calls_reach_the_library(library):
    for name, args in good().items():
        getattr(s1f, name)(*args)
        assert library.calls.pop() == "s1f_" + name and not library.calls
    for name, drop, positions in (("rope_fwd", (2, 10), 6), ("rope_bwd", (2, 10), 6), ("qk_norm_rope_fwd", (2, 13), 9), ("qk_norm_rope_bwd", (2, 15), 12)):
        args = good()[name]
        for i in drop:
            args[i] = None
        args[positions] = 7                                        # the first row's
        getattr(s1f, name)(*args)
        assert library.calls.pop() == "s1f_" + name


i64 = torch.int64
BAD = [(name, at, value) for name, q, k, v, rot, kc, vc, f, p in
       (("rope_fwd", 0, 1, 2, 8, 9, 10, 3, 6), ("qk_norm_rope_fwd", 0, 1, 2, 11, 12, 13, 6, 9)) for at, value in
       ((q, bf16(2, 4, 5, 8)), (q, bf16(4, 5, 16)), (q, f32(2, 4, 5, 16)), (q, bf16(2, 4, 5, 32)[..., ::2]), (q, bf16(1, 4, 5, 16)), (q, bf16(2, 4, 6, 16)),
        (k, bf16(2, 2, 6, 16)), (k, bf16(1, 2, 5, 16)), (k, f32(2, 2, 5, 16)), (k, bf16(2, 2, 5, 17)[..., 1:]), (v, bf16(2, 1, 5, 16)), (v, None),
        (v, bf16(2, 5, 2, 16).transpose(1, 2)), (rot, bf16(2, 4, 5, 17)), (rot, f32(2, 4, 5, 16)), (rot, bf16(2, 3, 5, 16)), (kc, bf16(2, 3, 9, 16)),
        (kc, f32(2, 2, 9, 16)), (kc, bf16(2, 2, 9, 8)), (kc, bf16(2, 2, 8, 16)), (vc, bf16(2, 2, 8, 16)), (vc, None), (f, torch.zeros(8)),
        (f, torch.zeros(9, dtype=torch.float64)), (f, torch.zeros(2, 4, dtype=torch.float64)), (f, torch.zeros(16, dtype=torch.float64)[::2]),
        (p, torch.zeros(2, 4, dtype=i64)), (p, torch.zeros(2, 5, dtype=torch.int32)), (p, torch.zeros(5, dtype=i64)), (p, torch.zeros(2, 10, dtype=i64)[:, ::2]),
        (p, 1 << 63), (p, None))]
BAD += [("rope_bwd", 1, bf16(2, 2, 9, 16)), ("rope_bwd", 2, bf16(2, 2, 9, 16)), ("rope_bwd", 2, None), ("rope_bwd", 10, None), ("rope_bwd", 8, f32(2, 4, 5, 16)),
        ("rope_bwd", 9, bf16(2, 2, 4, 16)), ("rope_bwd", 0, bf16(2, 4, 4, 16)), ("rope_bwd", 1, f32(2, 2, 9, 8)),
        ("qk_norm_rope_fwd", 3, bf16(15)), ("qk_norm_rope_fwd", 4, f32(16)), ("qk_norm_rope_fwd", 3, bf16(32)[::2]),
        ("qk_norm_rope_bwd", 3, bf16(2, 4, 5, 17)[..., 1:]), ("qk_norm_rope_bwd", 3, bf16(2, 4, 6, 16)), ("qk_norm_rope_bwd", 4, f32(2, 2, 5, 16)),
        ("qk_norm_rope_bwd", 4, bf16(2, 5, 2, 16).transpose(1, 2)), ("qk_norm_rope_bwd", 5, bf16(17)), ("qk_norm_rope_bwd", 16, bf16(16)),
        ("gated_ffn_fwd", 0, f32(2, 5, 16)), ("gated_ffn_fwd", 0, bf16(5, 16)), ("gated_ffn_fwd", 0, bf16(2, 5, 32)[..., ::2]), ("gated_ffn_fwd", 1, bf16(47, 16)),
        ("gated_ffn_fwd", 1, bf16(48, 15)), ("gated_ffn_fwd", 1, f32(48, 16)), ("gated_ffn_fwd", 1, bf16(16, 48).t()), ("gated_ffn_fwd", 2, bf16(16, 25)),
        ("gated_ffn_fwd", 2, bf16(15, 24)), ("gated_ffn_fwd", 2, bf16(24, 16).t()), ("gated_ffn_fwd", 4, bf16(2, 6, 16)), ("gated_ffn_fwd", 4, f32(2, 5, 16)),
        ("gated_ffn_fwd", 5, bf16(2, 5, 24)), ("gated_ffn_fwd", 5, f32(2, 5, 48)), ("gated_ffn_fwd", 5, bf16(2, 5, 96)[..., ::2]),
        ("gated_ffn_fwd", 6, torch.zeros(8, 8)[:, ::2]), ("gated_ffn_bwd", 0, bf16(2, 4, 16)), ("gated_ffn_bwd", 5, bf16(2, 5, 47)), ("gated_ffn_bwd", 5, f32(2, 5, 48)),
        ("gated_ffn_bwd", 6, bf16(2, 10, 16)[:, ::2]), ("gated_ffn_bwd", 6, f32(2, 5, 16)), ("gated_ffn_bwd", 7, f32(46, 16)), ("gated_ffn_bwd", 7, bf16(48, 16)),
        ("gated_ffn_bwd", 8, f32(16, 23)), ("gated_ffn_bwd", 8, bf16(16, 24)), ("gated_ffn_bwd", 7, f32(48, 16).half()),
        ("qk_norm_rope_bwd", 17, f32(15)), ("qk_norm_rope_bwd", 18, torch.zeros(8, 8)[:, ::2])]


@pytest.mark.parametrize("name,at,value", BAD)
def test_tensors_refused(library, name, at, value):
    args = good()[name]
    args[at] = value
    with pytest.raises((ValueError, TypeError)):
        getattr(s1f, name)(*args)
    assert library.calls == []


def test_tensors_of_another_device_are_refused():
    """Without a device every tensor is of another one."""
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    for name, args in good().items():
        with pytest.raises(ValueError):
            getattr(s1f, name)(*args)
