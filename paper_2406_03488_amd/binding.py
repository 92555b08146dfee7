"""ctypes binding of the C ABI declared in include/s1f.h (same names, same argument order)."""
from __future__ import annotations

import ctypes
import os
import warnings

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libs1f.so")
_lib = None

S1F_F32, S1F_BF16 = 0, 1


class S1FError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({strerror(status)})")


class Desc(ctypes.Structure):
    """Mirror of s1f_desc."""
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("q_stride_b", ctypes.c_int64), ("q_stride_h", ctypes.c_int64), ("q_stride_s", ctypes.c_int64),
                ("kv_stride_b", ctypes.c_int64), ("kv_stride_h", ctypes.c_int64), ("kv_stride_s", ctypes.c_int64),
                ("kv_capacity", ctypes.c_int64)]


class Rows(ctypes.Structure):
    """Mirror of s1f_rows."""
    _fields_ = [("batch", ctypes.c_int32), ("hidden", ctypes.c_int32), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("rows", ctypes.c_int64), ("x_stride_b", ctypes.c_int64), ("x_stride_s", ctypes.c_int64),
                ("y_stride_b", ctypes.c_int64), ("y_stride_s", ctypes.c_int64)]


class Heads(ctypes.Structure):
    """Mirror of s1f_heads."""
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "dtype", "rotary_dim", "interleaved", "reserved")] + [
        (n, ctypes.c_int64) for n in ("rows", "q_stride_b", "q_stride_h", "q_stride_s", "kv_stride_b", "kv_stride_h", "kv_stride_s", "rot_stride_b",
                                      "rot_stride_h", "rot_stride_s", "cache_stride_b", "cache_stride_h", "cache_stride_s", "cache_capacity")]


class Pass(ctypes.Structure):
    _fields_ = [("micro_batch", ctypes.c_int32), ("segment", ctypes.c_int32), ("backward", ctypes.c_int32)]


class StagePass(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("micro_batch", ctypes.c_int32), ("segment", ctypes.c_int32),
                ("chunk", ctypes.c_int32)]


class PipelineDesc(ctypes.Structure):
    """Mirror of s1f_pipeline_desc."""
    _fields_ = [("pp_size", ctypes.c_int32), ("n_micro", ctypes.c_int32), ("n_seg", ctypes.c_int32),
                ("n_chunks", ctypes.c_int32), ("split_weight_grad", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("max_pending_wgrad", ctypes.c_int64), ("t_comm", ctypes.c_int64),
                ("t_fwd", ctypes.POINTER(ctypes.c_int64)), ("t_bwd", ctypes.POINTER(ctypes.c_int64)),
                ("t_wgrad", ctypes.POINTER(ctypes.c_int64)), ("seg_tokens", ctypes.POINTER(ctypes.c_int64))]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libs1f.so (built in-tree by paper_2406_03488_amd.build).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} not found: build it with `python -m paper_2406_03488_amd.build` "
                          "(there is no fallback implementation)")
    lib = ctypes.CDLL(_LIB_PATH)
    i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
    dp = ctypes.POINTER(Desc)
    lib.s1f_partition.argtypes = [i64, i32, i32, i32, ctypes.POINTER(i64)]
    lib.s1f_partition.restype = ctypes.c_int
    lib.s1f_partition_ex.argtypes = [i64, i32, i32, i32, i32, i64, ctypes.POINTER(i64)]
    lib.s1f_partition_ex.restype = ctypes.c_int
    lib.s1f_partition_rebalance.argtypes = [i32, ctypes.POINTER(i64), ctypes.POINTER(i64), i64, ctypes.POINTER(i64)]
    lib.s1f_partition_rebalance.restype = ctypes.c_int
    lib.s1f_seg_attn_fwd.argtypes = [dp, vp, vp, vp, i64, i64, vp, vp, vp]
    lib.s1f_seg_attn_fwd.restype = ctypes.c_int
    lib.s1f_seg_attn_fwd_ws.argtypes = [dp, vp, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    lib.s1f_seg_attn_fwd_ws.restype = ctypes.c_int
    lib.s1f_fwd_workspace_bytes.argtypes = [dp, i64, i64]
    lib.s1f_fwd_workspace_bytes.restype = sz
    lib.s1f_seg_attn_bwd.argtypes = [dp, vp, vp, vp, vp, vp, vp, i64, i64, vp, vp, vp, vp, sz, vp]
    lib.s1f_seg_attn_bwd.restype = ctypes.c_int
    lib.s1f_seg_attn_bwd_dq.argtypes = [dp, vp, vp, vp, vp, vp, vp, i64, i64, vp, vp, sz, vp]
    lib.s1f_seg_attn_bwd_dq.restype = ctypes.c_int
    lib.s1f_seg_attn_bwd_dkdv.argtypes = [dp, vp, vp, vp, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    lib.s1f_seg_attn_bwd_dkdv.restype = ctypes.c_int
    lib.s1f_seg_attn_bwd_noalloc.argtypes = [dp, vp, vp, vp, vp, vp, vp, i64, i64, vp, vp, vp, vp]
    lib.s1f_seg_attn_bwd_noalloc.restype = ctypes.c_int
    lib.s1f_static_scratch_rows.argtypes = []
    lib.s1f_static_scratch_rows.restype = sz
    lib.s1f_bwd_workspace_bytes.argtypes = [dp, i64, i64]
    lib.s1f_bwd_workspace_bytes.restype = sz
    lib.s1f_launch_plan.argtypes = [dp, i32, i64, i64, ctypes.POINTER(i64)]
    lib.s1f_launch_plan.restype = ctypes.c_int
    lib.s1f_launch_paths.argtypes = [dp, i64, i64, ctypes.POINTER(i64)]
    lib.s1f_launch_paths.restype = ctypes.c_int
    lib.s1f_kv_append.argtypes = [dp, vp, vp, i64, i64, i64, i64, i64, vp, vp, vp]
    lib.s1f_kv_append.restype = ctypes.c_int
    lib.s1f_kv_grad_emit.argtypes = [dp, vp, vp, i64, i64, vp, vp, i64, i64, i64, vp]
    lib.s1f_kv_grad_emit.restype = ctypes.c_int
    rp, f32 = ctypes.POINTER(Rows), ctypes.c_float
    lib.s1f_embed_fwd.argtypes = [rp, vp, i64, vp, i64, i64, f32, vp, vp]
    lib.s1f_embed_bwd.argtypes = [rp, vp, i64, vp, i64, f32, vp, i64, vp, sz, vp]
    lib.s1f_embed_bwd_workspace_bytes.argtypes = [rp, i64]
    lib.s1f_layer_norm_fwd.argtypes = [rp, vp, vp, vp, f32, vp, vp, vp, vp]
    lib.s1f_layer_norm_bwd.argtypes = [rp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.s1f_layer_norm_bwd_workspace_bytes.argtypes = [rp]
    lib.s1f_token_loss_fwd.argtypes = [rp, vp, vp, i64, i64, vp, i64, vp, vp, vp, sz, vp]
    lib.s1f_token_loss_bwd.argtypes = [rp, vp, vp, vp, i64, i64, vp, i64, vp, vp, vp, i64, i32, vp, sz, vp]
    lib.s1f_token_loss_fwd_workspace_bytes.argtypes = lib.s1f_token_loss_bwd_workspace_bytes.argtypes = [rp, i64, i64]
    for f in (lib.s1f_embed_fwd, lib.s1f_embed_bwd, lib.s1f_layer_norm_fwd, lib.s1f_layer_norm_bwd, lib.s1f_token_loss_fwd,
              lib.s1f_token_loss_bwd):
        f.restype = ctypes.c_int
    for f in (lib.s1f_embed_bwd_workspace_bytes, lib.s1f_layer_norm_bwd_workspace_bytes, lib.s1f_token_loss_fwd_workspace_bytes,
              lib.s1f_token_loss_bwd_workspace_bytes):
        f.restype = sz
    hp, f64 = ctypes.POINTER(Heads), ctypes.c_double
    turn = [vp, f32, vp, i64, i64, i64]                     # freqs, magnitude, positions, their stride, first_position, seg_off
    lib.s1f_rope_frequencies.argtypes = [i32, f64, i32, f64, i64, f64, f64, ctypes.POINTER(f64), ctypes.POINTER(f32)]
    lib.s1f_rope_fwd.argtypes = [hp, vp, vp, vp, *turn, vp, vp, vp, vp]
    lib.s1f_rope_bwd.argtypes = [hp, vp, vp, vp, *turn, vp, vp, vp, vp]
    lib.s1f_qk_norm_rope_fwd.argtypes = [hp, vp, vp, vp, vp, vp, f32, *turn, vp, vp, vp, vp]
    lib.s1f_qk_norm_rope_bwd.argtypes = [hp, vp, vp, vp, vp, vp, vp, vp, f32, *turn, vp, vp, vp, vp, vp, vp, sz, vp]
    for f in (lib.s1f_rope_frequencies, lib.s1f_rope_fwd, lib.s1f_rope_bwd, lib.s1f_qk_norm_rope_fwd, lib.s1f_qk_norm_rope_bwd):
        f.restype = ctypes.c_int
    lib.s1f_qk_norm_rope_bwd_workspace_bytes.argtypes = [hp]
    lib.s1f_qk_norm_rope_bwd_workspace_bytes.restype = sz
    lib.s1f_gated_ffn_fwd.argtypes = [rp, vp, vp, i64, vp, i64, i64, i32, vp, vp, vp, sz, vp]
    lib.s1f_gated_ffn_bwd.argtypes = [rp, vp, vp, vp, i64, vp, i64, i64, i32, vp, vp, vp, i64, vp, i64, i32, vp, sz, vp]
    lib.s1f_gated_ffn_fwd.restype = lib.s1f_gated_ffn_bwd.restype = ctypes.c_int
    for f in (lib.s1f_gated_ffn_fwd_workspace_bytes, lib.s1f_gated_ffn_bwd_workspace_bytes):
        f.argtypes, f.restype = [rp, i64, i64, i64], sz
    lib.s1f_seq1f1b_warmup.argtypes = [i32, i32, i32, i32, ctypes.POINTER(i64)]
    lib.s1f_seq1f1b_warmup.restype = ctypes.c_int
    lib.s1f_seq1f1b_order.argtypes = [i32, i32, i32, i32, ctypes.POINTER(Pass), i64, ctypes.POINTER(i64)]
    lib.s1f_seq1f1b_order.restype = ctypes.c_int
    lib.s1f_seq1f1b_interleaved_warmup.argtypes = [i32, i32, i32, i32, i32, ctypes.POINTER(i64)]
    lib.s1f_seq1f1b_interleaved_warmup.restype = ctypes.c_int
    lib.s1f_seq1f1b_interleaved_order.argtypes = [i32, i32, i32, i32, i32, ctypes.POINTER(StagePass), i64,
                                                  ctypes.POINTER(i64)]
    lib.s1f_seq1f1b_interleaved_order.restype = ctypes.c_int
    lib.s1f_seq1f1b_peak_memory_share.argtypes = [i32, i32, i32, i32, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.s1f_seq1f1b_peak_memory_share.restype = ctypes.c_int
    lib.s1f_pipeline_simulate.argtypes = [ctypes.POINTER(PipelineDesc), ctypes.POINTER(i64), ctypes.POINTER(i64),
                                          ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_double)]
    lib.s1f_pipeline_simulate.restype = ctypes.c_int
    lib.s1f_strerror.argtypes = [ctypes.c_int]
    lib.s1f_strerror.restype = ctypes.c_char_p
    lib.s1f_version.argtypes = []
    lib.s1f_version.restype = ctypes.c_int
    _lib = lib
    return lib


def strerror(status: int) -> str:
    return load_library().s1f_strerror(int(status)).decode()


def version() -> int:
    return int(load_library().s1f_version())


def partition(seq_len: int, n_seg: int, hidden: int, heads: int):
    """s1f_partition: list of n_seg + 1 boundaries."""
    lib = load_library()
    out = (ctypes.c_int64 * (max(int(n_seg), 0) + 1))()
    rc = lib.s1f_partition(int(seq_len), int(n_seg), int(hidden), int(heads), out)
    if rc != 0:
        raise S1FError(rc, "s1f_partition")
    return list(out)


COST_ADDITIVE, COST_LITERAL = 0, 1


def partition_ex(seq_len: int, n_seg: int, hidden: int, heads: int, cost_model: int = COST_ADDITIVE, align: int = 1):
    """s1f_partition_ex: list of n_seg + 1 boundaries under the chosen cost model and alignment."""
    out = (ctypes.c_int64 * (max(int(n_seg), 0) + 1))()
    rc = load_library().s1f_partition_ex(int(seq_len), int(n_seg), int(hidden), int(heads), int(cost_model),
                                         int(align), out)
    if rc != 0:
        raise S1FError(rc, "s1f_partition_ex")
    return list(out)


def partition_rebalance(boundaries, seg_cost, align: int = 1):
    """s1f_partition_rebalance: new boundaries from the measured integer cost of each segment."""
    k = len(boundaries) - 1
    if k < 1 or len(seg_cost) != k:
        raise S1FError(1, "s1f_partition_rebalance")
    b_in = (ctypes.c_int64 * (k + 1))(*[int(x) for x in boundaries])
    cost = (ctypes.c_int64 * k)(*[int(x) for x in seg_cost])
    out = (ctypes.c_int64 * (k + 1))()
    rc = load_library().s1f_partition_rebalance(k, b_in, cost, int(align), out)
    if rc != 0:
        raise S1FError(rc, "s1f_partition_rebalance")
    return list(out)


def seq1f1b_warmup(pp_size: int, device: int, n_micro: int, n_seg: int) -> int:
    """s1f_seq1f1b_warmup: sub-sequences forwarded before the first backward pass."""
    w = ctypes.c_int64(0)
    rc = load_library().s1f_seq1f1b_warmup(int(pp_size), int(device), int(n_micro), int(n_seg), ctypes.byref(w))
    if rc != 0:
        raise S1FError(rc, "s1f_seq1f1b_warmup")
    return int(w.value)


def seq1f1b_peak_memory_share(pp_size: int, device: int, n_micro: int, n_seg: int):
    """s1f_seq1f1b_peak_memory_share: (numerator, denominator) of w_i / sum_j w_j."""
    num, den = ctypes.c_int64(0), ctypes.c_int64(0)
    rc = load_library().s1f_seq1f1b_peak_memory_share(int(pp_size), int(device), int(n_micro), int(n_seg),
                                                      ctypes.byref(num), ctypes.byref(den))
    if rc != 0:
        raise S1FError(rc, "s1f_seq1f1b_peak_memory_share")
    return int(num.value), int(den.value)


def seq1f1b_order(pp_size: int, device: int, n_micro: int, n_seg: int):
    """s1f_seq1f1b_order: list of ("F" | "B", micro_batch, segment) in execution order."""
    lib = load_library()
    n = ctypes.c_int64(0)
    cap = 2 * max(int(n_micro), 0) * max(int(n_seg), 0)
    buf = (Pass * max(cap, 1))()
    rc = lib.s1f_seq1f1b_order(int(pp_size), int(device), int(n_micro), int(n_seg), buf, cap, ctypes.byref(n))
    if rc != 0:
        raise S1FError(rc, "s1f_seq1f1b_order")
    return [("B" if buf[i].backward else "F", int(buf[i].micro_batch), int(buf[i].segment)) for i in range(n.value)]


def seq1f1b_interleaved_warmup(pp_size: int, device: int, n_micro: int, n_seg: int, n_chunks: int) -> int:
    """s1f_seq1f1b_interleaved_warmup: sub-sequences forwarded before the first backward pass (Eq. 5-6)."""
    w = ctypes.c_int64(0)
    rc = load_library().s1f_seq1f1b_interleaved_warmup(int(pp_size), int(device), int(n_micro), int(n_seg),
                                                       int(n_chunks), ctypes.byref(w))
    if rc != 0:
        raise S1FError(rc, "s1f_seq1f1b_interleaved_warmup")
    return int(w.value)


def seq1f1b_interleaved_order(pp_size: int, device: int, n_micro: int, n_seg: int, n_chunks: int):
    """s1f_seq1f1b_interleaved_order: list of ("F" | "B", micro_batch, segment, chunk) in execution order."""
    n = ctypes.c_int64(0)
    cap = 2 * max(int(n_micro), 0) * max(int(n_seg), 0) * max(int(n_chunks), 0)
    buf = (StagePass * max(cap, 1))()
    rc = load_library().s1f_seq1f1b_interleaved_order(int(pp_size), int(device), int(n_micro), int(n_seg),
                                                      int(n_chunks), buf, cap, ctypes.byref(n))
    if rc != 0:
        raise S1FError(rc, "s1f_seq1f1b_interleaved_order")
    return [("B" if buf[i].kind else "F", int(buf[i].micro_batch), int(buf[i].segment), int(buf[i].chunk))
            for i in range(n.value)]


def pipeline_simulate(pp_size: int, n_micro: int, n_seg: int, n_chunks: int, t_fwd, t_bwd, t_wgrad=None,
                      t_comm: int = 0, max_pending_wgrad: int = 0, seg_tokens=None):
    """s1f_pipeline_simulate: dict with makespan, busy, peak_live, peak_pending (lists over devices) and
    bubble_ratio, all as the library returns them."""
    k, P = int(n_seg), int(pp_size)
    if k < 1 or P < 1 or len(t_fwd) != k or len(t_bwd) != k or (t_wgrad is not None and len(t_wgrad) != k) or (
            seg_tokens is not None and len(seg_tokens) != k):
        raise S1FError(1, "s1f_pipeline_simulate")
    arr = lambda xs: (ctypes.c_int64 * k)(*[int(x) for x in xs])
    keep = [arr(t_fwd), arr(t_bwd), arr(t_wgrad) if t_wgrad is not None else None,
            arr(seg_tokens) if seg_tokens is not None else None]
    desc = PipelineDesc(P, int(n_micro), k, int(n_chunks), 1 if t_wgrad is not None else 0, 0, int(max_pending_wgrad),
                        int(t_comm), keep[0], keep[1], keep[2], keep[3])
    span = ctypes.c_int64(0)
    busy, live, pend = ((ctypes.c_int64 * P)() for _ in range(3))
    bubble = ctypes.c_double(0.0)
    rc = load_library().s1f_pipeline_simulate(ctypes.byref(desc), ctypes.byref(span), busy, live, pend,
                                              ctypes.byref(bubble))
    if rc != 0:
        raise S1FError(rc, "s1f_pipeline_simulate")
    return {"makespan": int(span.value), "busy": list(busy), "peak_live": list(live), "peak_pending": list(pend),
            "bubble_ratio": float(bubble.value)}


def _dtype_code(t):
    import torch
    if t.dtype == torch.bfloat16:
        return S1F_BF16
    if t.dtype == torch.float32:
        return S1F_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def make_desc(q_like, kv_like) -> Desc:
    """Descriptor from a [B, Hq, S, D] query-shaped tensor and a [B, Hkv, C, D] prefix-shaped tensor."""
    qs, ks = q_like.stride(), kv_like.stride()
    if len(qs) != 4 or len(ks) != 4 or qs[3] != 1 or ks[3] != 1:
        raise ValueError("expected [batch, heads, seq, head_dim] tensors with contiguous head_dim")
    b, hq, _, d = q_like.shape
    _, hk, cap, _ = kv_like.shape
    return Desc(b, hq, hk, d, _dtype_code(q_like), 0, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], cap)


_raw_stream = None


def _stream_ptr():
    """torch's current stream on the current device, without building the Stream object around it (3 us of a call that
    launches one kernel takes 8)."""
    global _raw_stream
    import torch
    if _raw_stream is None:
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
    return _raw_stream(torch.cuda.current_device())


_calls, _calls_of = None, None


class _PythonForms:
    """In place of the compiled forms where they cannot be loaded: every call is left to the Python code."""
    fwd = fwd_ws = bwd = bwd_noalloc = append = emit = staticmethod(lambda *args: -1)
    embed_fwd = embed_bwd = layer_norm_fwd = layer_norm_bwd = token_loss_fwd = token_loss_bwd = fwd
    rope_fwd = rope_bwd = qk_norm_rope_fwd = qk_norm_rope_bwd = gated_ffn_fwd = gated_ffn_bwd = fwd


def _load_calls():
    """The module of the compiled forms.  It reads tensors by the layout that they have in the torch it was built against."""
    import torch
    try:
        from . import _torch_calls
        built_for = getattr(_torch_calls, "torch_version", None)
        if built_for != torch.__version__.split("+")[0]:
            raise ImportError(f"_torch_calls was built for torch {built_for}, this is {torch.__version__}")
        return _torch_calls
    except ImportError as e:
        warnings.warn(f"tensor calls in their Python forms, 8 to 12 us of host time each: {e}; "
                      "build with `python -m paper_2406_03488_amd.build`", RuntimeWarning, stacklevel=4)
        return None


def _native():
    """The compiled forms of the tensor calls below (csrc/torch_calls.cpp), bound to the loaded library.  They return a status,
    or -1 for arguments that are not the plain case, which the Python code then handles or refuses."""
    global _calls, _calls_of
    lib = _lib or load_library()
    if _calls_of is not lib:
        import torch
        _torch_calls = _load_calls()
        if _torch_calls is None:
            _calls, _calls_of = _PythonForms, lib
            return _calls
        entry = (lib.s1f_seg_attn_fwd, lib.s1f_seg_attn_fwd_ws, lib.s1f_seg_attn_bwd, lib.s1f_seg_attn_bwd_noalloc,
                 lib.s1f_kv_append, lib.s1f_kv_grad_emit, lib.s1f_embed_fwd, lib.s1f_embed_bwd, lib.s1f_layer_norm_fwd,
                 lib.s1f_layer_norm_bwd, lib.s1f_token_loss_fwd, lib.s1f_token_loss_bwd, lib.s1f_rope_fwd, lib.s1f_rope_bwd,
                 lib.s1f_qk_norm_rope_fwd, lib.s1f_qk_norm_rope_bwd, lib.s1f_gated_ffn_fwd, lib.s1f_gated_ffn_bwd)
        _torch_calls.bind(tuple(ctypes.cast(f, ctypes.c_void_p).value for f in entry), torch.cuda.current_device,
                          getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
                              lambda device: torch.cuda.current_stream(device).cuda_stream))
        _calls, _calls_of = _torch_calls, lib
    return _calls


def _done(rc, name):
    """True if the call has been made."""
    if rc > 0:
        raise S1FError(rc, name)
    return rc == 0


def _same_layout(ref, *others):
    shape, stride, dtype = ref.shape, ref.stride(), ref.dtype
    for t in others:
        if t.shape != shape or t.stride() != stride or t.dtype != dtype:
            raise ValueError("tensors sharing a stride set must have identical shape, strides and dtype")


def _check_covers(big, small, what):
    """The kernels take the number of batch entries and head_dim from `small` and address `big` with them; one that has more
    of either is read in part."""
    if big.shape[0] < small.shape[0] or big.shape[3] < small.shape[3]:
        raise ValueError(f"{what}: fewer batch entries or a smaller head_dim than the tensors it goes with")


def _check_prefix(k_prefix, q_seg):
    if k_prefix.dtype != q_seg.dtype:
        raise TypeError("queries and prefix must share the element type")
    _check_covers(k_prefix, q_seg, "k_prefix")


def seg_attn_fwd(q_seg, k_prefix, v_prefix, seg_off: int, out, lse):
    """s1f_seg_attn_fwd on torch device tensors.

    q_seg/out [B, Hq, seg_len, D]; k_prefix/v_prefix [B, Hkv, capacity, D] (row 0 of the cache);
    lse [B, Hq, seg_len] fp32 contiguous.  Enqueued on torch's current stream.
    """
    if _done(_native().fwd(q_seg, k_prefix, v_prefix, seg_off, out, lse), "s1f_seg_attn_fwd"):
        return
    lib = load_library()
    _same_layout(q_seg, out)
    _same_layout(k_prefix, v_prefix)
    _check_lse(lse, q_seg)
    desc = make_desc(q_seg, k_prefix)
    _check_prefix(k_prefix, q_seg)
    rc = lib.s1f_seg_attn_fwd(ctypes.byref(desc), q_seg.data_ptr(), k_prefix.data_ptr(), v_prefix.data_ptr(),
                              int(seg_off), int(q_seg.shape[2]), out.data_ptr(), lse.data_ptr(), _stream_ptr())
    if rc != 0:
        raise S1FError(rc, "s1f_seg_attn_fwd")


def fwd_workspace_bytes(q_seg, k_prefix, seg_off: int) -> int:
    desc = make_desc(q_seg, k_prefix)
    return int(load_library().s1f_fwd_workspace_bytes(ctypes.byref(desc), int(seg_off), int(q_seg.shape[2])))


PLAN_FWD, PLAN_FWD_WS, PLAN_DQ, PLAN_DKDV = range(4)


def launch_plan(q_seg, k_prefix, seg_off: int, launch: int):
    """s1f_launch_plan: (rows per unit, whole units, cut units, chunks per cut unit, units of a second launch)."""
    desc, plan = make_desc(q_seg, k_prefix), (ctypes.c_int64 * 5)()
    rc = load_library().s1f_launch_plan(ctypes.byref(desc), int(launch), int(seg_off), int(q_seg.shape[2]), plan)
    if rc != 0:
        raise S1FError(rc, "s1f_launch_plan")
    return tuple(plan)


def launch_paths(q_seg, k_prefix, seg_off: int):
    """s1f_launch_paths: (backward in one launch, rows per unit of its dQ half, dQ half first, one launch without a workspace,
    forward's tiles per head of partly filled units in the second launch)."""
    desc, paths = make_desc(q_seg, k_prefix), (ctypes.c_int64 * 5)()
    rc = load_library().s1f_launch_paths(ctypes.byref(desc), int(seg_off), int(q_seg.shape[2]), paths)
    if rc != 0:
        raise S1FError(rc, "s1f_launch_paths")
    return tuple(paths)


def seg_attn_fwd_ws(q_seg, k_prefix, v_prefix, seg_off: int, out, lse, workspace):
    """s1f_seg_attn_fwd_ws on torch device tensors: seg_attn_fwd with a device workspace of at least
    fwd_workspace_bytes(...) bytes (None is accepted when that is 0)."""
    if _done(_native().fwd_ws(q_seg, k_prefix, v_prefix, seg_off, out, lse, workspace), "s1f_seg_attn_fwd_ws"):
        return
    lib = load_library()
    _same_layout(q_seg, out)
    _same_layout(k_prefix, v_prefix)
    _check_lse(lse, q_seg)
    desc = make_desc(q_seg, k_prefix)
    _check_prefix(k_prefix, q_seg)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    rc = lib.s1f_seg_attn_fwd_ws(ctypes.byref(desc), q_seg.data_ptr(), k_prefix.data_ptr(), v_prefix.data_ptr(),
                                 int(seg_off), int(q_seg.shape[2]), out.data_ptr(), lse.data_ptr(), ws_ptr, ws_bytes,
                                 _stream_ptr())
    if rc != 0:
        raise S1FError(rc, "s1f_seg_attn_fwd_ws")


def bwd_workspace_bytes(q_seg, k_prefix, seg_off: int) -> int:
    desc = make_desc(q_seg, k_prefix)
    return int(load_library().s1f_bwd_workspace_bytes(ctypes.byref(desc), int(seg_off), int(q_seg.shape[2])))


def _check_lse(lse, q_seg):
    import torch
    if lse.dtype != torch.float32:
        raise TypeError("lse is fp32")
    if not lse.is_contiguous() or lse.shape != q_seg.shape[:3]:
        raise ValueError("lse must be a contiguous [B, Hq, seg_len] fp32 tensor")


def _check_acc(k_prefix, v_prefix, dk_prefix_acc, dv_prefix_acc):
    import torch
    _same_layout(k_prefix, v_prefix)
    _same_layout(dk_prefix_acc, dv_prefix_acc)
    if dk_prefix_acc.shape != k_prefix.shape or dk_prefix_acc.stride() != k_prefix.stride():
        raise ValueError("gradient accumulators must have the shape and strides of k_prefix")
    if dk_prefix_acc.dtype != torch.float32:
        raise TypeError("accumulators are fp32")


def _check_bwd_tensors(dout, q_seg, k_prefix, v_prefix, out, lse, dq, dk_prefix_acc, dv_prefix_acc):
    _same_layout(q_seg, dout, out, dq)
    _check_acc(k_prefix, v_prefix, dk_prefix_acc, dv_prefix_acc)
    _check_lse(lse, q_seg)


def seg_attn_bwd(dout, q_seg, k_prefix, v_prefix, out, lse, seg_off: int, dq, dk_prefix_acc, dv_prefix_acc, workspace):
    """s1f_seg_attn_bwd on torch device tensors.

    dk_prefix_acc/dv_prefix_acc are fp32 tensors with the shape and strides of k_prefix; workspace is any
    device tensor of at least bwd_workspace_bytes(...) bytes.
    """
    if _done(_native().bwd(dout, q_seg, k_prefix, v_prefix, out, lse, seg_off,
                           dq, dk_prefix_acc, dv_prefix_acc, workspace), "s1f_seg_attn_bwd"):
        return
    lib = load_library()
    _check_bwd_tensors(dout, q_seg, k_prefix, v_prefix, out, lse, dq, dk_prefix_acc, dv_prefix_acc)
    desc = make_desc(q_seg, k_prefix)
    _check_prefix(k_prefix, q_seg)
    rc = lib.s1f_seg_attn_bwd(ctypes.byref(desc), dout.data_ptr(), q_seg.data_ptr(), k_prefix.data_ptr(),
                              v_prefix.data_ptr(), out.data_ptr(), lse.data_ptr(), int(seg_off), int(q_seg.shape[2]),
                              dq.data_ptr(), dk_prefix_acc.data_ptr(), dv_prefix_acc.data_ptr(),
                              workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr())
    if rc != 0:
        raise S1FError(rc, "s1f_seg_attn_bwd")


def static_scratch_rows() -> int:
    return int(load_library().s1f_static_scratch_rows())


def seg_attn_bwd_noalloc(dout, q_seg, k_prefix, v_prefix, out, lse, seg_off: int, dq, dk_prefix_acc, dv_prefix_acc):
    """s1f_seg_attn_bwd_noalloc on torch device tensors: s1f_seg_attn_bwd without a workspace argument."""
    if _done(_native().bwd_noalloc(dout, q_seg, k_prefix, v_prefix, out, lse, seg_off,
                                   dq, dk_prefix_acc, dv_prefix_acc), "s1f_seg_attn_bwd_noalloc"):
        return
    lib = load_library()
    _check_bwd_tensors(dout, q_seg, k_prefix, v_prefix, out, lse, dq, dk_prefix_acc, dv_prefix_acc)
    desc = make_desc(q_seg, k_prefix)
    _check_prefix(k_prefix, q_seg)
    rc = lib.s1f_seg_attn_bwd_noalloc(ctypes.byref(desc), dout.data_ptr(), q_seg.data_ptr(), k_prefix.data_ptr(),
                                      v_prefix.data_ptr(), out.data_ptr(), lse.data_ptr(), int(seg_off),
                                      int(q_seg.shape[2]), dq.data_ptr(), dk_prefix_acc.data_ptr(),
                                      dv_prefix_acc.data_ptr(), _stream_ptr())
    if rc != 0:
        raise S1FError(rc, "s1f_seg_attn_bwd_noalloc")


def seg_attn_bwd_dq(dout, q_seg, k_prefix, v_prefix, out, lse, seg_off: int, dq, workspace):
    """s1f_seg_attn_bwd_dq: first half of the backward (dq, and delta into the workspace)."""
    lib = load_library()
    _same_layout(q_seg, dout, out, dq)
    _same_layout(k_prefix, v_prefix)
    _check_lse(lse, q_seg)
    desc = make_desc(q_seg, k_prefix)
    _check_prefix(k_prefix, q_seg)
    rc = lib.s1f_seg_attn_bwd_dq(ctypes.byref(desc), dout.data_ptr(), q_seg.data_ptr(), k_prefix.data_ptr(),
                                 v_prefix.data_ptr(), out.data_ptr(), lse.data_ptr(), int(seg_off),
                                 int(q_seg.shape[2]), dq.data_ptr(), workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream_ptr())
    if rc != 0:
        raise S1FError(rc, "s1f_seg_attn_bwd_dq")


def seg_attn_bwd_dkdv(dout, q_seg, k_prefix, v_prefix, lse, seg_off: int, dk_prefix_acc, dv_prefix_acc, workspace):
    """s1f_seg_attn_bwd_dkdv: second half of the backward (prefix dK/dV accumulation)."""
    lib = load_library()
    _same_layout(q_seg, dout)
    _check_acc(k_prefix, v_prefix, dk_prefix_acc, dv_prefix_acc)
    _check_lse(lse, q_seg)
    desc = make_desc(q_seg, k_prefix)
    _check_prefix(k_prefix, q_seg)
    rc = lib.s1f_seg_attn_bwd_dkdv(ctypes.byref(desc), dout.data_ptr(), q_seg.data_ptr(), k_prefix.data_ptr(),
                                   v_prefix.data_ptr(), lse.data_ptr(), int(seg_off), int(q_seg.shape[2]),
                                   dk_prefix_acc.data_ptr(), dv_prefix_acc.data_ptr(), workspace.data_ptr(),
                                   workspace.numel() * workspace.element_size(), _stream_ptr())
    if rc != 0:
        raise S1FError(rc, "s1f_seg_attn_bwd_dkdv")


def _kv_desc(cache) -> Desc:
    """Descriptor for the cache-side calls: only the kv_* fields, dtype, batch and head_dim are read."""
    s = cache.stride()
    if len(s) != 4 or s[3] != 1:
        raise ValueError("expected a [batch, kv_heads, capacity, head_dim] tensor with contiguous head_dim")
    b, h, cap, d = cache.shape
    return Desc(b, h, h, d, 0, 0, 0, 0, d, s[0], s[1], s[2], cap)


def _check_segment(seg, cache):
    _check_covers(seg, cache, "segment")
    if seg.shape[1] < cache.shape[1]:
        raise ValueError("segment: fewer heads than the cache")


def kv_append(k_seg, v_seg, seg_off: int, k_cache, v_cache):
    """s1f_kv_append: rows of the segment -> rows [seg_off, seg_off + seg_len) of the caches."""
    if _done(_native().append(k_seg, v_seg, seg_off, k_cache, v_cache), "s1f_kv_append"):
        return
    lib = load_library()
    _same_layout(k_seg, v_seg)
    _same_layout(k_cache, v_cache)
    desc = _kv_desc(k_cache)
    desc.dtype = _dtype_code(k_cache)
    s = k_seg.stride()
    if k_seg.dtype != k_cache.dtype or s[3] != 1:
        raise ValueError("segment and cache must share the element type; head_dim must be contiguous")
    _check_segment(k_seg, k_cache)
    rc = lib.s1f_kv_append(ctypes.byref(desc), k_seg.data_ptr(), v_seg.data_ptr(), s[0], s[1], s[2], int(seg_off),
                           k_seg.shape[2], k_cache.data_ptr(), v_cache.data_ptr(), _stream_ptr())
    if rc != 0:
        raise S1FError(rc, "s1f_kv_append")


def kv_grad_emit(dk_prefix_acc, dv_prefix_acc, seg_off: int, dk_seg, dv_seg):
    """s1f_kv_grad_emit: final rows [seg_off, seg_off + seg_len) of the fp32 accumulators -> dk_seg, dv_seg."""
    if _done(_native().emit(dk_prefix_acc, dv_prefix_acc, seg_off, dk_seg, dv_seg), "s1f_kv_grad_emit"):
        return
    import torch
    lib = load_library()
    _same_layout(dk_prefix_acc, dv_prefix_acc)
    _same_layout(dk_seg, dv_seg)
    s = dk_seg.stride()
    if dk_prefix_acc.dtype != torch.float32 or s[3] != 1:
        raise ValueError("accumulators must be fp32; head_dim must be contiguous")
    desc = _kv_desc(dk_prefix_acc)
    _check_segment(dk_seg, dk_prefix_acc)
    desc.dtype = _dtype_code(dk_seg)
    rc = lib.s1f_kv_grad_emit(ctypes.byref(desc), dk_prefix_acc.data_ptr(), dv_prefix_acc.data_ptr(), int(seg_off),
                              dk_seg.shape[2], dk_seg.data_ptr(), dv_seg.data_ptr(), s[0], s[1], s[2], _stream_ptr())
    if rc != 0:
        raise S1FError(rc, "s1f_kv_grad_emit")


# ---- heads on their way from the projections to the attention, and back --------------------------------------------------------------

ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_PARTS = range(4)


def rope_frequencies(rotary_dim: int, base: float = 10000.0, scaling: int = ROPE_PLAIN, factor: float = 1.0, trained_rows: int = 0,
                     slow_turns: float = 1.0, fast_turns: float = 32.0):
    """s1f_rope_frequencies: (list of the rotary_dim / 2 frequencies in radians per token, magnitude).  The rotations take the
    frequencies as an fp64 tensor on their device."""
    out, magnitude = (ctypes.c_double * max(int(rotary_dim) // 2, 1))(), ctypes.c_float(0.0)
    rc = load_library().s1f_rope_frequencies(int(rotary_dim), float(base), int(scaling), float(factor), int(trained_rows), float(slow_turns),
                                             float(fast_turns), out, ctypes.byref(magnitude))
    if rc != 0:
        raise S1FError(rc, "s1f_rope_frequencies")
    return list(out), float(magnitude.value)


def _head_strides(t):
    """(batch, head, row) strides of a [batch, heads, rows, head_dim] tensor, 0 where it has one of them."""
    return tuple(t.stride(i) if t.shape[i] > 1 else 0 for i in range(3))


def _head_shape(t, shape, dtype, what):
    if t.dim() != 4 or (t.stride(3) != 1 and t.shape[3] > 1):
        raise ValueError(f"{what}: expected [batch, heads, rows, head_dim] with contiguous head_dim")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: expected {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{what}: expected {dtype}, got {t.dtype}")


def _heads_desc(q, q_rot, kv, caches, gradients, freqs, interleaved) -> Heads:
    """Descriptor of a call on q and kv (k and v, or their gradients; v may be None) on one side, q_rot and caches on the other; with
    `gradients` the caches are fp32 accumulators."""
    import torch
    if q.dim() != 4 or kv[0].dim() != 4 or caches[0].dim() != 4:
        raise ValueError("expected [batch, heads, rows, head_dim] tensors")
    if (kv[1] is None) != (caches[1] is None):
        raise ValueError("values need a place to go to, or neither is given")
    b, hq, n, d = q.shape
    hk, capacity = kv[0].shape[1], caches[0].shape[2]
    _head_shape(q, q.shape, q.dtype, "queries")
    _head_shape(q_rot, q.shape, q.dtype, "queries")
    for t in kv:
        if t is not None:
            _head_shape(t, (b, hk, n, d), q.dtype, "keys and values")
            if _head_strides(t) != _head_strides(kv[0]):
                raise ValueError("keys and values must have identical strides")
    for t in caches:
        if t is not None:
            _head_shape(t, (b, hk, capacity, d), torch.float32 if gradients else q.dtype, "accumulators" if gradients else "caches")
            if _head_strides(t) != _head_strides(caches[0]):
                raise ValueError("caches must have identical strides")
    if freqs.dtype != torch.float64:
        raise TypeError("frequencies are fp64")
    if freqs.dim() != 1 or not freqs.is_contiguous() or 2 * freqs.shape[0] > d:
        raise ValueError("frequencies must be a contiguous vector, one for each pair of a head")
    return Heads(b, hq, hk, d, _dtype_code(q), 2 * freqs.shape[0], 1 if interleaved else 0, 0, n, *_head_strides(q), *_head_strides(kv[0]),
                 *_head_strides(q_rot), *_head_strides(caches[0]), capacity)


def _turn(q, freqs, magnitude, positions, seg_off):
    """The arguments between a call's inputs and its outputs.  positions: [batch, rows] int64, or the first row's."""
    import torch
    if isinstance(positions, torch.Tensor):
        if positions.dtype != torch.int64:
            raise TypeError("positions are int64")
        if positions.shape != (q.shape[0], q.shape[2]) or (positions.shape[1] > 1 and positions.stride(1) != 1):
            raise ValueError("positions must be [batch, rows] with contiguous rows")
        at, sb, first = positions.data_ptr(), positions.stride(0) if positions.shape[0] > 1 else 0, 0
    else:
        at, sb, first = None, 0, int(positions)
        if not -2 ** 62 < first < 2 ** 62:
            raise ValueError("position out of range")
    return freqs.data_ptr() or None, float(magnitude), at, sb, first, int(seg_off)


def _on_device(*tensors):
    """The tensors among a call's arguments."""
    import torch
    _check_device(*[t for t in tensors if isinstance(t, torch.Tensor)])


def _ptr(t):
    return None if t is None else t.data_ptr()


def rope_fwd(q, k, v, freqs, magnitude: float, interleaved: bool, positions, seg_off: int, q_rot, k_cache, v_cache):
    """s1f_rope_fwd on torch device tensors: q rotated into q_rot, k rotated and v as it is into rows [seg_off, seg_off + rows) of the caches.

    q, q_rot [B, Hq, rows, D]; k, v [B, Hkv, rows, D]; k_cache, v_cache [B, Hkv, capacity, D]; v and v_cache may both be None; freqs fp64, one
    per pair (rope_frequencies); positions [B, rows] int64 on the device, or an integer: the first row's.  Enqueued on torch's current stream.
    """
    if _done(_native().rope_fwd(q, k, v, freqs, magnitude, interleaved, positions, seg_off, q_rot, k_cache, v_cache), "s1f_rope_fwd"):
        return
    _on_device(q, k, v, freqs, positions, q_rot, k_cache, v_cache)
    desc = _heads_desc(q, q_rot, (k, v), (k_cache, v_cache), False, freqs, interleaved)
    _checked(load_library().s1f_rope_fwd(ctypes.byref(desc), q.data_ptr(), k.data_ptr(), _ptr(v), *_turn(q, freqs, magnitude, positions, seg_off),
                                         q_rot.data_ptr(), k_cache.data_ptr(), _ptr(v_cache), _stream_ptr()), "s1f_rope_fwd")


def rope_bwd(dq_rot, dk_prefix_acc, dv_prefix_acc, freqs, magnitude: float, interleaved: bool, positions, seg_off: int, dq, dk, dv):
    """s1f_rope_bwd on torch device tensors: dq_rot, and rows [seg_off, seg_off + rows) of the fp32 accumulators [B, Hkv, capacity, D], back to
    dq, dk, dv (shaped like q, k, v; overwritten); dv_prefix_acc and dv may both be None."""
    if _done(_native().rope_bwd(dq_rot, dk_prefix_acc, dv_prefix_acc, freqs, magnitude, interleaved, positions, seg_off, dq, dk, dv), "s1f_rope_bwd"):
        return
    _on_device(dq_rot, dk_prefix_acc, dv_prefix_acc, freqs, positions, dq, dk, dv)
    desc = _heads_desc(dq, dq_rot, (dk, dv), (dk_prefix_acc, dv_prefix_acc), True, freqs, interleaved)
    _checked(load_library().s1f_rope_bwd(ctypes.byref(desc), dq_rot.data_ptr(), dk_prefix_acc.data_ptr(), _ptr(dv_prefix_acc),
                                         *_turn(dq, freqs, magnitude, positions, seg_off), dq.data_ptr(), dk.data_ptr(), _ptr(dv), _stream_ptr()),
             "s1f_rope_bwd")


def qk_norm_rope_fwd(q, k, v, q_gain, k_gain, eps: float, freqs, magnitude: float, interleaved: bool, positions, seg_off: int, q_rot, k_cache, v_cache):
    """s1f_qk_norm_rope_fwd on torch device tensors: rope_fwd of q and k with every head divided by its root mean square and multiplied by q_gain or
    k_gain [D], of the tensors' type."""
    if _done(_native().qk_norm_rope_fwd(q, k, v, q_gain, k_gain, eps, freqs, magnitude, interleaved, positions, seg_off, q_rot, k_cache, v_cache),
             "s1f_qk_norm_rope_fwd"):
        return
    _on_device(q, k, v, q_gain, k_gain, freqs, positions, q_rot, k_cache, v_cache)
    desc = _heads_desc(q, q_rot, (k, v), (k_cache, v_cache), False, freqs, interleaved)
    _vectors(q.shape[3], q.dtype, q_gain, k_gain)
    _checked(load_library().s1f_qk_norm_rope_fwd(ctypes.byref(desc), q.data_ptr(), k.data_ptr(), _ptr(v), q_gain.data_ptr(), k_gain.data_ptr(), float(eps),
                                                 *_turn(q, freqs, magnitude, positions, seg_off), q_rot.data_ptr(), k_cache.data_ptr(), _ptr(v_cache),
                                                 _stream_ptr()), "s1f_qk_norm_rope_fwd")


def qk_norm_rope_bwd_workspace_bytes(dq_rot, dk_prefix_acc) -> int:
    b, hq, n, d = dq_rot.shape
    desc = Heads(b, hq, dk_prefix_acc.shape[1], d, _dtype_code(dq_rot), 0, 0, 0, n, *[1 << 30] * 12, n)
    return int(load_library().s1f_qk_norm_rope_bwd_workspace_bytes(ctypes.byref(desc)))


def qk_norm_rope_bwd(dq_rot, dk_prefix_acc, dv_prefix_acc, q, k, q_gain, k_gain, eps: float, freqs, magnitude: float, interleaved: bool, positions,
                     seg_off: int, dq, dk, dv, dq_gain_acc, dk_gain_acc, workspace):
    """s1f_qk_norm_rope_bwd on torch device tensors: rope_bwd behind which the gradients pass the norm.  q, k as the forward took them, with the strides of
    dq and dk; dq_gain_acc, dk_gain_acc [D] fp32 are added to; workspace is any device tensor of at least qk_norm_rope_bwd_workspace_bytes(...) bytes."""
    if _done(_native().qk_norm_rope_bwd(dq_rot, dk_prefix_acc, dv_prefix_acc, q, k, q_gain, k_gain, eps, freqs, magnitude, interleaved, positions, seg_off,
                                        dq, dk, dv, dq_gain_acc, dk_gain_acc, workspace), "s1f_qk_norm_rope_bwd"):
        return
    import torch
    _on_device(dq_rot, dk_prefix_acc, dv_prefix_acc, q, k, q_gain, k_gain, freqs, positions, dq, dk, dv, dq_gain_acc, dk_gain_acc, workspace)
    desc = _heads_desc(dq, dq_rot, (dk, dv), (dk_prefix_acc, dv_prefix_acc), True, freqs, interleaved)
    for t, like in ((q, dq), (k, dk)):
        _head_shape(t, like.shape, like.dtype, "queries and keys")
        if _head_strides(t) != _head_strides(like):
            raise ValueError("gradients must have the strides of what they are the gradients of")
    _vectors(dq.shape[3], dq.dtype, q_gain, k_gain)
    _vectors(dq.shape[3], torch.float32, dq_gain_acc, dk_gain_acc)
    _checked(load_library().s1f_qk_norm_rope_bwd(ctypes.byref(desc), dq_rot.data_ptr(), dk_prefix_acc.data_ptr(), _ptr(dv_prefix_acc), q.data_ptr(),
                                                 k.data_ptr(), q_gain.data_ptr(), k_gain.data_ptr(), float(eps),
                                                 *_turn(dq, freqs, magnitude, positions, seg_off), dq.data_ptr(), dk.data_ptr(), _ptr(dv),
                                                 dq_gain_acc.data_ptr(), dk_gain_acc.data_ptr(), *_space(workspace), _stream_ptr()),
             "s1f_qk_norm_rope_bwd")


# ---- rows of hidden states: embedding, layer norm, token loss ---------------------------------------------------------------------

def _strides(t):
    """(batch, row) strides of a [batch, rows, hidden] tensor.  torch gives a dimension of one element any stride: such a one is
    not used, and 0 here."""
    s = t.stride()
    return (s[0] if t.shape[0] > 1 else 0, s[1] if t.shape[1] > 1 else 0)


def _rows_desc(x=None, y=None) -> Rows:
    """Descriptor from [batch, rows, hidden] tensors on either side of a call."""
    a = y if x is None else x
    for t in (x, y):
        if t is None:
            continue
        if t.dim() != 3 or (t.stride(2) != 1 and t.shape[2] > 1):
            raise ValueError("expected [batch, rows, hidden] tensors with contiguous hidden")
        if t.shape != a.shape:
            raise ValueError("tensors of a call must have the same [batch, rows, hidden]")
        if t.dtype != a.dtype:
            raise TypeError("tensors of a call must share the element type")
    b, n, h = a.shape
    return Rows(b, h, _dtype_code(a), 0, n, *(_strides(x) if x is not None else (0, 0)), *(_strides(y) if y is not None else (0, 0)))


def _same_rows(ref, other):
    """Two tensors of one side of a call."""
    if other.shape != ref.shape or _strides(other) != _strides(ref) or (other.stride(2) != 1 and other.shape[2] > 1):
        raise ValueError("tensors of one side of a call must have identical shape and strides")
    if other.dtype != ref.dtype:
        raise TypeError("tensors of a call must share the element type")


def _check_device(*tensors):
    """All on the current device: the call runs on its stream."""
    import torch
    device = tensors[0].device
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError("all tensors of a call must be on the same device")
    if device.type != "cuda":
        raise ValueError(f"expected tensors in device memory, got {device}")
    if device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}, the current device is {torch.cuda.current_device()}")


def _tokens(t, like):
    """Pointer and batch stride of [batch, rows] int64 tokens."""
    import torch
    if t.dtype != torch.int64:
        raise TypeError("tokens are int64")
    if t.shape != like.shape[:2] or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("tokens must be [batch, rows] with contiguous rows")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else 0


def _row_values(like, *values):
    import torch
    for v in values:
        if v.dtype != torch.float32:
            raise TypeError("per-row values are fp32")
        if not v.is_contiguous() or v.shape != like.shape[:2]:
            raise ValueError("per-row values must be contiguous [batch, rows] tensors")


def _matrix(t, hidden, dtype, what):
    """Row stride of a [vocab, hidden] tensor."""
    if t.dtype != dtype:
        raise TypeError(f"{what}: expected {dtype}")
    if t.dim() != 2 or t.shape[1] != hidden or (t.stride(1) != 1 and hidden > 1):
        raise ValueError(f"{what} must be [vocab, hidden] with contiguous hidden")
    return t.stride(0) if t.shape[0] > 1 else hidden


def _vectors(hidden, dtype, *vectors):
    for v in vectors:
        if v.dtype != dtype:
            raise TypeError(f"expected a vector of {dtype}")
        if v.shape != (hidden,) or not v.is_contiguous():
            raise ValueError("expected contiguous [hidden] vectors")


def _space(workspace):
    """Pointer and bytes of a workspace, or of none."""
    if workspace is None:
        return None, 0
    if not workspace.is_contiguous():
        raise ValueError("a workspace must be contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _checked(rc, name):
    if rc != 0:
        raise S1FError(rc, name)


def embed_fwd(ids, table, scale: float, out):
    """s1f_embed_fwd on torch device tensors: out[b, r] = scale * table[ids[b, r]], zeros where the token is outside the table.

    ids [B, rows] int64; table [vocab, hidden]; out [B, rows, hidden] of the table's type.  Enqueued on torch's current stream.
    """
    if _done(_native().embed_fwd(ids, table, scale, out), "s1f_embed_fwd"):
        return
    _check_device(out, ids, table)
    desc = _rows_desc(y=out)
    at, ids_sb = _tokens(ids, out)
    stride = _matrix(table, out.shape[2], out.dtype, "table")
    _checked(load_library().s1f_embed_fwd(ctypes.byref(desc), at, ids_sb, table.data_ptr(), stride, table.shape[0], float(scale),
                                          out.data_ptr(), _stream_ptr()), "s1f_embed_fwd")


def embed_bwd_workspace_bytes(ids, dout, dtable_acc) -> int:
    return int(load_library().s1f_embed_bwd_workspace_bytes(ctypes.byref(_rows_desc(y=dout)), dtable_acc.shape[0]))


def embed_bwd(ids, dout, scale: float, dtable_acc, workspace):
    """s1f_embed_bwd on torch device tensors: adds scale times the rows of dout to the fp32 rows of dtable_acc [vocab, hidden] that
    their tokens name; workspace is any device tensor of at least embed_bwd_workspace_bytes(...) bytes."""
    if _done(_native().embed_bwd(ids, dout, scale, dtable_acc, workspace), "s1f_embed_bwd"):
        return
    import torch
    _check_device(dout, ids, dtable_acc, workspace)
    desc = _rows_desc(y=dout)
    at, ids_sb = _tokens(ids, dout)
    stride = _matrix(dtable_acc, dout.shape[2], torch.float32, "dtable_acc")
    _checked(load_library().s1f_embed_bwd(ctypes.byref(desc), at, ids_sb, dout.data_ptr(), dtable_acc.shape[0], float(scale),
                                          dtable_acc.data_ptr(), stride, *_space(workspace), _stream_ptr()), "s1f_embed_bwd")


def layer_norm_fwd(x, gamma, beta, eps: float, y, mean, rstd):
    """s1f_layer_norm_fwd on torch device tensors: x, y [B, rows, hidden]; gamma, beta [hidden] of their type; mean, rstd
    [B, rows] fp32, overwritten.  Enqueued on torch's current stream."""
    if _done(_native().layer_norm_fwd(x, gamma, beta, eps, y, mean, rstd), "s1f_layer_norm_fwd"):
        return
    _check_device(x, gamma, beta, y, mean, rstd)
    desc = _rows_desc(x, y)
    _vectors(x.shape[2], x.dtype, gamma, beta)
    _row_values(x, mean, rstd)
    _checked(load_library().s1f_layer_norm_fwd(ctypes.byref(desc), x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), float(eps), y.data_ptr(),
                                               mean.data_ptr(), rstd.data_ptr(), _stream_ptr()), "s1f_layer_norm_fwd")


def layer_norm_bwd_workspace_bytes(dy, x) -> int:
    return int(load_library().s1f_layer_norm_bwd_workspace_bytes(ctypes.byref(_rows_desc(x, dy))))


def layer_norm_bwd(dy, x, gamma, mean, rstd, dx, dgamma_acc, dbeta_acc, workspace):
    """s1f_layer_norm_bwd on torch device tensors: dx, with the shape and strides of x, is overwritten; dgamma_acc and dbeta_acc
    [hidden] fp32 are added to; workspace is any device tensor of at least layer_norm_bwd_workspace_bytes(...) bytes."""
    if _done(_native().layer_norm_bwd(dy, x, gamma, mean, rstd, dx, dgamma_acc, dbeta_acc, workspace), "s1f_layer_norm_bwd"):
        return
    import torch
    _check_device(dy, x, gamma, mean, rstd, dx, dgamma_acc, dbeta_acc, workspace)
    desc = _rows_desc(x, dy)
    _same_rows(x, dx)
    _vectors(x.shape[2], x.dtype, gamma)
    _vectors(x.shape[2], torch.float32, dgamma_acc, dbeta_acc)
    _row_values(x, mean, rstd)
    _checked(load_library().s1f_layer_norm_bwd(ctypes.byref(desc), dy.data_ptr(), x.data_ptr(), gamma.data_ptr(), mean.data_ptr(),
                                               rstd.data_ptr(), dx.data_ptr(), dgamma_acc.data_ptr(), dbeta_acc.data_ptr(),
                                               *_space(workspace), _stream_ptr()), "s1f_layer_norm_bwd")


def token_loss_fwd_workspace_bytes(x, weight) -> int:
    stride = _matrix(weight, x.shape[2], x.dtype, "weight")
    return int(load_library().s1f_token_loss_fwd_workspace_bytes(ctypes.byref(_rows_desc(x)), weight.shape[0], stride))


def token_loss_fwd(x, weight, targets, loss, lse, workspace):
    """s1f_token_loss_fwd on torch device tensors: cross entropy of every row of x [B, rows, hidden] over the scores x weight^T,
    weight [vocab, hidden].

    targets [B, rows] int64 (outside [0, vocab): the row takes no part); loss, lse [B, rows] fp32, overwritten; workspace is any device
    tensor of at least token_loss_fwd_workspace_bytes(...) bytes.  Enqueued on torch's current stream.
    """
    if _done(_native().token_loss_fwd(x, weight, targets, loss, lse, workspace), "s1f_token_loss_fwd"):
        return
    _check_device(x, weight, targets, loss, lse, workspace)
    desc = _rows_desc(x)
    stride = _matrix(weight, x.shape[2], x.dtype, "weight")
    at, targets_sb = _tokens(targets, x)
    _row_values(x, loss, lse)
    _checked(load_library().s1f_token_loss_fwd(ctypes.byref(desc), x.data_ptr(), weight.data_ptr(), stride, weight.shape[0], at, targets_sb,
                                               loss.data_ptr(), lse.data_ptr(), *_space(workspace), _stream_ptr()), "s1f_token_loss_fwd")


def token_loss_bwd_workspace_bytes(x, weight) -> int:
    stride = _matrix(weight, x.shape[2], x.dtype, "weight")
    return int(load_library().s1f_token_loss_bwd_workspace_bytes(ctypes.byref(_rows_desc(x)), weight.shape[0], stride))


def token_loss_bwd(dloss, x, weight, targets, lse, dx, dweight, workspace):
    """s1f_token_loss_bwd on torch device tensors.

    dloss, lse [B, rows] fp32; dx, with the shape and strides of x, is overwritten; dweight [vocab, hidden] is added to if it is fp32 and
    overwritten if it is bf16 (bf16 rows only); workspace is any device tensor of at least token_loss_bwd_workspace_bytes(...) bytes.
    """
    if _done(_native().token_loss_bwd(dloss, x, weight, targets, lse, dx, dweight, workspace), "s1f_token_loss_bwd"):
        return
    _check_device(dloss, x, weight, targets, lse, dx, dweight, workspace)
    desc = _rows_desc(x)
    _same_rows(x, dx)
    stride = _matrix(weight, x.shape[2], x.dtype, "weight")
    code = _dtype_code(dweight)
    into = _matrix(dweight, x.shape[2], dweight.dtype, "dweight")
    if dweight.shape != weight.shape:
        raise ValueError("dweight must have the shape of weight")
    at, targets_sb = _tokens(targets, x)
    _row_values(x, dloss, lse)
    _checked(load_library().s1f_token_loss_bwd(ctypes.byref(desc), dloss.data_ptr(), x.data_ptr(), weight.data_ptr(), stride,
                                               weight.shape[0], at, targets_sb, lse.data_ptr(), dx.data_ptr(), dweight.data_ptr(), into,
                                               code, *_space(workspace), _stream_ptr()), "s1f_token_loss_bwd")


SILU, GELU, GELU_TANH = range(3)


def _ffn_weights(x, w_in, w_out, what=("w_in", "w_out"), dtype=None):
    """(inner, row strides of w_in [2 * inner, hidden] and w_out [hidden, inner])"""
    hidden, dtype = x.shape[2], dtype or x.dtype
    in_stride = _matrix(w_in, hidden, dtype, what[0])
    if w_in.shape[0] % 2 != 0:
        raise ValueError(f"{what[0]} must be [2 * inner, hidden]")
    inner = w_in.shape[0] // 2
    if w_out.dim() != 2 or w_out.shape[0] != hidden:
        raise ValueError(f"{what[1]} must be [hidden, inner]")
    return inner, in_stride, _matrix(w_out, inner, dtype, what[1])


def _check_gate_up(gate_up, x, inner):
    if gate_up.dtype != x.dtype:
        raise TypeError("gate_up must share the element type")
    if not gate_up.is_contiguous() or gate_up.shape != (*x.shape[:2], 2 * inner):
        raise ValueError("gate_up must be a contiguous [batch, rows, 2 * inner] tensor")


def gated_ffn_fwd_workspace_bytes(x, w_in, w_out) -> int:
    return int(load_library().s1f_gated_ffn_fwd_workspace_bytes(ctypes.byref(_rows_desc(x, x)), *_ffn_weights(x, w_in, w_out)))


def gated_ffn_fwd(x, w_in, w_out, act: int, y, gate_up, workspace):
    """s1f_gated_ffn_fwd on torch device tensors: y = (act(g) * u) w_out^T with [g | u] = x w_in^T.

    x, y [B, rows, hidden]; w_in [2 * inner, hidden], g's rows first; w_out [hidden, inner]; act SILU, GELU or GELU_TANH; gate_up [B, rows, 2 * inner]
    is overwritten with [g | u] for the backward, None: not kept; workspace is any device tensor of at least gated_ffn_fwd_workspace_bytes(...)
    bytes; y may be x.  Enqueued on torch's current stream.
    """
    if _done(_native().gated_ffn_fwd(x, w_in, w_out, act, y, gate_up, workspace), "s1f_gated_ffn_fwd"):
        return
    _on_device(x, w_in, w_out, y, gate_up, workspace)
    desc = _rows_desc(x, y)
    inner, in_stride, out_stride = _ffn_weights(x, w_in, w_out)
    if gate_up is not None:
        _check_gate_up(gate_up, x, inner)
    _checked(load_library().s1f_gated_ffn_fwd(ctypes.byref(desc), x.data_ptr(), w_in.data_ptr(), in_stride, w_out.data_ptr(), out_stride, inner, int(act),
                                              y.data_ptr(), _ptr(gate_up), *_space(workspace), _stream_ptr()), "s1f_gated_ffn_fwd")


def gated_ffn_bwd_workspace_bytes(dy, x, w_in, w_out) -> int:
    return int(load_library().s1f_gated_ffn_bwd_workspace_bytes(ctypes.byref(_rows_desc(x, dy)), *_ffn_weights(x, w_in, w_out)))


def gated_ffn_bwd(dy, x, w_in, w_out, act: int, gate_up, dx, dw_in, dw_out, workspace):
    """s1f_gated_ffn_bwd on torch device tensors, from the gate_up that the forward has kept.

    dx, with the shape and strides of x, is overwritten; dw_in and dw_out, of one type, are added to if they are fp32 and overwritten if they are bf16 (bf16 rows only);
    workspace is any device tensor of at least gated_ffn_bwd_workspace_bytes(...) bytes; dx may be x or dy.
    """
    if _done(_native().gated_ffn_bwd(dy, x, w_in, w_out, act, gate_up, dx, dw_in, dw_out, workspace), "s1f_gated_ffn_bwd"):
        return
    _on_device(dy, x, w_in, w_out, gate_up, dx, dw_in, dw_out, workspace)
    desc = _rows_desc(x, dy)
    _same_rows(x, dx)
    inner, in_stride, out_stride = _ffn_weights(x, w_in, w_out)
    code = _dtype_code(dw_in)
    into, dw_in_stride, dw_out_stride = _ffn_weights(x, dw_in, dw_out, ("dw_in", "dw_out"), dw_in.dtype)
    if into != inner:
        raise ValueError("dw_in and dw_out must have the shapes of w_in and w_out")
    _check_gate_up(gate_up, x, inner)
    _checked(load_library().s1f_gated_ffn_bwd(ctypes.byref(desc), dy.data_ptr(), x.data_ptr(), w_in.data_ptr(), in_stride, w_out.data_ptr(), out_stride, inner,
                                              int(act), gate_up.data_ptr(), dx.data_ptr(), dw_in.data_ptr(), dw_in_stride, dw_out.data_ptr(),
                                              dw_out_stride, code, *_space(workspace), _stream_ptr()), "s1f_gated_ffn_bwd")
