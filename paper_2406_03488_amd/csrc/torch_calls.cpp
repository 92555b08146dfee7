// The tensor calls of binding.py without the interpreter: checks the arguments as the Python functions do, fills the descriptor and
// calls the C ABI.  A function returns the call's status, or -1 for whatever is not the plain case (a tensor subclass, a mode
// that intercepts tensor functions, a tensor of another device, any argument the Python code would refuse): the
// caller then takes the Python path, which raises what it always raised.
// Why: a call of the Python path costs 8 to 12 us of host time in attribute look-ups and conversions, more than its launches;
// steps of small segments were bound by it (2 x 1357
// tokens in 4 segments, bf16, head_dim 64, with the cache calls: 18 calls, 218 us a step; now 159, bound by the kernels).
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <torch/version.h>

#include <cstring>

#include "s1f.h"

namespace {

// Entry points of the library that binding.py has loaded, and torch's current device and stream.
struct Api {
  decltype(&s1f_seg_attn_fwd) fwd;
  decltype(&s1f_seg_attn_fwd_ws) fwd_ws;
  decltype(&s1f_seg_attn_bwd) bwd;
  decltype(&s1f_seg_attn_bwd_noalloc) bwd_noalloc;
  decltype(&s1f_kv_append) append;
  decltype(&s1f_kv_grad_emit) emit;
  decltype(&s1f_embed_fwd) embed_fwd;
  decltype(&s1f_embed_bwd) embed_bwd;
  decltype(&s1f_layer_norm_fwd) layer_norm_fwd;
  decltype(&s1f_layer_norm_bwd) layer_norm_bwd;
  decltype(&s1f_token_loss_fwd) token_loss_fwd;
  decltype(&s1f_token_loss_bwd) token_loss_bwd;
  decltype(&s1f_rope_fwd) rope_fwd;
  decltype(&s1f_rope_bwd) rope_bwd;
  decltype(&s1f_qk_norm_rope_fwd) qk_norm_rope_fwd;
  decltype(&s1f_qk_norm_rope_bwd) qk_norm_rope_bwd;
  decltype(&s1f_gated_ffn_fwd) gated_ffn_fwd;
  decltype(&s1f_gated_ffn_bwd) gated_ffn_bwd;
};
Api api = {};
PyObject *get_device = nullptr, *get_stream = nullptr;

constexpr int kPython = -1;

// A plain tensor of the current kind of device, or null.
const at::Tensor *plain(PyObject *x) {
  if (!THPVariable_CheckExact(x)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(x);
  return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}

struct Args {
  const at::Tensor *t[10];
  int64_t off = 0;
  void *stream = nullptr;
  // n arguments; number `off_at` is the offset, number `optional` may be None (then a null pointer)
  bool read(PyObject *const *args, Py_ssize_t n, Py_ssize_t want, Py_ssize_t off_at, Py_ssize_t optional) {
    if (n != want || get_device == nullptr || at::impl::PythonTorchFunctionTLS::stack_len() > 0) return false;
    for (Py_ssize_t i = 0, k = 0; i < n; ++i) {
      if (i == off_at) {
        int overflow = 0;
        if (!PyLong_CheckExact(args[i])) return false;
        off = PyLong_AsLongLongAndOverflow(args[i], &overflow);
        if (overflow != 0) return false;
        continue;
      }
      t[k] = i == optional && args[i] == Py_None ? nullptr : plain(args[i]);
      if (t[k] == nullptr && !(i == optional && args[i] == Py_None)) return false;
      ++k;
    }
    return true;
  }
  bool read_stream() {
    PyObject *dev = PyObject_CallNoArgs(get_device);
    PyObject *st = dev ? PyObject_CallOneArg(get_stream, dev) : nullptr;
    Py_XDECREF(dev);
    if (st == nullptr) return PyErr_Clear(), false;
    stream = PyLong_AsVoidPtr(st);
    Py_DECREF(st);
    return PyErr_Occurred() == nullptr || (PyErr_Clear(), false);
  }
};

bool same_layout(const at::Tensor &a, const at::Tensor &b) {
  return a.sizes() == b.sizes() && a.strides() == b.strides() && a.scalar_type() == b.scalar_type();
}
bool rows_of(const at::Tensor &t) { return t.dim() == 4 && t.stride(3) == 1; }
bool dtype_of(const at::Tensor &t, int32_t *code) {
  *code = t.scalar_type() == at::kBFloat16 ? S1F_BF16 : S1F_F32;
  return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kFloat;
}
bool fits(int64_t x) { return x >= 0 && x <= 0x7fffffff; }

// Batch entries and head_dim of `small` are what the kernels address `big` with.
bool covers(const at::Tensor &big, const at::Tensor &small) { return big.size(0) >= small.size(0) && big.size(3) >= small.size(3); }

bool desc_of(const at::Tensor &q, const at::Tensor &kv, s1f_desc *d) {
  *d = {};
  if (!rows_of(q) || !rows_of(kv) || !dtype_of(q, &d->dtype) || kv.scalar_type() != q.scalar_type() || !covers(kv, q)) return false;
  if (!fits(q.size(0)) || !fits(q.size(1)) || !fits(kv.size(1)) || !fits(q.size(3))) return false;
  d->batch = (int32_t)q.size(0); d->n_q_heads = (int32_t)q.size(1); d->n_kv_heads = (int32_t)kv.size(1); d->head_dim = (int32_t)q.size(3);
  d->q_stride_b = q.stride(0); d->q_stride_h = q.stride(1); d->q_stride_s = q.stride(2);
  d->kv_stride_b = kv.stride(0); d->kv_stride_h = kv.stride(1); d->kv_stride_s = kv.stride(2);
  d->kv_capacity = kv.size(2);
  return true;
}
bool cache_desc_of(const at::Tensor &cache, const at::Tensor &typed, s1f_desc *d) {
  *d = {};
  if (!rows_of(cache) || !dtype_of(typed, &d->dtype) || !fits(cache.size(0)) || !fits(cache.size(1)) || !fits(cache.size(3))) return false;
  d->batch = (int32_t)cache.size(0); d->n_q_heads = d->n_kv_heads = (int32_t)cache.size(1); d->head_dim = (int32_t)cache.size(3);
  d->q_stride_s = cache.size(3);
  d->kv_stride_b = cache.stride(0); d->kv_stride_h = cache.stride(1); d->kv_stride_s = cache.stride(2);
  d->kv_capacity = cache.size(2);
  return true;
}
bool segment_ok(const at::Tensor &seg, const at::Tensor &cache) {
  return rows_of(seg) && covers(seg, cache) && seg.size(1) >= cache.size(1);
}
bool lse_ok(const at::Tensor &lse, const at::Tensor &q) {
  return lse.scalar_type() == at::kFloat && lse.is_contiguous() && lse.sizes() == q.sizes().slice(0, 3);
}
bool acc_ok(const at::Tensor &k, const at::Tensor &dk, const at::Tensor &dv) {
  return same_layout(dk, dv) && dk.sizes() == k.sizes() && dk.strides() == k.strides() && dk.scalar_type() == at::kFloat;
}
template <typename T = void> T *ptr(const at::Tensor *t) { return static_cast<T *>(t->data_ptr()); }
size_t bytes(const at::Tensor *t) { return t ? (size_t)t->numel() * t->element_size() : 0; }

// The call itself without the interpreter lock; a C++ exception out of a tensor (one without memory) is the Python path's to report.
template <typename F> PyObject *call(F f) {
  int rc = kPython;
  try {
    rc = f();
  } catch (...) {
    rc = kPython;
  }
  return PyLong_FromLong(rc);
}
struct Unlocked {
  PyThreadState *state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

// (q, k, v, off, out, lse)
PyObject *fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    Args x;
    s1f_desc d;
    if (!x.read(args, n, 6, 3, -1)) return kPython;
    auto &[q, k, v, out, lse] = reinterpret_cast<const at::Tensor *(&)[5]>(x.t);
    if (!same_layout(*q, *out) || !same_layout(*k, *v) || !desc_of(*q, *k, &d) || !lse_ok(*lse, *q) || !x.read_stream()) return kPython;
    void *const p[] = {ptr(q), ptr(k), ptr(v), ptr(out), ptr(lse)};
    Unlocked u;
    return api.fwd(&d, p[0], p[1], p[2], x.off, q->size(2), p[3], static_cast<float *>(p[4]), x.stream);
  });
}
// (q, k, v, off, out, lse, workspace or None)
PyObject *fwd_ws(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    Args x;
    s1f_desc d;
    if (!x.read(args, n, 7, 3, 6)) return kPython;
    auto &[q, k, v, out, lse, ws] = reinterpret_cast<const at::Tensor *(&)[6]>(x.t);
    if (!same_layout(*q, *out) || !same_layout(*k, *v) || !desc_of(*q, *k, &d) || !lse_ok(*lse, *q) || !x.read_stream()) return kPython;
    void *const p[] = {ptr(q), ptr(k), ptr(v), ptr(out), ptr(lse), ws ? ptr(ws) : nullptr};
    Unlocked u;
    return api.fwd_ws(&d, p[0], p[1], p[2], x.off, q->size(2), p[3], static_cast<float *>(p[4]), p[5], bytes(ws), x.stream);
  });
}
// (dout, q, k, v, out, lse, off, dq, dk, dv[, workspace])
PyObject *bwd_any(PyObject *const *args, Py_ssize_t n, bool has_ws) {
  return call([&]() -> int {
    Args x;
    s1f_desc d;
    if (!x.read(args, n, has_ws ? 11 : 10, 6, -1)) return kPython;
    auto &[dout, q, k, v, out, lse, dq, dk, dv, ws] = x.t;
    if (!same_layout(*q, *dout) || !same_layout(*q, *out) || !same_layout(*q, *dq) || !same_layout(*k, *v) || !acc_ok(*k, *dk, *dv) ||
        !lse_ok(*lse, *q) || !desc_of(*q, *k, &d) || !x.read_stream())
      return kPython;
    void *const p[] = {ptr(dout), ptr(q), ptr(k), ptr(v), ptr(out), ptr(lse), ptr(dq), ptr(dk), ptr(dv), has_ws ? ptr(ws) : nullptr};
    const float *l = static_cast<const float *>(p[5]);
    float *dkp = static_cast<float *>(p[7]), *dvp = static_cast<float *>(p[8]);
    const size_t ws_bytes = has_ws ? bytes(ws) : 0;
    Unlocked u;
    return has_ws ? api.bwd(&d, p[0], p[1], p[2], p[3], p[4], l, x.off, q->size(2), p[6], dkp, dvp, p[9], ws_bytes, x.stream)
                  : api.bwd_noalloc(&d, p[0], p[1], p[2], p[3], p[4], l, x.off, q->size(2), p[6], dkp, dvp, x.stream);
  });
}
PyObject *bwd(PyObject *, PyObject *const *args, Py_ssize_t n) { return bwd_any(args, n, true); }
PyObject *bwd_noalloc(PyObject *, PyObject *const *args, Py_ssize_t n) { return bwd_any(args, n, false); }
// (k_seg, v_seg, off, k_cache, v_cache)
PyObject *append(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    Args x;
    s1f_desc d;
    if (!x.read(args, n, 5, 2, -1)) return kPython;
    auto &[ks, vs, kc, vc] = reinterpret_cast<const at::Tensor *(&)[4]>(x.t);
    if (!same_layout(*ks, *vs) || !same_layout(*kc, *vc) || !cache_desc_of(*kc, *kc, &d) || !segment_ok(*ks, *kc) ||
        ks->scalar_type() != kc->scalar_type() || !x.read_stream())
      return kPython;
    void *const p[] = {ptr(ks), ptr(vs), ptr(kc), ptr(vc)};
    Unlocked u;
    return api.append(&d, p[0], p[1], ks->stride(0), ks->stride(1), ks->stride(2), x.off, ks->size(2), p[2], p[3], x.stream);
  });
}
// (dk, dv, off, dk_seg, dv_seg)
PyObject *emit(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    Args x;
    s1f_desc d;
    if (!x.read(args, n, 5, 2, -1)) return kPython;
    auto &[dk, dv, ks, vs] = reinterpret_cast<const at::Tensor *(&)[4]>(x.t);
    if (!same_layout(*dk, *dv) || !same_layout(*ks, *vs) || dk->scalar_type() != at::kFloat || !cache_desc_of(*dk, *ks, &d) ||
        !segment_ok(*ks, *dk) || !x.read_stream())
      return kPython;
    void *const p[] = {ptr(dk), ptr(dv), ptr(ks), ptr(vs)};
    Unlocked u;
    return api.emit(&d, static_cast<const float *>(p[0]), static_cast<const float *>(p[1]), x.off, ks->size(2), p[2], p[3], ks->stride(0),
                    ks->stride(1), ks->stride(2), x.stream);
  });
}
// ---- rows of hidden states: embedding, layer norm, token loss --------------------------------------------------------------------------

// Plain tensors of the current device, number `real_at` a float, number `optional` maybe None; and the device's stream.
struct RowArgs {
  const at::Tensor *t[10];
  double real = 0.0;
  void *stream = nullptr;
  bool read(PyObject *const *args, Py_ssize_t n, Py_ssize_t want, Py_ssize_t real_at, Py_ssize_t optional) {
    if (n != want || get_device == nullptr || at::impl::PythonTorchFunctionTLS::stack_len() > 0) return false;
    int64_t device = -1;
    for (Py_ssize_t i = 0, k = 0; i < n; ++i) {
      if (i == real_at) {
        if (!PyFloat_CheckExact(args[i])) return false;
        real = PyFloat_AS_DOUBLE(args[i]);
        continue;
      }
      t[k] = i == optional && args[i] == Py_None ? nullptr : plain(args[i]);
      if (t[k] == nullptr && !(i == optional && args[i] == Py_None)) return false;
      if (t[k] != nullptr) {
        if (device >= 0 && t[k]->get_device() != device) return false;
        device = t[k]->get_device();
      }
      ++k;
    }
    PyObject *dev = PyObject_CallNoArgs(get_device);
    const long current = dev ? PyLong_AsLong(dev) : -1;
    PyObject *st = dev ? PyObject_CallOneArg(get_stream, dev) : nullptr;
    Py_XDECREF(dev);
    if (st == nullptr || current != device) {
      Py_XDECREF(st);
      return PyErr_Clear(), false;
    }
    stream = PyLong_AsVoidPtr(st);
    Py_DECREF(st);
    return PyErr_Occurred() == nullptr || (PyErr_Clear(), false);
  }
};

bool hidden_ok(const at::Tensor &t) { return t.dim() == 3 && (t.stride(2) == 1 || t.size(2) <= 1); }
int64_t stride_of(const at::Tensor &t, int i) { return t.size(i) > 1 ? t.stride(i) : 0; }
// x, y: tensors on either side of a call, or null
bool rows_desc_of(const at::Tensor *x, const at::Tensor *y, s1f_rows *d) {
  *d = {};
  const at::Tensor &a = x ? *x : *y;
  if (!hidden_ok(a) || !dtype_of(a, &d->dtype) || !fits(a.size(0)) || !fits(a.size(2))) return false;
  if (x && y && (!hidden_ok(*y) || y->sizes() != x->sizes() || y->scalar_type() != x->scalar_type())) return false;
  d->batch = (int32_t)a.size(0); d->hidden = (int32_t)a.size(2); d->rows = a.size(1);
  if (x) { d->x_stride_b = stride_of(*x, 0); d->x_stride_s = stride_of(*x, 1); }
  if (y) { d->y_stride_b = stride_of(*y, 0); d->y_stride_s = stride_of(*y, 1); }
  return true;
}
bool same_rows(const at::Tensor &a, const at::Tensor &b) {
  return hidden_ok(b) && b.sizes() == a.sizes() && stride_of(a, 0) == stride_of(b, 0) && stride_of(a, 1) == stride_of(b, 1) &&
         b.scalar_type() == a.scalar_type();
}
bool tokens_ok(const at::Tensor &t, const at::Tensor &like) {
  return t.scalar_type() == at::kLong && t.sizes() == like.sizes().slice(0, 2) && (t.size(1) <= 1 || t.stride(1) == 1);
}
bool row_values_ok(const at::Tensor &v, const at::Tensor &like) {
  return v.scalar_type() == at::kFloat && v.is_contiguous() && v.sizes() == like.sizes().slice(0, 2);
}
bool matrix_ok(const at::Tensor &t, int64_t hidden, at::ScalarType type) {
  return t.scalar_type() == type && t.dim() == 2 && t.size(1) == hidden && (t.stride(1) == 1 || hidden <= 1);
}
int64_t matrix_stride(const at::Tensor &t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
bool vector_ok(const at::Tensor &t, int64_t hidden, at::ScalarType type) {
  return t.scalar_type() == type && t.dim() == 1 && t.size(0) == hidden && t.is_contiguous();
}
bool space_ok(const at::Tensor *ws) { return ws == nullptr || ws->is_contiguous(); }
const int64_t *tokens_of(const at::Tensor *t) { return static_cast<const int64_t *>(t->data_ptr()); }
const float *values_of(const at::Tensor *t) { return static_cast<const float *>(t->data_ptr()); }

// (ids, table, scale, out)
PyObject *embed_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    RowArgs x;
    s1f_rows d;
    if (!x.read(args, n, 4, 2, -1)) return kPython;
    auto &[ids, table, out] = reinterpret_cast<const at::Tensor *(&)[3]>(x.t);
    if (!rows_desc_of(nullptr, out, &d) || !tokens_ok(*ids, *out) || !matrix_ok(*table, out->size(2), out->scalar_type())) return kPython;
    const int64_t *i = tokens_of(ids);
    void *const p[] = {ptr(table), ptr(out)};
    Unlocked u;
    return api.embed_fwd(&d, i, stride_of(*ids, 0), p[0], matrix_stride(*table), table->size(0), (float)x.real, p[1], x.stream);
  });
}
// (ids, dout, scale, dtable_acc, workspace)
PyObject *embed_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    RowArgs x;
    s1f_rows d;
    if (!x.read(args, n, 5, 2, 4)) return kPython;
    auto &[ids, dout, acc, ws] = reinterpret_cast<const at::Tensor *(&)[4]>(x.t);
    if (!rows_desc_of(nullptr, dout, &d) || !tokens_ok(*ids, *dout) || !matrix_ok(*acc, dout->size(2), at::kFloat) || !space_ok(ws)) return kPython;
    const int64_t *i = tokens_of(ids);
    void *const p[] = {ptr(dout), ptr(acc), ws ? ptr(ws) : nullptr};
    Unlocked u;
    return api.embed_bwd(&d, i, stride_of(*ids, 0), p[0], acc->size(0), (float)x.real, static_cast<float *>(p[1]), matrix_stride(*acc), p[2],
                         bytes(ws), x.stream);
  });
}
// (x, gamma, beta, eps, y, mean, rstd)
PyObject *layer_norm_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    RowArgs a;
    s1f_rows d;
    if (!a.read(args, n, 7, 3, -1)) return kPython;
    auto &[x, gamma, beta, y, mean, rstd] = reinterpret_cast<const at::Tensor *(&)[6]>(a.t);
    if (!rows_desc_of(x, y, &d) || !vector_ok(*gamma, x->size(2), x->scalar_type()) || !vector_ok(*beta, x->size(2), x->scalar_type()) ||
        !row_values_ok(*mean, *x) || !row_values_ok(*rstd, *x))
      return kPython;
    void *const p[] = {ptr(x), ptr(gamma), ptr(beta), ptr(y), ptr(mean), ptr(rstd)};
    Unlocked u;
    return api.layer_norm_fwd(&d, p[0], p[1], p[2], (float)a.real, p[3], static_cast<float *>(p[4]), static_cast<float *>(p[5]), a.stream);
  });
}
// (dy, x, gamma, mean, rstd, dx, dgamma_acc, dbeta_acc, workspace)
PyObject *layer_norm_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    RowArgs a;
    s1f_rows d;
    if (!a.read(args, n, 9, -1, 8)) return kPython;
    auto &[dy, x, gamma, mean, rstd, dx, dg, db, ws] = reinterpret_cast<const at::Tensor *(&)[9]>(a.t);
    if (!rows_desc_of(x, dy, &d) || !same_rows(*x, *dx) || !vector_ok(*gamma, x->size(2), x->scalar_type()) ||
        !vector_ok(*dg, x->size(2), at::kFloat) || !vector_ok(*db, x->size(2), at::kFloat) || !row_values_ok(*mean, *x) ||
        !row_values_ok(*rstd, *x) || !space_ok(ws))
      return kPython;
    void *const p[] = {ptr(dy), ptr(x), ptr(gamma), ptr(dx), ptr(dg), ptr(db), ws ? ptr(ws) : nullptr};
    const float *m = values_of(mean), *r = values_of(rstd);
    Unlocked u;
    return api.layer_norm_bwd(&d, p[0], p[1], p[2], m, r, p[3], static_cast<float *>(p[4]), static_cast<float *>(p[5]), p[6], bytes(ws), a.stream);
  });
}
// (x, weight, targets, loss, lse, workspace)
PyObject *token_loss_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    RowArgs a;
    s1f_rows d;
    if (!a.read(args, n, 6, -1, 5)) return kPython;
    auto &[x, weight, targets, loss, lse, ws] = reinterpret_cast<const at::Tensor *(&)[6]>(a.t);
    if (!rows_desc_of(x, nullptr, &d) || !matrix_ok(*weight, x->size(2), x->scalar_type()) || !tokens_ok(*targets, *x) ||
        !row_values_ok(*loss, *x) || !row_values_ok(*lse, *x) || !space_ok(ws))
      return kPython;
    const int64_t *i = tokens_of(targets);
    void *const p[] = {ptr(x), ptr(weight), ptr(loss), ptr(lse), ws ? ptr(ws) : nullptr};
    Unlocked u;
    return api.token_loss_fwd(&d, p[0], p[1], matrix_stride(*weight), weight->size(0), i, stride_of(*targets, 0), static_cast<float *>(p[2]),
                              static_cast<float *>(p[3]), p[4], bytes(ws), a.stream);
  });
}
// (dloss, x, weight, targets, lse, dx, dweight, workspace)
PyObject *token_loss_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    RowArgs a;
    s1f_rows d;
    int32_t code;
    if (!a.read(args, n, 8, -1, 7)) return kPython;
    auto &[dloss, x, weight, targets, lse, dx, dw, ws] = reinterpret_cast<const at::Tensor *(&)[8]>(a.t);
    if (!rows_desc_of(x, nullptr, &d) || !same_rows(*x, *dx) || !matrix_ok(*weight, x->size(2), x->scalar_type()) || !dtype_of(*dw, &code) ||
        !matrix_ok(*dw, x->size(2), dw->scalar_type()) || dw->sizes() != weight->sizes() || !tokens_ok(*targets, *x) ||
        !row_values_ok(*dloss, *x) || !row_values_ok(*lse, *x) || !space_ok(ws))
      return kPython;
    const int64_t *i = tokens_of(targets);
    const float *g = values_of(dloss), *l = values_of(lse);
    void *const p[] = {ptr(x), ptr(weight), ptr(dx), ptr(dw), ws ? ptr(ws) : nullptr};
    Unlocked u;
    return api.token_loss_bwd(&d, g, p[0], p[1], matrix_stride(*weight), weight->size(0), i, stride_of(*targets, 0), l, p[2], p[3],
                              matrix_stride(*dw), code, p[4], bytes(ws), a.stream);
  });
}

// ---- heads on their way from the projections to the attention, and back ------------------------------------------------------------------

// Arguments by kinds: t a plain tensor of the current device, o one or None, f a float, b a truth value, i an integer, p an integer or a
// plain tensor; and the device's stream.
struct MixedArgs {
  const at::Tensor *t[18];
  double real[2] = {0.0, 0.0};
  int64_t whole[2] = {0, 0};
  bool truth = false;
  const at::Tensor *positions = nullptr;
  int64_t first = 0;
  void *stream = nullptr;
  static bool integer(PyObject *x, int64_t *to) {
    int overflow = 0;
    if (!PyLong_CheckExact(x)) return false;
    *to = PyLong_AsLongLongAndOverflow(x, &overflow);
    return overflow == 0;
  }
  bool read(PyObject *const *args, Py_ssize_t n, const char *kinds) {
    if (n != (Py_ssize_t)std::strlen(kinds) || get_device == nullptr || at::impl::PythonTorchFunctionTLS::stack_len() > 0) return false;
    int64_t device = -1;
    int tensors = 0, reals = 0, wholes = 0;
    for (Py_ssize_t i = 0; i < n; ++i) {
      const at::Tensor *x = nullptr;
      switch (kinds[i]) {
        case 'f':
          if (!PyFloat_CheckExact(args[i])) return false;
          real[reals++] = PyFloat_AS_DOUBLE(args[i]);
          continue;
        case 'b':
          if (!PyBool_Check(args[i])) return false;
          truth = args[i] == Py_True;
          continue;
        case 'i':
          if (!integer(args[i], &whole[wholes++])) return false;
          continue;
        case 'p':
          if (integer(args[i], &first)) {
            if (first <= -(int64_t(1) << 62) || first >= int64_t(1) << 62) return false;
            continue;
          }
          x = positions = plain(args[i]);
          break;
        default:
          x = t[tensors++] = kinds[i] == 'o' && args[i] == Py_None ? nullptr : plain(args[i]);
          if (x == nullptr && kinds[i] == 'o' && args[i] == Py_None) continue;
      }
      if (x == nullptr || (device >= 0 && x->get_device() != device)) return false;
      device = x->get_device();
    }
    PyObject *dev = PyObject_CallNoArgs(get_device);
    const long current = dev ? PyLong_AsLong(dev) : -1;
    PyObject *st = dev ? PyObject_CallOneArg(get_stream, dev) : nullptr;
    Py_XDECREF(dev);
    if (st == nullptr || current != device) {
      Py_XDECREF(st);
      return PyErr_Clear(), false;
    }
    stream = PyLong_AsVoidPtr(st);
    Py_DECREF(st);
    return PyErr_Occurred() == nullptr || (PyErr_Clear(), false);
  }
};

bool heads_ok(const at::Tensor &t, int64_t b, int64_t h, int64_t n, int64_t d, at::ScalarType type) {
  return t.dim() == 4 && t.size(0) == b && t.size(1) == h && t.size(2) == n && t.size(3) == d && (t.stride(3) == 1 || d <= 1) && t.scalar_type() == type;
}
bool same_strides(const at::Tensor &a, const at::Tensor &b) {   // (of tensors of one shape)
  return stride_of(a, 0) == stride_of(b, 0) && stride_of(a, 1) == stride_of(b, 1) && stride_of(a, 2) == stride_of(b, 2);
}
// q, k, v on one side, q_rot and the caches (of the type `cached`) on the other; v and v_cache: both or neither
bool heads_desc_of(const MixedArgs &x, const at::Tensor &q, const at::Tensor &q_rot, const at::Tensor &k, const at::Tensor *v, const at::Tensor &k_cache,
                   const at::Tensor *v_cache, bool gradients, const at::Tensor &freqs, s1f_heads *d) {
  *d = {};
  if (q.dim() != 4 || k.dim() != 4 || k_cache.dim() != 4 || (v == nullptr) != (v_cache == nullptr) || !dtype_of(q, &d->dtype)) return false;
  const int64_t b = q.size(0), hq = q.size(1), n = q.size(2), dim = q.size(3), hk = k.size(1), capacity = k_cache.size(2);
  const at::ScalarType type = q.scalar_type(), cached = gradients ? at::kFloat : type;
  if (!fits(b) || !fits(hq) || !fits(hk) || !fits(dim) || !heads_ok(q, b, hq, n, dim, type) || !heads_ok(q_rot, b, hq, n, dim, type)) return false;
  if (!heads_ok(k, b, hk, n, dim, type) || !heads_ok(k_cache, b, hk, capacity, dim, cached)) return false;
  if (v && (!heads_ok(*v, b, hk, n, dim, type) || !same_strides(*v, k) || !heads_ok(*v_cache, b, hk, capacity, dim, cached) || !same_strides(*v_cache, k_cache)))
    return false;
  if (freqs.scalar_type() != at::kDouble || freqs.dim() != 1 || !freqs.is_contiguous() || 2 * freqs.size(0) > dim) return false;
  if (x.positions && (x.positions->scalar_type() != at::kLong || x.positions->dim() != 2 || x.positions->size(0) != b || x.positions->size(1) != n ||
                      (n > 1 && x.positions->stride(1) != 1)))
    return false;
  d->batch = (int32_t)b; d->n_q_heads = (int32_t)hq; d->n_kv_heads = (int32_t)hk; d->head_dim = (int32_t)dim;
  d->rotary_dim = (int32_t)(2 * freqs.size(0)); d->interleaved = x.truth; d->rows = n;
  d->q_stride_b = stride_of(q, 0); d->q_stride_h = stride_of(q, 1); d->q_stride_s = stride_of(q, 2);
  d->kv_stride_b = stride_of(k, 0); d->kv_stride_h = stride_of(k, 1); d->kv_stride_s = stride_of(k, 2);
  d->rot_stride_b = stride_of(q_rot, 0); d->rot_stride_h = stride_of(q_rot, 1); d->rot_stride_s = stride_of(q_rot, 2);
  d->cache_stride_b = stride_of(k_cache, 0); d->cache_stride_h = stride_of(k_cache, 1); d->cache_stride_s = stride_of(k_cache, 2);
  d->cache_capacity = capacity;
  return true;
}
void *ptr_or_null(const at::Tensor *t) { return t ? ptr(t) : nullptr; }
// What follows a call's inputs.
struct Turn {
  const double *freqs;
  const int64_t *at = nullptr;
  int64_t sb = 0;
  Turn(const MixedArgs &x, const at::Tensor *f) : freqs(static_cast<const double *>(f->data_ptr())) {
    if (x.positions) {
      at = tokens_of(x.positions);
      sb = stride_of(*x.positions, 0);
    }
  }
};

// (q, k, v or None[, q_gain, k_gain, eps], freqs, magnitude, interleaved, positions, seg_off, q_rot, k_cache, v_cache or None)
PyObject *rope_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    MixedArgs x;
    s1f_heads d;
    if (!x.read(args, n, "ttotfbpitto")) return kPython;
    auto &[q, k, v, freqs, q_rot, kc, vc] = reinterpret_cast<const at::Tensor *(&)[7]>(x.t);
    if (!heads_desc_of(x, *q, *q_rot, *k, v, *kc, vc, false, *freqs, &d)) return kPython;
    const Turn turn(x, freqs);
    void *const p[] = {ptr(q), ptr(k), ptr_or_null(v), ptr(q_rot), ptr(kc), ptr_or_null(vc)};
    Unlocked u;
    return api.rope_fwd(&d, p[0], p[1], p[2], turn.freqs, (float)x.real[0], turn.at, turn.sb, x.first, x.whole[0], p[3], p[4], p[5], x.stream);
  });
}
PyObject *qk_norm_rope_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    MixedArgs x;
    s1f_heads d;
    if (!x.read(args, n, "ttottftfbpitto")) return kPython;
    auto &[q, k, v, q_gain, k_gain, freqs, q_rot, kc, vc] = reinterpret_cast<const at::Tensor *(&)[9]>(x.t);
    if (!heads_desc_of(x, *q, *q_rot, *k, v, *kc, vc, false, *freqs, &d) || !vector_ok(*q_gain, d.head_dim, q->scalar_type()) ||
        !vector_ok(*k_gain, d.head_dim, q->scalar_type()))
      return kPython;
    const Turn turn(x, freqs);
    void *const p[] = {ptr(q), ptr(k), ptr_or_null(v), ptr(q_gain), ptr(k_gain), ptr(q_rot), ptr(kc), ptr_or_null(vc)};
    Unlocked u;
    return api.qk_norm_rope_fwd(&d, p[0], p[1], p[2], p[3], p[4], (float)x.real[0], turn.freqs, (float)x.real[1], turn.at, turn.sb, x.first, x.whole[0], p[5],
                                p[6], p[7], x.stream);
  });
}
// (dq_rot, dk_acc, dv_acc or None, freqs, magnitude, interleaved, positions, seg_off, dq, dk, dv or None)
PyObject *rope_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    MixedArgs x;
    s1f_heads d;
    if (!x.read(args, n, "ttotfbpitto")) return kPython;
    auto &[dq_rot, dka, dva, freqs, dq, dk, dv] = reinterpret_cast<const at::Tensor *(&)[7]>(x.t);
    if (!heads_desc_of(x, *dq, *dq_rot, *dk, dv, *dka, dva, true, *freqs, &d)) return kPython;
    const Turn turn(x, freqs);
    void *const p[] = {ptr(dq_rot), ptr(dka), ptr_or_null(dva), ptr(dq), ptr(dk), ptr_or_null(dv)};
    Unlocked u;
    return api.rope_bwd(&d, p[0], static_cast<const float *>(p[1]), static_cast<const float *>(p[2]), turn.freqs, (float)x.real[0], turn.at, turn.sb, x.first,
                        x.whole[0], p[3], p[4], p[5], x.stream);
  });
}
// (dq_rot, dk_acc, dv_acc or None, q, k, q_gain, k_gain, eps, freqs, magnitude, interleaved, positions, seg_off, dq, dk, dv or None, dq_gain_acc,
// dk_gain_acc, workspace)
PyObject *qk_norm_rope_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    MixedArgs x;
    s1f_heads d;
    if (!x.read(args, n, "ttottttftfbpittotto")) return kPython;
    auto &[dq_rot, dka, dva, q, k, q_gain, k_gain, freqs, dq, dk, dv, dqg, dkg, ws] = reinterpret_cast<const at::Tensor *(&)[14]>(x.t);
    if (!heads_desc_of(x, *dq, *dq_rot, *dk, dv, *dka, dva, true, *freqs, &d)) return kPython;
    if (!heads_ok(*q, d.batch, d.n_q_heads, d.rows, d.head_dim, dq->scalar_type()) || !same_strides(*q, *dq) ||
        !heads_ok(*k, d.batch, d.n_kv_heads, d.rows, d.head_dim, dq->scalar_type()) || !same_strides(*k, *dk) ||
        !vector_ok(*q_gain, d.head_dim, dq->scalar_type()) || !vector_ok(*k_gain, d.head_dim, dq->scalar_type()) ||
        !vector_ok(*dqg, d.head_dim, at::kFloat) || !vector_ok(*dkg, d.head_dim, at::kFloat) || !space_ok(ws))
      return kPython;
    const Turn turn(x, freqs);
    void *const p[] = {ptr(dq_rot), ptr(dka), ptr_or_null(dva), ptr(q), ptr(k), ptr(q_gain), ptr(k_gain), ptr(dq), ptr(dk), ptr_or_null(dv), ptr(dqg), ptr(dkg),
                       ptr_or_null(ws)};
    Unlocked u;
    return api.qk_norm_rope_bwd(&d, p[0], static_cast<const float *>(p[1]), static_cast<const float *>(p[2]), p[3], p[4], p[5], p[6], (float)x.real[0],
                                turn.freqs, (float)x.real[1], turn.at, turn.sb, x.first, x.whole[0], p[7], p[8], p[9], static_cast<float *>(p[10]),
                                static_cast<float *>(p[11]), p[12], bytes(ws), x.stream);
  });
}

// ---- gated feed-forward block ----------------------------------------------------------------------------------------------------------

bool ffn_weights_ok(const at::Tensor &x, const at::Tensor &w_in, const at::Tensor &w_out, at::ScalarType type) {
  return matrix_ok(w_in, x.size(2), type) && w_in.size(0) % 2 == 0 && w_out.dim() == 2 && w_out.size(0) == x.size(2) && matrix_ok(w_out, w_in.size(0) / 2, type);
}
bool gate_up_ok(const at::Tensor &t, const at::Tensor &x, const at::Tensor &w_in) {
  return t.scalar_type() == x.scalar_type() && t.is_contiguous() && t.dim() == 3 && t.size(0) == x.size(0) && t.size(1) == x.size(1) && t.size(2) == w_in.size(0);
}
// (x, w_in, w_out, act, y, gate_up or None, workspace)
PyObject *gated_ffn_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    MixedArgs a;
    s1f_rows d;
    if (!a.read(args, n, "tttitoo")) return kPython;
    auto &[x, w_in, w_out, y, gate_up, ws] = reinterpret_cast<const at::Tensor *(&)[6]>(a.t);
    if (!fits(a.whole[0]) || !rows_desc_of(x, y, &d) || !ffn_weights_ok(*x, *w_in, *w_out, x->scalar_type()) || (gate_up && !gate_up_ok(*gate_up, *x, *w_in)) ||
        !space_ok(ws))
      return kPython;
    void *const p[] = {ptr(x), ptr(w_in), ptr(w_out), ptr(y), ptr_or_null(gate_up), ptr_or_null(ws)};
    Unlocked u;
    return api.gated_ffn_fwd(&d, p[0], p[1], matrix_stride(*w_in), p[2], matrix_stride(*w_out), w_in->size(0) / 2, (int32_t)a.whole[0], p[3], p[4], p[5], bytes(ws),
                             a.stream);
  });
}
// (dy, x, w_in, w_out, act, gate_up, dx, dw_in, dw_out, workspace)
PyObject *gated_ffn_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return call([&]() -> int {
    MixedArgs a;
    s1f_rows d;
    int32_t code;
    if (!a.read(args, n, "ttttitttto")) return kPython;
    auto &[dy, x, w_in, w_out, gate_up, dx, dw_in, dw_out, ws] = reinterpret_cast<const at::Tensor *(&)[9]>(a.t);
    if (!fits(a.whole[0]) || !rows_desc_of(x, dy, &d) || !same_rows(*x, *dx) || !ffn_weights_ok(*x, *w_in, *w_out, x->scalar_type()) || !dtype_of(*dw_in, &code) ||
        !ffn_weights_ok(*x, *dw_in, *dw_out, dw_in->scalar_type()) || dw_in->sizes() != w_in->sizes() || !gate_up_ok(*gate_up, *x, *w_in) || !space_ok(ws))
      return kPython;
    void *const p[] = {ptr(dy), ptr(x), ptr(w_in), ptr(w_out), ptr(gate_up), ptr(dx), ptr(dw_in), ptr(dw_out), ptr_or_null(ws)};
    Unlocked u;
    return api.gated_ffn_bwd(&d, p[0], p[1], p[2], matrix_stride(*w_in), p[3], matrix_stride(*w_out), w_in->size(0) / 2, (int32_t)a.whole[0], p[4], p[5], p[6],
                             matrix_stride(*dw_in), p[7], matrix_stride(*dw_out), code, p[8], bytes(ws), a.stream);
  });
}

// (addresses of the entry points in the order of Api, torch's functions for the current device and for a device's stream)
PyObject *bind(PyObject *, PyObject *args) {
  PyObject *addresses, *dev, *st;
  if (!PyArg_ParseTuple(args, "O!OO", &PyTuple_Type, &addresses, &dev, &st)) return nullptr;
  constexpr Py_ssize_t kEntries = sizeof(Api) / sizeof(void *);
  if (PyTuple_GET_SIZE(addresses) != kEntries) return PyErr_Format(PyExc_ValueError, "expected %zd entry points", kEntries);
  void *at[kEntries];
  for (Py_ssize_t i = 0; i < kEntries; ++i) {
    at[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
    if (PyErr_Occurred()) return nullptr;
  }
  static_assert(sizeof(at) == sizeof(Api), "an Api is its entry points");
  std::memcpy(&api, at, sizeof(Api));
  Py_INCREF(dev);
  Py_INCREF(st);
  Py_XDECREF(get_device);
  Py_XDECREF(get_stream);
  get_device = dev;
  get_stream = st;
  Py_RETURN_NONE;
}

#define S1F_METHOD(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f))
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         {"fwd", S1F_METHOD(fwd), METH_FASTCALL, nullptr},
                         {"fwd_ws", S1F_METHOD(fwd_ws), METH_FASTCALL, nullptr},
                         {"bwd", S1F_METHOD(bwd), METH_FASTCALL, nullptr},
                         {"bwd_noalloc", S1F_METHOD(bwd_noalloc), METH_FASTCALL, nullptr},
                         {"append", S1F_METHOD(append), METH_FASTCALL, nullptr},
                         {"emit", S1F_METHOD(emit), METH_FASTCALL, nullptr},
                         {"embed_fwd", S1F_METHOD(embed_fwd), METH_FASTCALL, nullptr},
                         {"embed_bwd", S1F_METHOD(embed_bwd), METH_FASTCALL, nullptr},
                         {"layer_norm_fwd", S1F_METHOD(layer_norm_fwd), METH_FASTCALL, nullptr},
                         {"layer_norm_bwd", S1F_METHOD(layer_norm_bwd), METH_FASTCALL, nullptr},
                         {"token_loss_fwd", S1F_METHOD(token_loss_fwd), METH_FASTCALL, nullptr},
                         {"token_loss_bwd", S1F_METHOD(token_loss_bwd), METH_FASTCALL, nullptr},
                         {"rope_fwd", S1F_METHOD(rope_fwd), METH_FASTCALL, nullptr},
                         {"rope_bwd", S1F_METHOD(rope_bwd), METH_FASTCALL, nullptr},
                         {"qk_norm_rope_fwd", S1F_METHOD(qk_norm_rope_fwd), METH_FASTCALL, nullptr},
                         {"qk_norm_rope_bwd", S1F_METHOD(qk_norm_rope_bwd), METH_FASTCALL, nullptr},
                         {"gated_ffn_fwd", S1F_METHOD(gated_ffn_fwd), METH_FASTCALL, nullptr},
                         {"gated_ffn_bwd", S1F_METHOD(gated_ffn_bwd), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls() {
  PyObject *m = PyModule_Create(&module);
  if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) != 0) Py_CLEAR(m);
  return m;
}
