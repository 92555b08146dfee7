// What the calls on rows of hidden states share (embedding, layer norm, token loss): checks of s1f_rows, addresses of rows, 16-byte
// pieces of them as fp32 values.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_device.hpp"
#include "s1f.h"

namespace s1f {

// Rows [batch, rows] of one side of a call.  The strides are in elements.
struct RowsOf {
  int64_t sb, ss;
  Divisor by_rows;
  S1F_DEV int64_t offset(int row) const {
    int b, r;
    div_mod(row, by_rows, b, r);
    return b * sb + r * ss;
  }
};

// A row's elements in pieces of N: 16 bytes where everything is aligned to them (WIDE), else single elements.
template <typename T, bool WIDE> struct Piece {
  static constexpr int N = WIDE ? Elem<T>::CE : 1;
  typedef float Values[N];
  S1F_DEV static void load(const T *p, Values &v) {
    if constexpr (!WIDE) {
      v[0] = (float)*p;
    } else if constexpr (sizeof(T) == 4) {
      const f32x4 x = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = x[e];
    } else {
      const bf16x8 x = *reinterpret_cast<const bf16x8 *>(p);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = (float)x[e];
    }
  }
  S1F_DEV static void store(T *p, const Values &v) {
    if constexpr (!WIDE) {
      *p = (T)v[0];
    } else if constexpr (sizeof(T) == 4) {
      f32x4 x;
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = v[e];
      *reinterpret_cast<f32x4 *>(p) = x;
    } else {
      bf16x8 x;
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = (bf16_t)v[e];
      *reinterpret_cast<bf16x8 *>(p) = x;
    }
  }
};
// N consecutive fp32 values (N = 1, 4 or 8)
template <int N> S1F_DEV void load_f32(const float *p, float (&v)[N]) {
  if constexpr (N == 1) {
    v[0] = *p;
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4 *>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = x[e];
    }
  }
}
template <int N> S1F_DEV void store_f32(float *p, const float (&v)[N]) {
  if constexpr (N == 1) {
    *p = v[0];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4 *>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
  }
}

constexpr int64_t kMostRows = int64_t(1) << 24;   // batch * rows: numbers of rows are 32 bits, grids one launch
constexpr int32_t kMostHidden = 16384;

inline bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool on4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
inline bool on_element(const void *p, int32_t dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == S1F_BF16 ? 1 : 3)) == 0; }

// strides of one side: rows do not overlap
inline bool strides_ok(const s1f_rows *d, int64_t sb, int64_t ss) {
  return (d->rows == 1 || ss >= d->hidden) && (d->batch == 1 || sb >= d->hidden);
}
// use_x, use_y: sides that the call reads or writes
inline int check_rows(const s1f_rows *d, bool use_x, bool use_y) {
  if (!d || d->batch < 1 || d->hidden < 1 || d->reserved != 0) return S1F_EINVAL;
  if (d->dtype != S1F_F32 && d->dtype != S1F_BF16) return S1F_EUNSUPPORTED;
  if (d->hidden > kMostHidden) return S1F_EUNSUPPORTED;
  if ((use_x && !strides_ok(d, d->x_stride_b, d->x_stride_s)) || (use_y && !strides_ok(d, d->y_stride_b, d->y_stride_s))) return S1F_EINVAL;
  if (d->rows < 1) return S1F_ERANGE;
  if (d->rows > kMostRows || d->batch * d->rows > kMostRows) return S1F_EUNSUPPORTED;
  return S1F_OK;
}
inline RowsOf x_rows(const s1f_rows *d) { return RowsOf{d->x_stride_b, d->x_stride_s, Divisor::of(d->rows)}; }
inline RowsOf y_rows(const s1f_rows *d) { return RowsOf{d->y_stride_b, d->y_stride_s, Divisor::of(d->rows)}; }
inline int64_t elements_of_16_bytes(int32_t dtype) { return dtype == S1F_BF16 ? 8 : 4; }
// whether every row of a side starts on 16 bytes and has a whole number of them, given that the tensors do
inline bool wide_rows(const s1f_rows *d, int64_t sb, int64_t ss) {
  const int64_t n = elements_of_16_bytes(d->dtype);
  return d->hidden % n == 0 && (d->rows == 1 || ss % n == 0) && (d->batch == 1 || sb % n == 0);
}

template <typename ARGS> int launch_rows_kernel(void (*kernel)(ARGS), int64_t grid, int threads, ARGS a, hipStream_t st, int lds = 0) {
  void *params[] = {&a};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)grid), dim3(threads), params, lds, st);
  return e == hipSuccess ? S1F_OK : S1F_EDEVICE;
}

}  // namespace s1f
