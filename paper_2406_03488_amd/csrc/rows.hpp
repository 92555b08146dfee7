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

// A row's elements in pieces of 16 bytes.  WIDE: rows start on 16 bytes and hold a whole number of pieces; else a piece lies wherever its elements do
// (memory takes accesses of 16 bytes on any element: a layer norm gradient of 2714 rows of 2563 elements element by element took 40 us), and the last one may
// be short: `left` elements of the row are there from the piece on.
template <typename T, bool WIDE> struct Piece {
  static constexpr int N = Elem<T>::CE;
  typedef T Wide __attribute__((ext_vector_type(N)));
  typedef T Loose __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  typedef Wide Raw;
  typedef float Values[N];
  S1F_DEV static Raw get(const T *p, int left) {
    if constexpr (WIDE) {
      return *reinterpret_cast<const Wide *>(p);
    } else {
      if (left >= N) return *reinterpret_cast<const Loose *>(p);
      Raw r;
#pragma unroll
      for (int e = 0; e < N; ++e) r[e] = e < left ? p[e] : (T)0.f;
      return r;
    }
  }
  S1F_DEV static Raw none() {
    Raw r;
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = (T)0.f;
    return r;
  }
  S1F_DEV static void values(const Raw &r, Values &v) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (float)r[e];
  }
  S1F_DEV static void load(const T *p, int left, Values &v) { values(get(p, left), v); }
  S1F_DEV static void store(T *p, int left, const Values &v) {
    Raw r;
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = (T)v[e];
    if constexpr (WIDE) {
      *reinterpret_cast<Wide *>(p) = r;
    } else if (left >= N) {
      *reinterpret_cast<Loose *>(p) = r;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < left) p[e] = r[e];
    }
  }
};
// The same for N consecutive fp32 values, N = 4 or 8.
template <int N, bool WIDE> S1F_DEV void load_f32(const float *p, int left, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f32x4 x = Piece<float, WIDE>::get(p + i, left - i);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[i + e] = x[e];
  }
}
template <int N, bool WIDE> S1F_DEV void store_f32(float *p, int left, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) Piece<float, WIDE>::store(p + i, left - i, {v[i], v[i + 1], v[i + 2], v[i + 3]});
}

constexpr int64_t kMostRows = int64_t(1) << 21;   // batch * rows: a launch of 1024 threads for each holds fewer than 2^32, more would not all run
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
