// Layer norm of the rows of a segment, and its gradient.
//
//   forward    mean = sum(x) / h,  rstd = 1 / sqrt(sum((x - mean)^2) / h + eps),  y = (x - mean) * rstd * gamma + beta
//   backward   xhat = (x - mean) * rstd,  g = dy * gamma,
//              dx = rstd * (g - sum(g) / h - xhat * sum(g * xhat) / h);  dgamma += sum over rows of dy * xhat,  dbeta += of dy
//
// Bound by memory: a row is read once and stays in registers between its sums and its result.  The squares are summed around the mean, not
// from the moments, which lose the variance of rows whose mean is large beside it.  All sums are fp32.
// The gradients of gamma and beta sum over rows: a workgroup walks many rows, its threads keep the columns they own in registers, and a
// second kernel adds up what the workgroups have left, in their order: the same bits every time.
#include "rows.hpp"

namespace s1f {
namespace {

struct NormArgs {
  const void *x, *dy, *gamma, *beta;
  const float *mean_in, *rstd_in;
  void *y, *dx;
  float *mean, *rstd;
  float *part;                    // [workgroup][dgamma, dbeta][part_ld]
  float *dgamma, *dbeta;
  RowsOf xs, ys;
  int32_t n, hidden, pieces, part_ld, parts;
  float eps, inv_hidden;
};

// Sum over the TPR threads that share a row (64, 256, 512 or 1024); every one of them gets it.  `lds`: a float per wave, not written
// before all have read the sum before the last.
S1F_DEV float wave_sum(float x) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) x += __shfl_xor(x, s);
  return x;
}
template <int TPR, int K> S1F_DEV void row_sums(float (&x)[K], float *lds) {
#pragma unroll
  for (int k = 0; k < K; ++k) x[k] = wave_sum(x[k]);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) lds[k * W + (threadIdx.x >> 6)] = x[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      x[k] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) x[k] += lds[k * W + w];
    }
  }
}

// E: elements of a row per thread.  4096 rows of 4096 bf16 elements, 67 MB: 12.4 to 13.4 us, 5 TB/s and more, some of it out of the caches (a large copy: 4.8);
// 256 rows of 256 fp32 elements 3 us, the latency of a load, two sums over a wave and a store.
template <typename T, bool WIDE, int TPR, int E> __global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_fwd_kernel(const NormArgs a) {
  typedef Piece<T, WIDE> P;
  constexpr int NP = E / P::N, THREADS = TPR < 256 ? 256 : TPR;
  __shared__ float lds[2][16];
  const int row = blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR, t = threadIdx.x % TPR;
  if (row >= a.n) return;   // (whole waves; with more threads to a row there is one row to a workgroup)
  const T *x = reinterpret_cast<const T *>(a.x) + a.xs.offset(row);
  typename P::Raw raw[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int p = t + i * TPR;
    raw[i] = p < a.pieces ? P::get(x + p * P::N, a.hidden - p * P::N) : P::none();
  }
  typename P::Values v[NP];
  float s[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    P::values(raw[i], v[i]);
#pragma unroll
    for (int e = 0; e < P::N; ++e) s[0] += v[i][e];
  }
  row_sums<TPR>(s, lds[0]);
  const float mean = s[0] * a.inv_hidden;
  s[0] = 0.f;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int left = a.hidden - (t + i * TPR) * P::N;
#pragma unroll
    for (int e = 0; e < P::N; ++e) {
      v[i][e] -= mean;
      if (WIDE ? left > 0 : e < left) s[0] += v[i][e] * v[i][e];
    }
  }
  row_sums<TPR>(s, lds[1]);
  const float rstd = 1.f / sqrtf(s[0] * a.inv_hidden + a.eps);
  T *y = reinterpret_cast<T *>(a.y) + a.ys.offset(row);
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int p = t + i * TPR, left = a.hidden - p * P::N;
    if (p >= a.pieces) break;
    typename P::Values g, b;
    P::load(reinterpret_cast<const T *>(a.gamma) + p * P::N, left, g);
    P::load(reinterpret_cast<const T *>(a.beta) + p * P::N, left, b);
#pragma unroll
    for (int e = 0; e < P::N; ++e) v[i][e] = v[i][e] * rstd * g[e] + b[e];
    P::store(y + p * P::N, left, v[i]);
  }
  if (t == 0) {
    a.mean[row] = mean;
    a.rstd[row] = rstd;
  }
}

// A workgroup's rows one after the other; the next one is asked for before the sums of this one, which a workgroup waits for together.  Rows stay as they
// were loaded and are computed with twice, which takes half the registers of fp32 values.  8774 rows of 8192 bf16 elements, 431 MB: 86 to 90 us, 4.8 TB/s, what a
// large copy reaches; 2714 rows of 2563 elements, whose rows do not start on 16 bytes, 17 to 19 us, 2.3 TB/s: six rows to a workgroup, the last of them alone.
template <typename T, bool WIDE, int TPR, int E> __global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_bwd_kernel(const NormArgs a) {
  typedef Piece<T, WIDE> P;
  constexpr int NP = E / P::N, THREADS = TPR < 256 ? 256 : TPR, R = THREADS / TPR;
  __shared__ float lds[2][2 * 16];
  __shared__ float other[R > 1 ? R - 1 : 1][R > 1 ? 2 * TPR * E : 1];
  const int t = threadIdx.x % TPR, group = threadIdx.x / TPR, step = gridDim.x * R;
  float dg[NP][P::N], db[NP][P::N];
  typename P::Raw gain[NP], x[NP], dy[NP], next_x[NP], next_dy[NP];
  float mean = 0.f, rstd = 0.f, next_mean = 0.f, next_rstd = 0.f;
  auto ask = [&](int row) {
    const T *from_x = reinterpret_cast<const T *>(a.x) + a.xs.offset(row), *from_dy = reinterpret_cast<const T *>(a.dy) + a.ys.offset(row);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int p = t + i * TPR, left = a.hidden - p * P::N;
      next_x[i] = p < a.pieces ? P::get(from_x + p * P::N, left) : P::none();
      next_dy[i] = p < a.pieces ? P::get(from_dy + p * P::N, left) : P::none();
    }
    next_mean = a.mean_in[row];
    next_rstd = a.rstd_in[row];
  };
  int row = blockIdx.x * R + group;
  if (row < a.n) ask(row);
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int p = t + i * TPR;
    gain[i] = p < a.pieces ? P::get(reinterpret_cast<const T *>(a.gamma) + p * P::N, a.hidden - p * P::N) : P::none();
#pragma unroll
    for (int e = 0; e < P::N; ++e) dg[i][e] = db[i][e] = 0.f;
  }
  int turn = 0;
  // (rows that share a workgroup never wait for each other: one row to a wave, or one to a workgroup)
  for (; row < a.n; row += step, turn ^= 1) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      x[i] = next_x[i];
      dy[i] = next_dy[i];
    }
    mean = next_mean;
    rstd = next_rstd;
    if (row + step < a.n) ask(row + step);
    float s[2] = {0.f, 0.f};
    // (behind the end of a row dy is 0)
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int e = 0; e < P::N; ++e) {
        const float xh = ((float)x[i][e] - mean) * rstd, d = (float)dy[i][e], g = d * (float)gain[i][e];
        const bool is = WIDE || e < a.hidden - (t + i * TPR) * P::N;
        dg[i][e] += is ? d * xh : 0.f;
        db[i][e] += d;
        s[0] += g;
        s[1] += is ? g * xh : 0.f;
      }
    row_sums<TPR>(s, lds[turn]);
    const float c0 = s[0] * a.inv_hidden, c1 = s[1] * a.inv_hidden;
    T *dx = reinterpret_cast<T *>(a.dx) + a.xs.offset(row);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int p = t + i * TPR;
      if (p >= a.pieces) break;
      // (else the compiler keeps the fp32 values after all)
      settle(x[i]);
      settle(dy[i]);
      settle(gain[i]);
      typename P::Values o;
#pragma unroll
      for (int e = 0; e < P::N; ++e) {
        const float xh = ((float)x[i][e] - mean) * rstd, g = (float)dy[i][e] * (float)gain[i][e];
        o[e] = rstd * (g - c0 - xh * c1);
      }
      P::store(dx + p * P::N, a.hidden - p * P::N, o);
    }
  }
  if constexpr (R > 1) {   // the groups' sums meet in the first one
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < P::N; ++e) {
          other[group - 1][(2 * (i * P::N + e)) * TPR + t] = dg[i][e];
          other[group - 1][(2 * (i * P::N + e) + 1) * TPR + t] = db[i][e];
        }
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int e = 0; e < P::N; ++e)
#pragma unroll
        for (int r = 0; r < R - 1; ++r) {
          dg[i][e] += other[r][(2 * (i * P::N + e)) * TPR + t];
          db[i][e] += other[r][(2 * (i * P::N + e) + 1) * TPR + t];
        }
  }
  float *part = a.part + (int64_t)blockIdx.x * 2 * a.part_ld;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int p = t + i * TPR;
    if (p >= a.pieces) break;
    store_f32<P::N, true>(part + p * P::N, P::N, dg[i]);
    store_f32<P::N, true>(part + a.part_ld + p * P::N, P::N, db[i]);
  }
}

// Adds the workgroups' sums: 64 columns of [dgamma, dbeta] per workgroup, its 16 waves a sixteenth of the workgroups each (four waves: 7.6 us for 512
// workgroups and 2563 columns, a chain of loads).
__global__ void __launch_bounds__(1024) norm_join_kernel(const NormArgs a) {
  __shared__ float of_wave[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, width = 2 * a.part_ld, c = blockIdx.x * 64 + lane, col = c < a.part_ld ? c : c - a.part_ld;
  float s = 0.f;
  if (c < width) {
    const int begin = a.parts * wave / 16, end = a.parts * (wave + 1) / 16;
#pragma unroll 8
    for (int w = begin; w < end; ++w) s += a.part[(int64_t)w * width + c];
  }
  of_wave[wave][lane] = s;
  __syncthreads();
  if (wave > 0 || c >= width || col >= a.hidden) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) s += of_wave[w][lane];
  float *to = (c < a.part_ld ? a.dgamma : a.dbeta) + col;
  *to += s;
}

constexpr int kParts = 512;   // most workgroups of a backward

// Instances by (threads per row, elements per thread): the narrowest that holds the row.
struct Shape {
  void (*kernel)(NormArgs);
  int threads, rows;
};
#define S1F_NORM_SHAPES(KERNEL)                                                                                  \
  template <typename T, bool WIDE> Shape KERNEL##_shape(int hidden) {                                            \
    if (hidden <= 64 * 8) return {&KERNEL##_kernel<T, WIDE, 64, 8>, 256, 4};                                     \
    if (hidden <= 64 * 16) return {&KERNEL##_kernel<T, WIDE, 64, 16>, 256, 4};                                   \
    if (hidden <= 256 * 8) return {&KERNEL##_kernel<T, WIDE, 256, 8>, 256, 1};                                   \
    if (hidden <= 256 * 16) return {&KERNEL##_kernel<T, WIDE, 256, 16>, 256, 1};                                 \
    if (hidden <= 512 * 16) return {&KERNEL##_kernel<T, WIDE, 512, 16>, 512, 1};                                 \
    return {&KERNEL##_kernel<T, WIDE, 1024, 16>, 1024, 1};                                                       \
  }
S1F_NORM_SHAPES(norm_fwd)
S1F_NORM_SHAPES(norm_bwd)
static_assert(kMostHidden <= 1024 * 16, "a row stays in registers");

#define S1F_BY_TYPE(SHAPE, dtype, wide, hidden)                                                            \
  ((dtype) == S1F_BF16 ? ((wide) ? SHAPE<bf16_t, true>(hidden) : SHAPE<bf16_t, false>(hidden))             \
                       : ((wide) ? SHAPE<float, true>(hidden) : SHAPE<float, false>(hidden)))

int32_t part_ld_of(const s1f_rows *d) { return (d->hidden + 7) / 8 * 8; }
NormArgs args_of(const s1f_rows *d) {
  NormArgs a = {};
  a.xs = x_rows(d); a.ys = y_rows(d);
  a.n = (int32_t)(d->batch * d->rows); a.hidden = d->hidden;
  a.pieces = (int32_t)((d->hidden + elements_of_16_bytes(d->dtype) - 1) / elements_of_16_bytes(d->dtype));
  a.part_ld = part_ld_of(d);
  a.inv_hidden = 1.f / (float)d->hidden;
  return a;
}
bool wide_call(const s1f_rows *d) { return wide_rows(d, d->x_stride_b, d->x_stride_s) && wide_rows(d, d->y_stride_b, d->y_stride_s); }

}  // namespace
}  // namespace s1f

using namespace s1f;

extern "C" int s1f_layer_norm_fwd(const s1f_rows *desc, const void *x, const void *gamma, const void *beta, float eps, void *y, float *mean,
                                  float *rstd, void *hip_stream) {
  const int rc = check_rows(desc, true, true);
  if (rc != S1F_OK) return rc;
  if (!x || !gamma || !beta || !y || !mean || !rstd || !(eps >= 0.f)) return S1F_EINVAL;
  for (const void *p : {x, gamma, beta, (const void *)y})
    if (!on_element(p, desc->dtype)) return S1F_EINVAL;
  if (!on4(mean) || !on4(rstd)) return S1F_EINVAL;
  const bool wide = wide_call(desc) && on16(x) && on16(gamma) && on16(beta) && on16(y);
  NormArgs a = args_of(desc);
  a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.mean = mean; a.rstd = rstd; a.eps = eps;
  const Shape s = S1F_BY_TYPE(norm_fwd_shape, desc->dtype, wide, desc->hidden);
  return launch_rows_kernel(s.kernel, (a.n + s.rows - 1) / s.rows, s.threads, a, reinterpret_cast<hipStream_t>(hip_stream));
}

extern "C" size_t s1f_layer_norm_bwd_workspace_bytes(const s1f_rows *desc) {
  if (check_rows(desc, true, true) != S1F_OK) return 0;
  const int64_t n = desc->batch * desc->rows;
  return (size_t)((n < kParts ? n : kParts) * 2 * part_ld_of(desc) * 4);
}

extern "C" int s1f_layer_norm_bwd(const s1f_rows *desc, const void *dy, const void *x, const void *gamma, const float *mean, const float *rstd,
                                  void *dx, float *dgamma_acc, float *dbeta_acc, void *workspace, size_t workspace_bytes, void *hip_stream) {
  const int rc = check_rows(desc, true, true);
  if (rc != S1F_OK) return rc;
  if (!dy || !x || !gamma || !mean || !rstd || !dx || !dgamma_acc || !dbeta_acc || !workspace || !on16(workspace)) return S1F_EINVAL;
  for (const void *p : {dy, x, gamma, (const void *)dx})
    if (!on_element(p, desc->dtype)) return S1F_EINVAL;
  if (!on4(mean) || !on4(rstd) || !on4(dgamma_acc) || !on4(dbeta_acc)) return S1F_EINVAL;
  if (workspace_bytes < s1f_layer_norm_bwd_workspace_bytes(desc)) return S1F_EINVAL;
  const bool wide = wide_call(desc) && on16(dy) && on16(x) && on16(gamma) && on16(dx);
  NormArgs a = args_of(desc);
  a.x = x; a.dy = dy; a.gamma = gamma; a.mean_in = mean; a.rstd_in = rstd; a.dx = dx;
  a.dgamma = dgamma_acc; a.dbeta = dbeta_acc; a.part = reinterpret_cast<float *>(workspace);
  const Shape s = S1F_BY_TYPE(norm_bwd_shape, desc->dtype, wide, desc->hidden);
  const int groups = (a.n + s.rows - 1) / s.rows;
  a.parts = groups < kParts ? groups : kParts;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const int e = launch_rows_kernel(s.kernel, a.parts, s.threads, a, st);
  if (e != S1F_OK) return e;
  return launch_rows_kernel(&norm_join_kernel, (2 * a.part_ld + 63) / 64, 1024, a, st);
}
