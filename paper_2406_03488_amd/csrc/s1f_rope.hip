// Queries and keys of a segment turned by their positions, on the way from a projection into the attention (queries) and the K/V cache
// (keys; values go along as they are), with or without a norm of every head in front, and the way back.
//
//   forward    y = x, or with the norm y = x * rstd * gain,  rstd = 1 / sqrt(sum(x^2) / d + eps)
//              pair i of the rotary_dim / 2 that are turned, as a complex number:  out_i = m * e^(i p f_i) * y_i;  p position, m magnitude
//   backward   dy_i = m * e^(-i p f_i) * dout_i;  with the norm  xhat = x * rstd,  dgain += sum over rows and heads of dy * xhat,
//              g = dy * gain,  dx = rstd * (g - xhat * sum(g * xhat) / d)
//
// Bound by memory: each element is read and written once, between which a row's angles, computed once for all heads that a thread takes, are
// next to nothing.  A row of a head lies in the registers of L lanes, a lane has PW pairs of it, both elements of each, so that no rotation asks
// another lane for anything.  Angles are products in 64 bits: at position 2^20 one in 32 bits is off by 2^-4.  The norm's sums are fp32, as is everything between
// load and store; results are rounded once.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "rows.hpp"

namespace s1f {
namespace {

struct HeadStrides {
  int64_t sb, sh, ss;
};

struct RopeArgs {
  const void *src_q, *src_k, *src_v;    // forward: projections; backward: gradients (k, v: fp32 accumulators)
  void *dst_q, *dst_k, *dst_v;
  const void *x_q, *x_k;                // backward with the norm: projections, strides of dst
  const void *gain_q, *gain_k;
  HeadStrides src_qs, src_ks, dst_qs, dst_ks;
  const double *freqs;
  const int64_t *positions;             // or null: first_position and on
  int64_t positions_sb, first_position;
  float *part;                          // [workgroup][q, k][dim]
  float *dgain_q, *dgain_k;
  Divisor by_rows;
  int32_t n, dim, half, rotary, items;  // batch * rows; half: pairs that are turned; items: lanes' shares of PW pairs in a row
  int32_t n_q, n_k, n_v;                // heads: the list of a row's heads is q, k, v
  int32_t log_rows;                     // rows that a workgroup works on side by side
  int32_t parts;
  float magnitude, eps, inv_dim;
};

// N consecutive elements, aligned to all of them or to 16 bytes.
template <typename T, int N> struct Run {
  static constexpr int BYTES = N * (int)sizeof(T), PIECE = BYTES > 16 ? 16 / (int)sizeof(T) : N, PIECES = N / PIECE;
  typedef T Vec __attribute__((ext_vector_type(PIECE)));
  Vec v[PIECES];
  S1F_DEV void load(const T *p) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) v[i] = reinterpret_cast<const Vec *>(p)[i];
  }
  S1F_DEV float operator[](int e) const { return (float)v[e / PIECE][e % PIECE]; }
  S1F_DEV void set(int e, float x) { v[e / PIECE][e % PIECE] = (T)x; }
  S1F_DEV void store(T *p) const {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) reinterpret_cast<Vec *>(p)[i] = v[i];
  }
};

// cos and sin of a 64-bit angle: the quarter turn and the rest in 64 bits (pi/2 as two numbers; a fused product takes off the first exactly), the rest's
// series in 32, to 2^-25 of the result.
S1F_DEV void cos_sin(double angle, float &c, float &s) {
  const double turns = rint(angle * 0.63661977236758134308);
  const float x = (float)fma(-turns, 6.123233995736766036e-17, fma(-turns, 1.5707963267948965580, angle));
  const int quarter = (int)(turns - 4.0 * floor(turns * 0.25));
  const float q = x * x;
  const float sn = x + x * q * (-1.f / 6 + q * (1.f / 120 + q * (-1.f / 5040 + q * (1.f / 362880))));
  const float cs = 1.f + q * (-0.5f + q * (1.f / 24 + q * (-1.f / 720 + q * (1.f / 40320 + q * (-1.f / 3628800)))));
  c = quarter & 1 ? sn : cs;
  s = quarter & 1 ? cs : sn;
  if (quarter == 1 || quarter == 2) c = -c;
  if (quarter >= 2) s = -s;
}

// Sum over L neighbouring lanes, in each of them.
template <int CTRL> S1F_DEV float plus_lane(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int L> S1F_DEV float sum_of(float x) {
  if constexpr (L >= 2) x = plus_lane<0xb1>(x);     // quad_perm 1 0 3 2
  if constexpr (L >= 4) x = plus_lane<0x4e>(x);     // quad_perm 2 3 0 1
  if constexpr (L >= 8) x = plus_lane<0x141>(x);    // mirrored in 8 lanes
  if constexpr (L >= 16) x = plus_lane<0x140>(x);   // mirrored in 16
  if constexpr (L >= 32) x += __shfl_xor(x, 16);
  if constexpr (L >= 64) x = sum_xor32(x);
  return x;
}

// The lane's share of a row: PW pairs, the elements [col(0), +PW) and [col(1), +PW).
template <int PW, bool PAIRS> struct Share {
  int at[2];
  S1F_DEV Share(const RopeArgs &a, int item) {
    if (PAIRS || item * PW >= a.half) {
      at[0] = PAIRS ? 2 * PW * item : a.rotary + 2 * (item * PW - a.half);
      at[1] = at[0] + PW;
    } else {
      at[0] = item * PW;
      at[1] = at[0] + a.half;
    }
  }
  // which of the lane's elements e < 2 PW is the first, the second of its pair i
  S1F_DEV static constexpr int first(int i) { return PAIRS ? 2 * i : i; }
  S1F_DEV static constexpr int second(int i) { return PAIRS ? 2 * i + 1 : PW + i; }
};

// T: type of the tensors, K: of the keys' and values' source (fp32 accumulators in the backward).  L lanes to a row, IT shares to a lane.  BACK: turn back.
// A workgroup works on 2^log_rows rows; its groups of L lanes beyond that share the heads of a row with each other and with the workgroups of the grid's y.
template <typename T, typename K, int PW, int L, int IT, bool PAIRS, bool NORM, bool BACK> __global__ void __launch_bounds__(256) rope_kernel(const RopeArgs a) {
  constexpr int E = 2 * PW, U = NORM && BACK ? 2 : 4;   // U: heads asked for together
  constexpr bool GAINS = NORM && BACK;
  const int group = threadIdx.x / L, in_row = group & ((1 << a.log_rows) - 1);
  const int slots_here = (256 / L) >> a.log_rows, slots = slots_here * gridDim.y, slot = blockIdx.y * slots_here + (group >> a.log_rows);
  float dg_q[IT][E], dg_k[IT][E];
  if constexpr (GAINS) {
#pragma unroll
    for (int t = 0; t < IT; ++t)
#pragma unroll
      for (int e = 0; e < E; ++e) dg_q[t][e] = dg_k[t][e] = 0.f;
  }
  for (int row = (blockIdx.x << a.log_rows) + in_row; row < a.n; row += gridDim.x << a.log_rows) {
    int b, r;
    div_mod(row, a.by_rows, b, r);
    const int64_t position = a.positions ? a.positions[b * a.positions_sb + r] : a.first_position + r;
    float c[IT][PW], s[IT][PW];
    int at[IT][2];
    bool has[IT];
#pragma unroll
    for (int t = 0; t < IT; ++t) {
      const int item = threadIdx.x % L + t * L;
      const Share<PW, PAIRS> share(a, item);
      has[t] = item < a.items;
      at[t][0] = share.at[0];
      at[t][1] = share.at[1];
#pragma unroll
      for (int i = 0; i < PW; ++i) {
        const int pair = item * PW + i;
        c[t][i] = 1.f;
        s[t][i] = 0.f;
        if (pair < a.half) {
          cos_sin((double)position * a.freqs[pair], c[t][i], s[t][i]);
          c[t][i] *= a.magnitude;
          s[t][i] *= BACK ? -a.magnitude : a.magnitude;
        }
      }
    }
    // heads [i, end) of the list, `from` the number of the first
    int head = slot;
    auto walk = [&](auto kind, int from, int end, const void *src, const HeadStrides &ss, void *dst, const HeadStrides &ds, const void *xs, const void *gains,
                    float (&dg)[IT][E]) {
      typedef decltype(kind) S;
      if (head >= end) return;
      float gain[IT][E];
      if constexpr (NORM) {
#pragma unroll
        for (int t = 0; t < IT; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            Run<T, PW> g;
            if (has[t]) g.load(reinterpret_cast<const T *>(gains) + at[t][h]);
#pragma unroll
            for (int e = 0; e < PW; ++e) gain[t][h * PW + e] = has[t] ? g[e] : 0.f;
          }
      }
      const S *p = reinterpret_cast<const S *>(src) + b * ss.sb + r * ss.ss;
      T *q = reinterpret_cast<T *>(dst) + b * ds.sb + r * ds.ss;
      const T *px = reinterpret_cast<const T *>(xs) + b * ds.sb + r * ds.ss;
      while (head < end) {
        Run<S, PW> in[U][IT][2];
        Run<T, PW> x[GAINS ? U : 1][IT][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = head + u * slots - from;
          if (h >= end - from) break;
#pragma unroll
          for (int t = 0; t < IT; ++t)
            if (has[t]) {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                in[u][t][k].load(p + h * ss.sh + at[t][k]);
                if constexpr (GAINS) x[u][t][k].load(px + h * ds.sh + at[t][k]);
              }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = head + u * slots - from;
          if (h >= end - from) break;
          float v[IT][E];
#pragma unroll
          for (int t = 0; t < IT; ++t)
#pragma unroll
            for (int e = 0; e < E; ++e) v[t][e] = has[t] ? in[u][t][e / PW][e % PW] : 0.f;
          if constexpr (NORM && !BACK) {
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < IT; ++t)
#pragma unroll
              for (int e = 0; e < E; ++e) sum += v[t][e] * v[t][e];
            const float rstd = 1.f / sqrtf(sum_of<L>(sum) * a.inv_dim + a.eps);
#pragma unroll
            for (int t = 0; t < IT; ++t)
#pragma unroll
              for (int e = 0; e < E; ++e) v[t][e] = v[t][e] * rstd * gain[t][e];
          }
#pragma unroll
          for (int t = 0; t < IT; ++t)
#pragma unroll
            for (int i = 0; i < PW; ++i) {
              constexpr auto F = &Share<PW, PAIRS>::first, G = &Share<PW, PAIRS>::second;
              float &re = v[t][F(i)], &im = v[t][G(i)];
              const bool turned = (int)(threadIdx.x % L + t * L) * PW + i < a.half;   // (the others stay what they are, infinities too)
              const float was = re;
              re = turned ? was * c[t][i] - im * s[t][i] : was;
              im = turned ? im * c[t][i] + was * s[t][i] : im;
            }
          if constexpr (GAINS) {
            float w[IT][E], squares = 0.f, along = 0.f;
#pragma unroll
            for (int t = 0; t < IT; ++t)
#pragma unroll
              for (int e = 0; e < E; ++e) {
                w[t][e] = has[t] ? x[u][t][e / PW][e % PW] : 0.f;
                squares += w[t][e] * w[t][e];
              }
            const float rstd = 1.f / sqrtf(sum_of<L>(squares) * a.inv_dim + a.eps);
#pragma unroll
            for (int t = 0; t < IT; ++t)
#pragma unroll
              for (int e = 0; e < E; ++e) {
                w[t][e] *= rstd;
                dg[t][e] += v[t][e] * w[t][e];
                v[t][e] *= gain[t][e];
                along += v[t][e] * w[t][e];
              }
            along = sum_of<L>(along) * a.inv_dim;
#pragma unroll
            for (int t = 0; t < IT; ++t)
#pragma unroll
              for (int e = 0; e < E; ++e) v[t][e] = rstd * (v[t][e] - w[t][e] * along);
          }
#pragma unroll
          for (int t = 0; t < IT; ++t)
            if (has[t]) {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                Run<T, PW> o;
#pragma unroll
                for (int e = 0; e < PW; ++e) o.set(e, v[t][k * PW + e]);
                o.store(q + h * ds.sh + at[t][k]);
              }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (head < end) head += slots;
      }
    };
    walk(T{}, 0, a.n_q, a.src_q, a.src_qs, a.dst_q, a.dst_qs, a.x_q, a.gain_q, dg_q);
    walk(K{}, a.n_q, a.n_q + a.n_k, a.src_k, a.src_ks, a.dst_k, a.dst_ks, a.x_k, a.gain_k, dg_k);
    // values: as they are, in runs of E elements one behind the other
    const int first_v = a.n_q + a.n_k, end = first_v + a.n_v;
    if (head >= end) continue;
    const K *p = reinterpret_cast<const K *>(a.src_v) + b * a.src_ks.sb + r * a.src_ks.ss;
    T *q = reinterpret_cast<T *>(a.dst_v) + b * a.dst_ks.sb + r * a.dst_ks.ss;
    while (head < end) {
      Run<K, PW> in[U][IT][2];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = head + u * slots - first_v;
        if (h >= a.n_v) break;
#pragma unroll
        for (int t = 0; t < IT; ++t)
          if (has[t]) {
#pragma unroll
            for (int k = 0; k < 2; ++k) in[u][t][k].load(p + h * a.src_ks.sh + E * (threadIdx.x % L + t * L) + k * PW);
          }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = head + u * slots - first_v;
        if (h >= a.n_v) break;
#pragma unroll
        for (int t = 0; t < IT; ++t)
          if (has[t]) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              Run<T, PW> o;
#pragma unroll
              for (int e = 0; e < PW; ++e) o.set(e, in[u][t][k][e]);
              o.store(q + h * a.dst_ks.sh + E * (threadIdx.x % L + t * L) + k * PW);
            }
          }
      }
      head += U * slots;
    }
  }
  if constexpr (GAINS) {   // the groups' sums of q, then of k, in their order; columns [item][element]
    constexpr int GROUPS = 256 / L, COLS = L * IT * E;
    __shared__ float sums[GROUPS][COLS + 1];
    float *part = a.part + (int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.dim;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      __syncthreads();
#pragma unroll
      for (int t = 0; t < IT; ++t)
#pragma unroll
        for (int e = 0; e < E; ++e) sums[group][(t * E + e) * L + threadIdx.x % L] = side ? dg_k[t][e] : dg_q[t][e];
      __syncthreads();
      for (int col = threadIdx.x; col < COLS; col += 256) {
        const int item = col % L + col / (L * E) * L, e = col / L % E;
        if (item >= a.items) continue;
        float sum = 0.f;
        for (int g = 0; g < GROUPS; ++g) sum += sums[g][col];
        const Share<PW, PAIRS> share(a, item);
        part[side * a.dim + share.at[e / PW] + e % PW] = sum;
      }
    }
  }
}

// Adds the workgroups' sums: 64 columns of [q, k][dim] per workgroup, its 16 waves a sixteenth of the parts each.
__global__ void __launch_bounds__(1024) rope_join_kernel(const RopeArgs a) {
  __shared__ float of_wave[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, width = 2 * a.dim, col = blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (col < width) {
    const int begin = a.parts * wave / 16, end = a.parts * (wave + 1) / 16;
#pragma unroll 8
    for (int p = begin; p < end; ++p) sum += a.part[(int64_t)p * width + col];
  }
  of_wave[wave][lane] = sum;
  __syncthreads();
  if (wave > 0 || col >= width) return;
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) sum += of_wave[w][lane];
  float *to = col < a.dim ? a.dgain_q + col : a.dgain_k + col - a.dim;
  *to += sum;
}

// ---- host ------------------------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostTokens = int64_t(1) << 26;
constexpr int32_t kMostHeads = 1 << 16, kMostDim = 256;
constexpr int kMostParts = 1024;   // workgroups of a backward with the norm

bool strides_fit(const s1f_heads *d, int heads, int64_t rows, int64_t sb, int64_t sh, int64_t ss) {
  return (rows == 1 || ss >= d->head_dim) && (heads == 1 || sh >= d->head_dim) && (d->batch == 1 || sb >= d->head_dim);
}
int check_heads(const s1f_heads *d) {
  if (!d || d->batch < 1 || d->n_q_heads < 1 || d->n_kv_heads < 1 || d->reserved != 0) return S1F_EINVAL;
  if (d->interleaved != 0 && d->interleaved != 1) return S1F_EINVAL;
  if (d->dtype != S1F_F32 && d->dtype != S1F_BF16) return S1F_EUNSUPPORTED;
  if (d->head_dim < 2 || d->head_dim % 2 != 0 || d->head_dim > kMostDim || d->n_q_heads > kMostHeads || d->n_kv_heads > kMostHeads) return S1F_EUNSUPPORTED;
  if (d->rotary_dim < 0 || d->rotary_dim % 2 != 0 || d->rotary_dim > d->head_dim) return S1F_EINVAL;
  if (d->rows < 1) return S1F_ERANGE;
  if (d->rows > kMostTokens || d->batch * d->rows > kMostTokens) return S1F_EUNSUPPORTED;
  if (!strides_fit(d, d->n_q_heads, d->rows, d->q_stride_b, d->q_stride_h, d->q_stride_s) || !strides_fit(d, d->n_q_heads, d->rows, d->rot_stride_b, d->rot_stride_h, d->rot_stride_s) ||
      !strides_fit(d, d->n_kv_heads, d->rows, d->kv_stride_b, d->kv_stride_h, d->kv_stride_s) ||
      !strides_fit(d, d->n_kv_heads, d->cache_capacity, d->cache_stride_b, d->cache_stride_h, d->cache_stride_s))
    return S1F_EINVAL;
  return S1F_OK;
}
int check_call(const s1f_heads *d, int64_t seg_off, const double *freqs, float magnitude, const int64_t *positions, bool values) {
  const int rc = check_heads(d);
  if (rc != S1F_OK) return rc;
  if ((d->rotary_dim > 0 && !freqs) || (reinterpret_cast<uintptr_t>(freqs) & 7) || (reinterpret_cast<uintptr_t>(positions) & 7)) return S1F_EINVAL;
  if (!(magnitude - magnitude == 0.f) || !values) return S1F_EINVAL;
  if (seg_off < 0 || d->cache_capacity < d->rows || seg_off > d->cache_capacity - d->rows) return S1F_ERANGE;
  return S1F_OK;
}

// Row stride, batch stride and head stride of one side, and its tensors, as far as elements of PW pairs can be read from there.
struct Alignment {
  uint64_t bits = 0;   // of addresses and strides, in bytes
  void strides(const s1f_heads *d, int heads, int64_t sb, int64_t sh, int64_t ss, int64_t esz) {
    if (d->batch > 1) bits |= (uint64_t)(sb * esz);
    if (heads > 1) bits |= (uint64_t)(sh * esz);
    if (d->rows > 1) bits |= (uint64_t)(ss * esz);
  }
  void pointer(const void *p) { bits |= reinterpret_cast<uintptr_t>(p); }
  bool at_least(int64_t bytes) const { return (bits & (uint64_t)((bytes < 16 ? bytes : 16) - 1)) == 0; }
};

// Pairs to a lane: as many as a row's halves and all addresses allow, 8 at most (16 bytes of bf16).
int pairs_per_lane(const s1f_heads *d, const Alignment &typed, const Alignment &wide, int64_t esz) {
  for (int pw = 8; pw > 1; pw /= 2) {
    if (d->head_dim % (2 * pw) != 0 || (!d->interleaved && d->rotary_dim / 2 % pw != 0)) continue;
    if (typed.at_least(pw * esz) && wide.at_least(pw * 4)) return pw;
  }
  return 1;
}

struct Instance {
  void (*kernel)(RopeArgs);
  int lanes;
};
template <typename T, typename K, bool PAIRS, bool NORM, bool BACK> Instance instance_of(int pw, int items) {
  if (pw == 8) {
    if (items <= 4) return {&rope_kernel<T, K, 8, 4, 1, PAIRS, NORM, BACK>, 4};
    if (items <= 8) return {&rope_kernel<T, K, 8, 8, 1, PAIRS, NORM, BACK>, 8};
    return {&rope_kernel<T, K, 8, 16, 1, PAIRS, NORM, BACK>, 16};
  }
  if (pw == 4) {
    if (items <= 16) return {&rope_kernel<T, K, 4, 16, 1, PAIRS, NORM, BACK>, 16};
    return {&rope_kernel<T, K, 4, 32, 1, PAIRS, NORM, BACK>, 32};
  }
  if (pw == 2) {
    if (items <= 32) return {&rope_kernel<T, K, 2, 32, 1, PAIRS, NORM, BACK>, 32};
    return {&rope_kernel<T, K, 2, 64, 1, PAIRS, NORM, BACK>, 64};
  }
  return {&rope_kernel<T, K, 1, 64, 2, PAIRS, NORM, BACK>, 64};
}
static_assert(kMostDim / 2 <= 64 * 2, "a row has a place in the lanes");

// Rows side by side in a workgroup, and workgroups: x along the rows, y along the heads.
struct Grid {
  int log_rows;
  int64_t x, y;
};
Grid grid_for(int64_t n, int heads, int lanes, bool gains) {
  const int groups = 256 / lanes;
  Grid g = {0, 0, 1};
  while ((2 << g.log_rows) <= groups && (int64_t(1) << g.log_rows) < n) ++g.log_rows;
  g.x = (n + (int64_t(1) << g.log_rows) - 1) >> g.log_rows;
  const int slots = groups >> g.log_rows;
  // one head to a group of lanes where there are few, four (those asked for together) where there are many workgroups
  const int64_t most = gains ? kMostParts : 4096;
  const int64_t y = (heads + slots - 1) / slots;
  while (g.y < y && g.x * g.y * 2 <= most) g.y *= 2;
  if (g.y > y) g.y = y;
  g.x = std::min(g.x, gains ? (int64_t)kMostParts : int64_t(1) << 20);   // (workgroups walk the rows; threads of a launch stay below 2^32)
  return g;
}

RopeArgs args_of(const s1f_heads *d, const double *freqs, float magnitude, const int64_t *positions, int64_t positions_sb, int64_t first_position) {
  RopeArgs a = {};
  a.freqs = freqs; a.magnitude = magnitude;
  a.positions = positions; a.positions_sb = positions_sb; a.first_position = first_position;
  a.by_rows = Divisor::of(d->rows);
  a.n = (int32_t)(d->batch * d->rows); a.dim = d->head_dim; a.rotary = d->rotary_dim; a.half = d->rotary_dim / 2;
  a.n_q = d->n_q_heads; a.n_k = d->n_kv_heads;
  a.inv_dim = 1.f / (float)d->head_dim;
  return a;
}

template <bool NORM, bool BACK> int launch(const s1f_heads *d, RopeArgs a, hipStream_t st) {
  const int64_t esz = d->dtype == S1F_BF16 ? 2 : 4;
  Alignment typed, wide;   // tensors of the type, and the fp32 accumulators
  Alignment &kv = BACK ? wide : typed;
  const int64_t kv_esz = BACK ? 4 : esz;
  typed.strides(d, d->n_q_heads, a.src_qs.sb, a.src_qs.sh, a.src_qs.ss, esz);
  typed.strides(d, d->n_q_heads, a.dst_qs.sb, a.dst_qs.sh, a.dst_qs.ss, esz);
  typed.strides(d, d->n_kv_heads, a.dst_ks.sb, a.dst_ks.sh, a.dst_ks.ss, esz);
  kv.strides(d, d->n_kv_heads, a.src_ks.sb, a.src_ks.sh, a.src_ks.ss, kv_esz);
  for (const void *p : {a.src_q, (const void *)a.dst_q, (const void *)a.dst_k, (const void *)a.dst_v, a.x_q, a.x_k, a.gain_q, a.gain_k}) typed.pointer(p);
  kv.pointer(a.src_k);
  kv.pointer(a.src_v);
  const int pw = pairs_per_lane(d, typed, wide, esz);
  a.items = d->head_dim / (2 * pw);
  auto pick = [&](auto t, auto k) {
    typedef decltype(t) T;
    typedef decltype(k) K;
    return d->interleaved ? instance_of<T, K, true, NORM, BACK>(pw, a.items) : instance_of<T, K, false, NORM, BACK>(pw, a.items);
  };
  const Instance in = d->dtype == S1F_F32 ? pick(float{}, float{}) : BACK ? pick(bf16_t{}, float{}) : pick(bf16_t{}, bf16_t{});
  const Grid g = grid_for(a.n, a.n_q + a.n_k + a.n_v, in.lanes, NORM && BACK);
  a.log_rows = g.log_rows;
  a.parts = (int32_t)(g.x * g.y);
  void *params[] = {&a};
  if (hipLaunchKernel(reinterpret_cast<const void *>(in.kernel), dim3((unsigned)g.x, (unsigned)g.y), dim3(256), params, 0, st) != hipSuccess) return S1F_EDEVICE;
  if (!(NORM && BACK)) return S1F_OK;
  return launch_rows_kernel(&rope_join_kernel, (2 * a.dim + 63) / 64, 1024, a, st);
}

// Tensors of a call: 0 where a pointer is missing or does not lie on an element.
bool tensors_ok(int32_t dtype, std::initializer_list<const void *> ps) {
  for (const void *p : ps)
    if (!p || !on_element(p, dtype)) return false;
  return true;
}

template <bool NORM>
int forward(const s1f_heads *d, const void *q, const void *k, const void *v, const void *q_gain, const void *k_gain, float eps, const double *freqs,
            float magnitude, const int64_t *positions, int64_t positions_sb, int64_t first_position, int64_t seg_off, void *q_rot, void *k_cache,
            void *v_cache, void *stream) {
  const int rc = check_call(d, seg_off, freqs, magnitude, positions, !v == !v_cache);
  if (rc != S1F_OK) return rc;
  if (!tensors_ok(d->dtype, {q, k, q_rot, k_cache}) || !on_element(v, d->dtype) || !on_element(v_cache, d->dtype)) return S1F_EINVAL;
  if (NORM && (!tensors_ok(d->dtype, {q_gain, k_gain}) || !(eps >= 0.f))) return S1F_EINVAL;
  RopeArgs a = args_of(d, freqs, magnitude, positions, positions_sb, first_position);
  const int64_t to = seg_off * d->cache_stride_s * (d->dtype == S1F_BF16 ? 2 : 4);
  a.src_q = q; a.src_k = k; a.src_v = v;
  a.dst_q = q_rot;
  a.dst_k = reinterpret_cast<char *>(k_cache) + to;
  a.dst_v = v ? reinterpret_cast<char *>(v_cache) + to : nullptr;
  a.n_v = v ? d->n_kv_heads : 0;
  a.gain_q = q_gain; a.gain_k = k_gain; a.eps = eps;
  a.src_qs = {d->q_stride_b, d->q_stride_h, d->q_stride_s};
  a.src_ks = {d->kv_stride_b, d->kv_stride_h, d->kv_stride_s};
  a.dst_qs = {d->rot_stride_b, d->rot_stride_h, d->rot_stride_s};
  a.dst_ks = {d->cache_stride_b, d->cache_stride_h, d->cache_stride_s};
  return launch<NORM, false>(d, a, reinterpret_cast<hipStream_t>(stream));
}

template <bool NORM>
int backward(const s1f_heads *d, const void *dq_rot, const float *dk_acc, const float *dv_acc, RopeArgs a, int64_t seg_off, void *dq, void *dk, void *dv,
             hipStream_t st) {
  const int64_t from = seg_off * d->cache_stride_s;
  a.src_q = dq_rot; a.src_k = dk_acc + from;
  a.src_v = dv ? dv_acc + from : nullptr;
  a.dst_q = dq; a.dst_k = dk; a.dst_v = dv;
  a.n_v = dv ? d->n_kv_heads : 0;
  a.src_qs = {d->rot_stride_b, d->rot_stride_h, d->rot_stride_s};
  a.src_ks = {d->cache_stride_b, d->cache_stride_h, d->cache_stride_s};
  a.dst_qs = {d->q_stride_b, d->q_stride_h, d->q_stride_s};
  a.dst_ks = {d->kv_stride_b, d->kv_stride_h, d->kv_stride_s};
  return launch<NORM, true>(d, a, st);
}
int check_backward(const s1f_heads *d, const void *dq_rot, const float *dk_acc, const float *dv_acc, int64_t seg_off, const double *freqs, float magnitude,
                   const int64_t *positions, void *dq, void *dk, void *dv) {
  const int rc = check_call(d, seg_off, freqs, magnitude, positions, !dv_acc == !dv);
  if (rc != S1F_OK) return rc;
  return tensors_ok(d->dtype, {dq_rot, dq, dk}) && on_element(dv, d->dtype) && dk_acc && on4(dk_acc) && on4(dv_acc) ? S1F_OK : S1F_EINVAL;
}

}  // namespace
}  // namespace s1f

using namespace s1f;

extern "C" int s1f_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, int64_t trained_rows, double slow_turns,
                                    double fast_turns, double *freqs, float *magnitude) {
  if (rotary_dim < 2 || rotary_dim % 2 != 0 || !freqs || !magnitude || !(base > 0.0) || !std::isfinite(base)) return S1F_EINVAL;
  if (scaling < S1F_ROPE_PLAIN || scaling > S1F_ROPE_PARTS) return S1F_EINVAL;
  if (scaling != S1F_ROPE_PLAIN && (!(factor > 0.0) || !std::isfinite(factor))) return S1F_EINVAL;
  if (scaling == S1F_ROPE_BASE && rotary_dim < 4) return S1F_EINVAL;
  if (scaling == S1F_ROPE_PARTS && (trained_rows < 1 || !(slow_turns >= 0.0) || !(fast_turns > slow_turns) || !std::isfinite(fast_turns) || factor < 1.0)) return S1F_EINVAL;
  constexpr double kTwoPi = 6.283185307179586477;
  if (scaling == S1F_ROPE_BASE) base *= std::pow(factor, (double)rotary_dim / (rotary_dim - 2));
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rotary_dim);
    if (scaling == S1F_ROPE_LINEAR) f /= factor;
    if (scaling == S1F_ROPE_PARTS) {
      const double turns = (double)trained_rows * f / kTwoPi, keep = std::fmin(std::fmax((turns - slow_turns) / (fast_turns - slow_turns), 0.0), 1.0);
      f = f * keep + f / factor * (1.0 - keep);
    }
    freqs[i] = f;
  }
  *magnitude = scaling == S1F_ROPE_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return S1F_OK;
}

extern "C" int s1f_rope_fwd(const s1f_heads *desc, const void *q, const void *k, const void *v, const double *freqs, float magnitude,
                            const int64_t *positions, int64_t positions_stride_b, int64_t first_position, int64_t seg_off, void *q_rot, void *k_cache,
                            void *v_cache, void *hip_stream) {
  return forward<false>(desc, q, k, v, nullptr, nullptr, 0.f, freqs, magnitude, positions, positions_stride_b, first_position, seg_off, q_rot, k_cache,
                        v_cache, hip_stream);
}

extern "C" int s1f_qk_norm_rope_fwd(const s1f_heads *desc, const void *q, const void *k, const void *v, const void *q_gain, const void *k_gain, float eps,
                                    const double *freqs, float magnitude, const int64_t *positions, int64_t positions_stride_b, int64_t first_position,
                                    int64_t seg_off, void *q_rot, void *k_cache, void *v_cache, void *hip_stream) {
  return forward<true>(desc, q, k, v, q_gain, k_gain, eps, freqs, magnitude, positions, positions_stride_b, first_position, seg_off, q_rot, k_cache,
                       v_cache, hip_stream);
}

extern "C" int s1f_rope_bwd(const s1f_heads *desc, const void *dq_rot, const float *dk_prefix_acc, const float *dv_prefix_acc, const double *freqs,
                            float magnitude, const int64_t *positions, int64_t positions_stride_b, int64_t first_position, int64_t seg_off, void *dq, void *dk,
                            void *dv, void *hip_stream) {
  const int rc = check_backward(desc, dq_rot, dk_prefix_acc, dv_prefix_acc, seg_off, freqs, magnitude, positions, dq, dk, dv);
  if (rc != S1F_OK) return rc;
  return backward<false>(desc, dq_rot, dk_prefix_acc, dv_prefix_acc, args_of(desc, freqs, magnitude, positions, positions_stride_b, first_position), seg_off, dq,
                         dk, dv, reinterpret_cast<hipStream_t>(hip_stream));
}

extern "C" size_t s1f_qk_norm_rope_bwd_workspace_bytes(const s1f_heads *desc) {
  if (check_heads(desc) != S1F_OK) return 0;
  // (of the launch with the most workgroups: how many lanes a row takes depends on the call's addresses)
  return (size_t)kMostParts * 2 * desc->head_dim * 4;
}

extern "C" int s1f_qk_norm_rope_bwd(const s1f_heads *desc, const void *dq_rot, const float *dk_prefix_acc, const float *dv_prefix_acc, const void *q,
                                    const void *k, const void *q_gain, const void *k_gain, float eps, const double *freqs, float magnitude,
                                    const int64_t *positions, int64_t positions_stride_b, int64_t first_position, int64_t seg_off, void *dq, void *dk,
                                    void *dv, float *dq_gain_acc, float *dk_gain_acc, void *workspace, size_t workspace_bytes, void *hip_stream) {
  const int rc = check_backward(desc, dq_rot, dk_prefix_acc, dv_prefix_acc, seg_off, freqs, magnitude, positions, dq, dk, dv);
  if (rc != S1F_OK) return rc;
  if (!tensors_ok(desc->dtype, {q, k, q_gain, k_gain}) || !(eps >= 0.f) || !dq_gain_acc || !dk_gain_acc || !on4(dq_gain_acc) || !on4(dk_gain_acc) ||
      !workspace || !on16(workspace) || workspace_bytes < s1f_qk_norm_rope_bwd_workspace_bytes(desc))
    return S1F_EINVAL;
  RopeArgs a = args_of(desc, freqs, magnitude, positions, positions_stride_b, first_position);
  a.x_q = q; a.x_k = k; a.gain_q = q_gain; a.gain_k = k_gain; a.eps = eps;
  a.dgain_q = dq_gain_acc; a.dgain_k = dk_gain_acc; a.part = reinterpret_cast<float *>(workspace);
  return backward<true>(desc, dq_rot, dk_prefix_acc, dv_prefix_acc, a, seg_off, dq, dk, dv, reinterpret_cast<hipStream_t>(hip_stream));
}
