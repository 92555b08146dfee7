// Cross entropy of every row of a segment over a large vocabulary, with its gradient: what the last stage of a pipeline does behind its
// last layer.  z = x W^T are the scores of a row, t its target.
//
//   forward    lse = log sum_v exp(z_v),  loss = lse - z_t
//   backward   dz_v = (exp(z_v - lse) - [v = t]) * dloss,  dx = dz W,  dW += dz^T x
//
// Scores never exist in memory as a whole.  The forward's tiles of scores leave a maximum and a sum of exponentials per row; the
// backward computes the scores of a piece of the vocabulary anew, writes that piece's dz in bf16 (rounded once, as the attention kernels round
// their score gradients; fp32 calls: three bf16 planes of it, nothing rounded), and both products read it.
// Rows without a target take no part: the others are gathered into consecutive rows first, so nothing is computed for them and whatever
// they hold, infinities and NaN included, stays theirs.  The number of rows that count is known on the device only; workgroups
// behind them end at once.
#include <algorithm>
#include <atomic>

#include "loss_tile.hpp"
#include "rows.hpp"

namespace s1f {
namespace {

struct LossArgs {
  const int64_t *targets;
  int64_t targets_sb;
  const float *dloss, *lse_in;
  const void *x, *weight;
  int64_t weight_stride;
  float *loss, *lse;
  void *dx, *dweight;
  int64_t dweight_stride;
  RowsOf xs;
  int32_t n, hidden, width, vocab;    // width: hidden rounded up to 8, as packed rows have it
  // workspace
  int32_t *count, *row_of, *slot_of, *target_of;   // counted rows; their numbers; a row's place among them (-1: none); targets
  float *target_score;                             // [slot]
  float *of_row;                                   // [slot][lse, dloss]
  float *stats;                                    // [tile of the vocabulary][slot][maximum, sum]
  bf16_t *rows, *packed, *dz;                      // counted rows; a piece of the weight; dz of the piece: planes of [.][width] or [.][dz_ld]
  int64_t rows_plane, packed_plane, dz_plane, dz_ld;
  float *part;                                     // dx in parts: [part][slot][width]
  // piece of the vocabulary, and of the launch
  int32_t first, piece, direct, splits, add, parts, wide;
  int32_t tiles_m, tiles_n;
  Divisor by_group, by_n, by_tiles, by_row;
};

// ---- rows that count -------------------------------------------------------------------------------------------------------------------

// One workgroup walks the targets, 8 of them per thread at a time.
template <bool FWD> __global__ void __launch_bounds__(1024) loss_rows_kernel(const LossArgs a) {
  __shared__ int of_wave[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int carry = 0;
  for (int at = 0; at < a.n; at += 8192) {
    int t[8], own = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int row = at + 8 * threadIdx.x + e;
      t[e] = -1;
      if (row < a.n) {
        int b, r;
        div_mod(row, a.xs.by_rows, b, r);
        const int64_t id = a.targets[b * a.targets_sb + r];
        if (id >= 0 && id < a.vocab) t[e] = (int)id;
      }
      own += t[e] >= 0;
    }
    int x = own;
    for (int s = 1; s < 64; s *= 2) {
      const int y = __shfl_up(x, s);
      if (lane >= s) x += y;
    }
    if (lane == 63) of_wave[wave] = x;
    __syncthreads();
    int before = carry + x - own;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before += of_wave[w];
      carry += of_wave[w];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int row = at + 8 * threadIdx.x + e;
      if (row >= a.n) break;
      a.slot_of[row] = t[e] >= 0 ? before : -1;
      if (t[e] >= 0) {
        a.row_of[before] = row;
        a.target_of[before] = t[e];
        ++before;
      } else if (FWD) {
        a.loss[row] = 0.f;
        a.lse[row] = 0.f;
      }
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) *a.count = carry;
}

// Rows as the products read them: bf16, `width` elements from one to the next, zeros behind `hidden`; fp32 ones as three planes.
// ROWS: the counted rows of x; else `piece` rows of the weight from `first` on.
template <typename T, bool WIDE, bool ROWS> __global__ void __launch_bounds__(256) loss_pack_kernel(const LossArgs a) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per_row = a.width / 8;
  const int64_t row64 = id / per_row;
  const int c = (int)(id - row64 * per_row);
  if (row64 >= (ROWS ? *a.count : a.piece)) return;
  const int row = (int)row64;
  if (ROWS && c == 0 && a.dloss) {   // (backward)
    a.of_row[2 * row] = a.lse_in[a.row_of[row]];
    a.of_row[2 * row + 1] = a.dloss[a.row_of[row]];
  }
  const T *from = ROWS ? reinterpret_cast<const T *>(a.x) + a.xs.offset(a.row_of[row])
                       : reinterpret_cast<const T *>(a.weight) + (a.first + row) * a.weight_stride;
  float v[8];
  if constexpr (WIDE) {
#pragma unroll
    for (int i = 0; i < 8; i += Piece<T, true>::N) {
      typename Piece<T, true>::Values p;
      Piece<T, true>::load(from + 8 * c + i, p);
#pragma unroll
      for (int e = 0; e < Piece<T, true>::N; ++e) v[i + e] = p[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 8 * c + e < a.hidden ? (float)from[8 * c + e] : 0.f;
  }
  bf16_t *to = (ROWS ? a.rows : a.packed) + row64 * a.width + 8 * c;
  if constexpr (sizeof(T) == 4) {
    const Planes p = split3(f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]});
#pragma unroll
    for (int i = 0; i < 3; ++i) *reinterpret_cast<bf16x8 *>(to + i * (ROWS ? a.rows_plane : a.packed_plane)) = p.p[i];
  } else {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (bf16_t)v[e];
    *reinterpret_cast<bf16x8 *>(to) = o;
  }
}

// ---- products --------------------------------------------------------------------------------------------------------------------------

// Workgroup -> tile.  The hardware hands workgroups to the 8 XCDs in turn; each takes consecutive tiles, in blocks of four columns of tiles
// walked down the rows, so that the 32 workgroups that an XCD runs side by side share eight row and four column panels in its L2.
S1F_DEV void decode_tile(const LossArgs &a, int tile, int &tm, int &tn) {
  const int tiles = a.tiles_m * a.tiles_n, per = tiles >> 3;
  if (tile < per * 8) tile = (tile & 7) * per + (tile >> 3);
  int group, in;
  div_mod(tile, a.by_group, group, in);               // 4 * tiles_m to a group
  const int left = a.tiles_n - 4 * group;
  if (left >= 4) {
    tm = in >> 2;
    tn = 4 * group + (in & 3);
  } else {
    tm = in / left;
    tn = 4 * group + in % left;
  }
}

S1F_DEV Matrix weight_matrix(const LossArgs &a) {
  return a.direct ? Matrix{reinterpret_cast<const bf16_t *>(a.weight) + a.first * a.weight_stride, a.weight_stride, 0}
                  : Matrix{a.packed, a.width, a.packed_plane};
}

// Scores of a tile of rows and vocabulary: STATS: maximum and sum of exponentials of each row (forward); else dz (backward).
template <typename T, int BM, int BN, int WM, int WN, bool STATS>
__global__ void __launch_bounds__(64 * WM * WN) loss_scores_kernel(const LossArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int PAIRS = sizeof(T) == 4 ? 6 : 1;
  typedef Product<BM, BN, WM, WN, false, false, PAIRS> P;
  const int count = *a.count;
  int tm, tn;
  decode_tile(a, blockIdx.x, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  if (m0 >= count) return;
  f32x4 acc[P::MB][P::NB];
  P::run(acc, Matrix{a.rows, a.width, a.rows_plane}, weight_matrix(a), m0, count, n0, a.piece, a.width, 0,
         (a.width + kDepth - 1) / kDepth * PAIRS, to_lds_addr(smem));
  const int lane = lane_id(), n = lane & 15, j = lane >> 4, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
  // A tile's results cost the vector unit about as long as four stages of products the matrix unit, so nothing is asked per element that can be
  // asked per tile or per 16 rows: whether the vocabulary ends in it, and whether a lane holds its row's target (one tile in hundreds).
  const int col0 = 16 * wn * P::NB + 4 * j;   // the lane's columns of the tile: col0 + 16 * nb + e
  const bool edge = n0 + BN > a.piece;
  int target[P::MB];                          // the lane's element 4 * nb + e that is its row's target, or none
#pragma unroll
  for (int mb = 0; mb < P::MB; ++mb) {
    const int slot = m0 + 16 * (wm * P::MB + mb) + n, t = (slot < count ? a.target_of[slot] : -1) - a.first - n0 - col0;
    target[mb] = t >= 0 && t < 16 * P::NB && (t & 15) < 4 ? (t >> 4) * 4 + (t & 3) : -1;
  }
  if constexpr (STATS) {
    float *red = reinterpret_cast<float *>(smem);     // [WN][BM][maximum, sum]
    if (edge) {
#pragma unroll
      for (int nb = 0; nb < P::NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n0 + col0 + 16 * nb + e >= a.piece) {
#pragma unroll
            for (int mb = 0; mb < P::MB; ++mb) acc[mb][nb][e] = -INFINITY;
          }
    }
#pragma unroll
    for (int mb = 0; mb < P::MB; ++mb) {
      const int in_tile = 16 * (wm * P::MB + mb) + n;
      if (target[mb] >= 0) {
#pragma unroll
        for (int nb = 0; nb < P::NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (target[mb] == 4 * nb + e) a.target_score[m0 + in_tile] = acc[mb][nb][e];
      }
      float most = -INFINITY;
#pragma unroll
      for (int nb = 0; nb < P::NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) most = fmaxf(most, acc[mb][nb][e]);
      most = max_over_rows(most);
      const float from = most == -INFINITY ? 0.f : most * kLog2e;
      float sum = 0.f;
#pragma unroll
      for (int nb = 0; nb < P::NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += exp2_fast(fmaf(acc[mb][nb][e], kLog2e, -from));
      sum = sum_over_rows(sum);
      if (j == 0) {
        red[2 * (wn * BM + in_tile)] = most;
        red[2 * (wn * BM + in_tile) + 1] = sum;
      }
    }
    __syncthreads();
    for (int r = threadIdx.x; r < BM && m0 + r < count; r += P::THREADS) {
      float most = red[2 * r], sum = 0.f;
#pragma unroll
      for (int w = 1; w < WN; ++w) most = fmaxf(most, red[2 * (w * BM + r)]);
      const float from = most == -INFINITY ? 0.f : most * kLog2e;
#pragma unroll
      for (int w = 0; w < WN; ++w) sum += red[2 * (w * BM + r) + 1] * exp2_fast(fmaf(red[2 * (w * BM + r)], kLog2e, -from));
      float *to = a.stats + 2 * ((int64_t)(a.first / BN + tn) * a.n + m0 + r);
      to[0] = most;
      to[1] = sum;
    }
  } else {
    float lse[P::MB], g[P::MB];
#pragma unroll
    for (int mb = 0; mb < P::MB; ++mb) {
      const int slot = m0 + 16 * (wm * P::MB + mb) + n, at = slot < count ? slot : count - 1;
      lse[mb] = a.of_row[2 * at];
      g[mb] = a.of_row[2 * at + 1];
    }
#pragma unroll
    for (int mb = 0; mb < P::MB; ++mb) {
      const int slot = m0 + 16 * (wm * P::MB + mb) + n;
      // exp((z - lse) log2 e) as two roundings: the difference, which is exact or small, first
#pragma unroll
      for (int nb = 0; nb < P::NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mb][nb][e] = exp2_fast((acc[mb][nb][e] - lse[mb]) * kLog2e);
      if (target[mb] >= 0) {
#pragma unroll
        for (int nb = 0; nb < P::NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (target[mb] == 4 * nb + e) acc[mb][nb][e] -= 1.f;
      }
      if (slot >= count) continue;
#pragma unroll
      for (int nb = 0; nb < P::NB; ++nb) {
        const int col = n0 + col0 + 16 * nb;
        f32x4 d = acc[mb][nb] * g[mb];
        if (edge) {
          if (col >= a.dz_ld) continue;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + e >= a.piece) d[e] = 0.f;
        }
        bf16_t *to = a.dz + (int64_t)slot * a.dz_ld + col;
        if constexpr (sizeof(T) == 4) {
          typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
          const Planes q = split3(d, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int i = 0; i < 3; ++i) {
            const u32x4 v = __builtin_bit_cast(u32x4, q.p[i]);
            *reinterpret_cast<u32x2 *>(to + i * a.dz_plane) = u32x2{v[0], v[1]};
          }
        } else {
          store4<bf16_t>(to, d[0], d[1], d[2], d[3]);
        }
      }
    }
  }
}

// The forward's statistics of each row joined: 64 rows per workgroup, its waves a quarter of the vocabulary's tiles each.
__global__ void __launch_bounds__(256) loss_join_kernel(const LossArgs a) {
  __shared__ float red[4][64][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, slot = blockIdx.x * 64 + lane, count = *a.count;
  if ((int)blockIdx.x * 64 >= count) return;
  float most = -INFINITY, sum = 0.f;
  if (slot < count)
    for (int t = a.parts * wave / 4; t < a.parts * (wave + 1) / 4; ++t) {
      const float *s = a.stats + 2 * ((int64_t)t * a.n + slot);
      const float m = fmaxf(most, s[0]), from = m == -INFINITY ? 0.f : m;
      sum = sum * exp2_fast((most - from) * kLog2e) + s[1] * exp2_fast((s[0] - from) * kLog2e);
      most = m;
    }
  red[wave][lane][0] = most;
  red[wave][lane][1] = sum;
  __syncthreads();
  if (wave > 0 || slot >= count) return;
  for (int w = 1; w < 4; ++w) most = fmaxf(most, red[w][lane][0]);
  const float from = most == -INFINITY ? 0.f : most;
  sum = 0.f;
  for (int w = 0; w < 4; ++w) sum += red[w][lane][1] * exp2_fast((red[w][lane][0] - from) * kLog2e);
  const int row = a.row_of[slot];
  const float lse = most + logf(sum);
  a.lse[row] = lse;
  a.loss[row] = lse - a.target_score[slot];
}

// dx = dz W over a piece of the vocabulary, in `splits` parts of it that run side by side.
template <int PAIRS, int BM, int BN, int WM, int WN> __global__ void __launch_bounds__(64 * WM * WN) loss_dx_kernel(const LossArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  typedef Product<BM, BN, WM, WN, false, true, PAIRS> P;
  const int count = *a.count;
  int part, tile, tm, tn;
  div_mod(blockIdx.x, a.by_tiles, part, tile);
  decode_tile(a, tile, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  if (m0 >= count) return;
  const int64_t stages = (int64_t)((a.piece + kDepth - 1) / kDepth) * PAIRS;
  f32x4 acc[P::MB][P::NB];
  P::run(acc, Matrix{a.dz, a.dz_ld, a.dz_plane}, weight_matrix(a), m0, count, n0, a.width, a.piece, (int)(stages * part / a.splits),
         (int)(stages * (part + 1) / a.splits), to_lds_addr(smem));
  const int lane = lane_id(), n = lane & 15, j = lane >> 4, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
#pragma unroll
  for (int mb = 0; mb < P::MB; ++mb) {
    const int slot = m0 + 16 * (wm * P::MB + mb) + n;
    if (slot >= count) continue;
#pragma unroll
    for (int nb = 0; nb < P::NB; ++nb) {
      const int col = n0 + 16 * (wn * P::NB + nb) + 4 * j;
      if (col >= a.width) continue;
      f32x4 *to = reinterpret_cast<f32x4 *>(a.part + ((int64_t)part * a.n + slot) * a.width + col);
      *to = a.add ? *to + acc[mb][nb] : acc[mb][nb];
    }
  }
}

// Parts of dx added up in their order, rounded, and put where the rows of x lie; zeros for rows without a target.
template <typename T, bool WIDE> __global__ void __launch_bounds__(256) loss_dx_join_kernel(const LossArgs a) {
  typedef Piece<T, WIDE> P;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per_row = a.hidden / P::N;
  const int64_t row = id / per_row;
  const int c = (int)(id - row * per_row);
  if (row >= a.n) return;
  const int slot = a.slot_of[row];
  float v[P::N], more[P::N];
#pragma unroll
  for (int e = 0; e < P::N; ++e) v[e] = 0.f;
  if (slot >= 0)
    for (int p = 0; p < a.parts; ++p) {
      load_f32<P::N>(a.part + ((int64_t)p * a.n + slot) * a.width + c * P::N, more);
#pragma unroll
      for (int e = 0; e < P::N; ++e) v[e] += more[e];
    }
  P::store(reinterpret_cast<T *>(a.dx) + a.xs.offset((int)row) + c * P::N, v);
}

// dW of a piece of the vocabulary: added into fp32 accumulators (ADD), or written in bf16.
template <int PAIRS, int BM, int BN, int WM, int WN, bool ADD> __global__ void __launch_bounds__(64 * WM * WN) loss_dw_kernel(const LossArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  typedef Product<BM, BN, WM, WN, true, true, PAIRS> P;
  int tm, tn;
  decode_tile(a, blockIdx.x, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN, count = *a.count;
  f32x4 acc[P::MB][P::NB];
  P::run(acc, Matrix{a.dz, a.dz_ld, a.dz_plane}, Matrix{a.rows, a.width, a.rows_plane}, m0, a.dz_ld, n0, a.width, count, 0,
         (count + kDepth - 1) / kDepth * PAIRS, to_lds_addr(smem));
  const int lane = lane_id(), n = lane & 15, j = lane >> 4, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
#pragma unroll
  for (int mb = 0; mb < P::MB; ++mb) {
    const int v = m0 + 16 * (wm * P::MB + mb) + n;
    if (v >= a.piece) continue;
#pragma unroll
    for (int nb = 0; nb < P::NB; ++nb) {
      const int col = n0 + 16 * (wn * P::NB + nb) + 4 * j;
      const int64_t at = (a.first + v) * a.dweight_stride + col;
      const f32x4 d = acc[mb][nb];
      if constexpr (ADD) {
        float *to = reinterpret_cast<float *>(a.dweight) + at;
        if (a.wide && col + 4 <= a.hidden) {
          *reinterpret_cast<f32x4 *>(to) = *reinterpret_cast<f32x4 *>(to) + d;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + e < a.hidden) to[e] += d[e];
        }
      } else {
        bf16_t *to = reinterpret_cast<bf16_t *>(a.dweight) + at;
        if (a.wide && col + 4 <= a.hidden) {
          store4<bf16_t>(to, d[0], d[1], d[2], d[3]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + e < a.hidden) to[e] = (bf16_t)d[e];
        }
      }
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostLossRows = int64_t(1) << 20, kMostLossVocab = int64_t(1) << 24, kMostWeightStride = int64_t(1) << 22;
constexpr int64_t kMostPacked = int64_t(1) << 28, kMostDz = int64_t(1) << 30;   // bytes of a piece of the weight, of its dz
constexpr int kTileBig = 256, kMostSplits = 16;
int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

struct LossPlan {
  int64_t n, width, planes, piece;
  bool direct;
  int splits;
  int64_t count, row_of, slot_of, target_of, target_score, of_row, stats, rows, packed, dz, part, bytes;   // offsets
};

int check_loss(const s1f_rows *d, int64_t vocab, int64_t weight_stride) {
  const int rc = check_rows(d, true, false);
  if (rc != S1F_OK) return rc;
  if (vocab < 1 || weight_stride < d->hidden) return S1F_EINVAL;
  if (vocab > kMostLossVocab || weight_stride >= kMostWeightStride || d->batch * d->rows > kMostLossRows) return S1F_EUNSUPPORTED;
  return S1F_OK;
}

// Parts into which the products of dx are cut along the vocabulary: the rounds of workgroups that the parts take on 256 compute units,
// in the length of a part.
int splits_for(int64_t tiles, int64_t stages) {
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= kMostSplits && (s == 1 || stages / s >= 8); ++s) {
    const double rounds = (double)((tiles * s + 255) / 256), time = rounds * ((double)stages / s + 8.0);
    if (time < 0.95 * least) {
      least = time;
      best = s;
    }
  }
  return best;
}

LossPlan plan_of(const s1f_rows *d, int64_t vocab, int64_t weight_stride, bool backward) {
  LossPlan p = {};
  p.n = d->batch * d->rows;
  p.width = up_to(d->hidden, 8);
  p.planes = d->dtype == S1F_F32 ? 3 : 1;
  p.direct = d->dtype == S1F_BF16 && d->hidden % 8 == 0 && weight_stride % 8 == 0;
  int64_t piece = vocab;
  if (!p.direct) piece = std::min(piece, kMostPacked / (p.planes * 2 * p.width));
  if (backward) piece = std::min(piece, kMostDz / (p.planes * 2 * p.n));
  p.piece = piece < vocab ? std::max<int64_t>(kTileBig, piece / kTileBig * kTileBig) : vocab;
  int64_t at = 0;
  auto take = [&at](int64_t bytes) { const int64_t was = at; at += up_to(bytes, 256); return was; };
  p.count = take(4);
  p.row_of = take(4 * p.n);
  p.slot_of = take(4 * p.n);
  p.target_of = take(4 * p.n);
  p.rows = take(p.planes * 2 * p.n * p.width);
  if (!p.direct) p.packed = take(p.planes * 2 * p.piece * p.width);
  if (backward) {
    const int64_t pairs = p.planes == 3 ? 6 : 1;
    p.splits = splits_for((p.n + kTileBig - 1) / kTileBig * ((p.width + kTileBig - 1) / kTileBig), (p.piece + kDepth - 1) / kDepth * pairs);
    p.of_row = take(8 * p.n);
    p.dz = take(p.planes * 2 * p.n * up_to(p.piece, 64));
    p.part = take(4 * (int64_t)p.splits * p.n * p.width);
  } else {
    p.target_score = take(4 * p.n);
    p.stats = take(8 * p.n * ((vocab + 63) / 64));
  }
  p.bytes = at;
  return p;
}

// Kernels that use more than 64 KiB of LDS are told so once per device.
template <auto KERNEL> int launch_tiles(int lds, int threads, int64_t grid, LossArgs a, hipStream_t st) {
  static std::atomic<bool> told[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return S1F_EDEVICE;
  const bool known = dev >= 0 && dev < 64;
  if (!known || !told[dev].load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return S1F_EDEVICE;
    if (known) told[dev].store(true, std::memory_order_release);
  }
  if (grid * threads >= (int64_t(1) << 32)) return S1F_EUNSUPPORTED;
  return launch_rows_kernel(KERNEL, grid, threads, a, st, lds);
}
void tiles_of(LossArgs &a, int64_t m, int64_t n, int bm, int bn) {
  a.tiles_m = (int32_t)((m + bm - 1) / bm);
  a.tiles_n = (int32_t)((n + bn - 1) / bn);
  a.by_group = Divisor::of(4 * a.tiles_m);
  a.by_tiles = Divisor::of((int64_t)a.tiles_m * a.tiles_n);
}

template <typename T> int pack(const LossArgs &a, bool rows, bool wide, int64_t most, hipStream_t st) {
  const int64_t grid = (most * (a.width / 8) + 255) / 256;
  if (grid * 256 >= (int64_t(1) << 32)) return S1F_EUNSUPPORTED;
  if (rows) return launch_rows_kernel(wide ? &loss_pack_kernel<T, true, true> : &loss_pack_kernel<T, false, true>, grid, 256, a, st);
  return launch_rows_kernel(wide ? &loss_pack_kernel<T, true, false> : &loss_pack_kernel<T, false, false>, grid, 256, a, st);
}

LossArgs args_of(const s1f_rows *d, const LossPlan &p, const int64_t *targets, int64_t targets_sb, const void *x, const void *weight,
                 int64_t weight_stride, int64_t vocab, void *workspace) {
  LossArgs a = {};
  char *ws = reinterpret_cast<char *>(workspace);
  a.targets = targets; a.targets_sb = targets_sb;
  a.x = x; a.weight = weight; a.weight_stride = weight_stride;
  a.xs = x_rows(d);
  a.n = (int32_t)p.n; a.hidden = d->hidden; a.width = (int32_t)p.width; a.vocab = (int32_t)vocab;
  a.count = reinterpret_cast<int32_t *>(ws + p.count);
  a.row_of = reinterpret_cast<int32_t *>(ws + p.row_of);
  a.slot_of = reinterpret_cast<int32_t *>(ws + p.slot_of);
  a.target_of = reinterpret_cast<int32_t *>(ws + p.target_of);
  a.target_score = reinterpret_cast<float *>(ws + p.target_score);
  a.of_row = reinterpret_cast<float *>(ws + p.of_row);
  a.stats = reinterpret_cast<float *>(ws + p.stats);
  a.rows = reinterpret_cast<bf16_t *>(ws + p.rows);
  a.rows_plane = p.n * p.width;
  a.packed = reinterpret_cast<bf16_t *>(ws + p.packed);
  a.packed_plane = p.piece * p.width;
  a.dz = reinterpret_cast<bf16_t *>(ws + p.dz);
  a.dz_ld = up_to(p.piece, 64);
  a.dz_plane = p.n * a.dz_ld;
  a.part = reinterpret_cast<float *>(ws + p.part);
  a.direct = p.direct;
  a.splits = p.splits;
  return a;
}
bool wide_weight(const s1f_rows *d, int64_t stride) { return d->hidden % 8 == 0 && stride % elements_of_16_bytes(d->dtype) == 0; }
bool wide_x(const s1f_rows *d, const void *p) { return on16(p) && d->hidden % 8 == 0 && wide_rows(d, d->x_stride_b, d->x_stride_s); }

template <typename T> int forward(const s1f_rows *d, LossArgs a, const LossPlan &p, hipStream_t st) {
  int e = launch_rows_kernel(&loss_rows_kernel<true>, 1, 1024, a, st);
  if (e == S1F_OK) e = pack<T>(a, true, wide_x(d, a.x), p.n, st);
  const bool small = p.n <= 128;
  for (int64_t at = 0; at < a.vocab && e == S1F_OK; at += p.piece) {
    a.first = (int32_t)at;
    a.piece = (int32_t)std::min(p.piece, a.vocab - at);
    if (!p.direct) e = pack<T>(a, false, wide_weight(d, a.weight_stride), a.piece, st);
    if (e != S1F_OK) break;
    if (small) {
      typedef Product<64, 128, 1, 4, false, false, 1> P;   // (sizes do not depend on the last)
      tiles_of(a, p.n, a.piece, 64, 128);
      e = launch_tiles<&loss_scores_kernel<T, 64, 128, 1, 4, true>>(P::LDS_BYTES, P::THREADS, (int64_t)a.tiles_m * a.tiles_n, a, st);
    } else {
      typedef Product<256, 256, 2, 4, false, false, 1> P;
      tiles_of(a, p.n, a.piece, 256, 256);
      e = launch_tiles<&loss_scores_kernel<T, 256, 256, 2, 4, true>>(P::LDS_BYTES, P::THREADS, (int64_t)a.tiles_m * a.tiles_n, a, st);
    }
  }
  if (e != S1F_OK) return e;
  a.parts = (int32_t)((a.vocab + (small ? 127 : 255)) / (small ? 128 : 256));
  return launch_rows_kernel(&loss_join_kernel, (p.n + 63) / 64, 256, a, st);
}

template <typename T, bool ADD> int backward(const s1f_rows *d, LossArgs a, const LossPlan &p, hipStream_t st) {
  constexpr int PAIRS = sizeof(T) == 4 ? 6 : 1;
  int e = launch_rows_kernel(&loss_rows_kernel<false>, 1, 1024, a, st);
  if (e == S1F_OK) e = pack<T>(a, true, wide_x(d, a.x), p.n, st);
  for (int64_t at = 0; at < a.vocab && e == S1F_OK; at += p.piece) {
    a.first = (int32_t)at;
    a.piece = (int32_t)std::min(p.piece, a.vocab - at);
    a.add = at > 0;
    if (!p.direct) e = pack<T>(a, false, wide_weight(d, a.weight_stride), a.piece, st);
    if (e != S1F_OK) break;
    {
      typedef Product<256, 256, 2, 4, false, false, 1> P;
      tiles_of(a, p.n, a.piece, 256, 256);
      e = launch_tiles<&loss_scores_kernel<T, 256, 256, 2, 4, false>>(P::LDS_BYTES, P::THREADS, (int64_t)a.tiles_m * a.tiles_n, a, st);
    }
    if (e != S1F_OK) break;
    {
      typedef Product<256, 256, 2, 4, false, true, 1> P;
      tiles_of(a, p.n, a.width, 256, 256);
      e = launch_tiles<&loss_dx_kernel<PAIRS, 256, 256, 2, 4>>(P::LDS_BYTES, P::THREADS, (int64_t)a.tiles_m * a.tiles_n * a.splits, a, st);
    }
    if (e != S1F_OK) break;
    {
      typedef Product<256, 256, 2, 4, true, true, 1> P;
      tiles_of(a, a.piece, a.width, 256, 256);
      a.wide = on16(a.dweight) && a.dweight_stride % 4 == 0;
      e = launch_tiles<&loss_dw_kernel<PAIRS, 256, 256, 2, 4, ADD>>(P::LDS_BYTES, P::THREADS, (int64_t)a.tiles_m * a.tiles_n, a, st);
    }
  }
  if (e != S1F_OK) return e;
  a.parts = a.splits;
  const bool wide = wide_x(d, a.dx);
  const int64_t per_row = wide ? d->hidden / elements_of_16_bytes(d->dtype) : d->hidden, grid = (p.n * per_row + 255) / 256;
  if (grid * 256 >= (int64_t(1) << 32)) return S1F_EUNSUPPORTED;
  return launch_rows_kernel(wide ? &loss_dx_join_kernel<T, true> : &loss_dx_join_kernel<T, false>, grid, 256, a, st);
}

}  // namespace
}  // namespace s1f

using namespace s1f;

extern "C" size_t s1f_token_loss_fwd_workspace_bytes(const s1f_rows *desc, int64_t vocab, int64_t weight_stride) {
  return check_loss(desc, vocab, weight_stride) == S1F_OK ? (size_t)plan_of(desc, vocab, weight_stride, false).bytes : 0;
}
extern "C" size_t s1f_token_loss_bwd_workspace_bytes(const s1f_rows *desc, int64_t vocab, int64_t weight_stride) {
  return check_loss(desc, vocab, weight_stride) == S1F_OK ? (size_t)plan_of(desc, vocab, weight_stride, true).bytes : 0;
}

extern "C" int s1f_token_loss_fwd(const s1f_rows *desc, const void *x, const void *weight, int64_t weight_stride, int64_t vocab,
                                  const int64_t *targets, int64_t targets_stride_b, float *loss, float *lse, void *workspace,
                                  size_t workspace_bytes, void *hip_stream) {
  const int rc = check_loss(desc, vocab, weight_stride);
  if (rc != S1F_OK) return rc;
  if (!x || !weight || !targets || !loss || !lse || !workspace || !on_element(x, desc->dtype) || !on16(weight) || !on16(workspace) ||
      !on4(loss) || !on4(lse) || (reinterpret_cast<uintptr_t>(targets) & 7))
    return S1F_EINVAL;
  const LossPlan p = plan_of(desc, vocab, weight_stride, false);
  if (workspace_bytes < (size_t)p.bytes) return S1F_EINVAL;
  LossArgs a = args_of(desc, p, targets, targets_stride_b, x, weight, weight_stride, vocab, workspace);
  a.loss = loss; a.lse = lse;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  return desc->dtype == S1F_BF16 ? forward<bf16_t>(desc, a, p, st) : forward<float>(desc, a, p, st);
}

extern "C" int s1f_token_loss_bwd(const s1f_rows *desc, const float *dloss, const void *x, const void *weight, int64_t weight_stride,
                                  int64_t vocab, const int64_t *targets, int64_t targets_stride_b, const float *lse, void *dx, void *dweight,
                                  int64_t dweight_stride, int32_t dweight_dtype, void *workspace, size_t workspace_bytes, void *hip_stream) {
  const int rc = check_loss(desc, vocab, weight_stride);
  if (rc != S1F_OK) return rc;
  if (dweight_dtype != S1F_F32 && !(dweight_dtype == S1F_BF16 && desc->dtype == S1F_BF16)) return S1F_EUNSUPPORTED;
  if (!dloss || !x || !weight || !targets || !lse || !dx || !dweight || !workspace || !on_element(x, desc->dtype) || !on_element(dx, desc->dtype) ||
      !on16(weight) || !on16(workspace) || !on_element(dweight, dweight_dtype) || !on4(dloss) || !on4(lse) ||
      (reinterpret_cast<uintptr_t>(targets) & 7) || dweight_stride < desc->hidden)
    return S1F_EINVAL;
  const LossPlan p = plan_of(desc, vocab, weight_stride, true);
  if (workspace_bytes < (size_t)p.bytes) return S1F_EINVAL;
  LossArgs a = args_of(desc, p, targets, targets_stride_b, x, weight, weight_stride, vocab, workspace);
  a.dloss = dloss; a.lse_in = lse; a.dx = dx; a.dweight = dweight; a.dweight_stride = dweight_stride;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  if (desc->dtype == S1F_F32) return backward<float, true>(desc, a, p, st);
  return dweight_dtype == S1F_F32 ? backward<bf16_t, true>(desc, a, p, st) : backward<bf16_t, false>(desc, a, p, st);
}
