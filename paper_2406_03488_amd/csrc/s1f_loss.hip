// Cross entropy of every row of a segment over a large vocabulary, with its gradient: what the last stage of a pipeline does behind its
// last layer.  z = x W^T are the scores of a row, t its target.
//
//   forward    lse = log sum_v exp(z_v),  loss = lse - z_t
//   backward   dz_v = (exp(z_v - lse) - [v = t]) * dloss,  dx = dz W,  dW += dz^T x
//
// Scores never exist in memory as a whole.  The forward's tiles of scores leave a maximum and a sum of exponentials per row; the
// backward computes the scores of a piece of the vocabulary anew, writes that piece's dz in bf16 (rounded once, as the attention kernels round
// their score gradients; by which dx of 1000 x 512 over
// 5000 tokens is 2.3e-3 off relative to its norm, 1.7e-3 of it the rounding of dx itself, and dW in fp32 1.5e-3; fp32 calls: in three bf16 planes that hold it whole), and both products read it.
// Rows without a target take no part: the others are gathered into consecutive rows first, so nothing is computed for them and whatever
// they hold, infinities and NaN included, stays theirs.  The number of rows that count is known on the device only; workgroups
// behind them end at once.
#include "attn_plain.hpp"
#include "product_launch.hpp"

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
  float *sum, *part;                               // dx: [slot][width]; what the parts of a cut tile but the first add: [part - 1][tile][row][column]
  // piece of the vocabulary, and of the launch
  int32_t first, piece, direct, add, parts, wide, row_groups;
  // tiles of the launch: their grid; the first one; whether a workgroup takes a quarter of one
  int32_t tiles_m, tiles_n, tile0, quarters;
  // dx: the tiles from `whole` on, `rest` of them, are cut into `splits` parts along the vocabulary (see DxParts)
  int32_t whole, rest, splits, most_splits;
  // dW: parts that fp32 sums are cut into if all rows count (see sums_of); what all but the first add: [part - 1][tile][row][column]
  int32_t dw_parts;
  float *dw_part;
};

// ---- rows that count -------------------------------------------------------------------------------------------------------------------

// One workgroup walks the targets, 8192 of them at a time: wave w has rows 1024 * e + 64 * w + lane, so that lanes read neighbours and a ballot numbers
// the rows of a wave (8 neighbours to a thread instead, added up over lanes: 10 us for 4099 rows).
template <bool FWD> __global__ void __launch_bounds__(1024) loss_rows_kernel(const LossArgs a) {
  __shared__ int counted[8][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int carry = 0;
  for (int at = 0; at < a.n; at += 8192) {
    int t[8];
    uint64_t has[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int row = at + 1024 * e + threadIdx.x;
      t[e] = -1;
      if (row < a.n) {
        int b, r;
        div_mod(row, a.xs.by_rows, b, r);
        const int64_t id = a.targets[b * a.targets_sb + r];
        if (id >= 0 && id < a.vocab) t[e] = (int)id;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      has[e] = __ballot(t[e] >= 0);
      if (lane == 0) counted[e][wave] = __builtin_popcountll(has[e]);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      int before = carry;
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        const int c = counted[e][w];
        carry += c;
        if (w < wave) before += c;
      }
      const int row = at + 1024 * e + threadIdx.x;
      if (row < a.n) {
        before += __builtin_popcountll(has[e] & ((uint64_t(1) << lane) - 1));
        a.slot_of[row] = t[e] >= 0 ? before : -1;
        if (t[e] >= 0) {
          a.row_of[before] = row;
          a.target_of[before] = t[e];
        } else if (FWD) {
          a.loss[row] = 0.f;
          a.lse[row] = 0.f;
        }
      }
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) *a.count = carry;
}

template <typename T, bool WIDE> S1F_DEV void pack_weight(const LossArgs &a, int64_t id) {
  const int per_row = a.width / 8;
  const int64_t row = id / per_row;
  const int c = (int)(id - row * per_row);
  if (row < a.piece)
    pack_eight<T, WIDE>(reinterpret_cast<const T *>(a.weight) + (a.first + row) * a.weight_stride, a.hidden, c, a.packed + row * a.width + 8 * c, a.packed_plane);
}
// Bound by memory: 4099 rows of 4096 bf16 elements, 67 MB, 14 us.  ROWS: the counted rows of x; else `piece` rows of the weight from `first` on.
template <typename T, bool WIDE, bool ROWS> __global__ void __launch_bounds__(256) loss_pack_kernel(const LossArgs a) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (!ROWS) return pack_weight<T, WIDE>(a, id);
  const int per_row = a.width / 8;
  const int64_t slot = id / per_row;
  const int c = (int)(id - slot * per_row);
  if (slot >= *a.count) return;
  const int row = a.row_of[slot];
  if (c == 0 && a.dloss) {   // (backward)
    a.of_row[2 * slot] = a.lse_in[row];
    a.of_row[2 * slot + 1] = a.dloss[row];
  }
  pack_eight<T, WIDE>(reinterpret_cast<const T *>(a.x) + a.xs.offset(row), a.hidden, c, a.rows + slot * a.width + 8 * c, a.rows_plane);
}

// All of it in one launch, for few rows: workgroups below `row_groups` take 8 rows of x each, for which they count the rows with a target in front of them
// themselves, the others a part of the first piece of the weight.
constexpr int kRowsPerGroup = 8;
template <typename T, bool WIDE_X, bool WIDE_W, bool FWD> __global__ void __launch_bounds__(1024) loss_prepare_kernel(const LossArgs a) {
  if ((int)blockIdx.x >= a.row_groups) return pack_weight<T, WIDE_W>(a, (int64_t)((int)blockIdx.x - a.row_groups) * 1024 + threadIdx.x);
  __shared__ int counted[16], own[kRowsPerGroup], slots[kRowsPerGroup];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = blockIdx.x * kRowsPerGroup;
  auto target = [&](int row) -> int {
    int b, r;
    div_mod(row, a.xs.by_rows, b, r);
    const int64_t id = a.targets[b * a.targets_sb + r];
    return id >= 0 && id < a.vocab ? (int)id : -1;
  };
  int before = 0;
  for (int i = threadIdx.x; i - (int)threadIdx.x < first; i += 1024) before += __builtin_popcountll(__ballot(i < first && target(i < first ? i : 0) >= 0));
  if (lane == 0) counted[wave] = before;
  if (threadIdx.x < kRowsPerGroup) own[threadIdx.x] = first + (int)threadIdx.x < a.n ? target(first + threadIdx.x) : -1;
  __syncthreads();
  before = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) before += counted[w];
  int after = before, at = -1;
#pragma unroll
  for (int r = 0; r < kRowsPerGroup; ++r) {
    if (r == (int)threadIdx.x && own[r] >= 0) at = after;
    after += own[r] >= 0;
  }
  if (threadIdx.x < kRowsPerGroup) slots[threadIdx.x] = at;
  const int row = first + threadIdx.x;
  if (threadIdx.x < kRowsPerGroup && row < a.n) {
    a.slot_of[row] = at;
    if (at >= 0) {
      a.row_of[at] = row;
      a.target_of[at] = own[threadIdx.x];
      if (!FWD) {
        a.of_row[2 * at] = a.lse_in[row];
        a.of_row[2 * at + 1] = a.dloss[row];
      }
    } else if (FWD) {
      a.loss[row] = 0.f;
      a.lse[row] = 0.f;
    }
  }
  if ((int)blockIdx.x == a.row_groups - 1 && threadIdx.x == 0) *a.count = after;
  __syncthreads();
  const int per_row = a.width / 8;
  for (int i = threadIdx.x; i < kRowsPerGroup * per_row; i += 1024) {
    const int r = i / per_row, c = i - r * per_row;
    if (slots[r] < 0) continue;
    pack_eight<T, WIDE_X>(reinterpret_cast<const T *>(a.x) + a.xs.offset(first + r), a.hidden, c, a.rows + (int64_t)slots[r] * a.width + 8 * c, a.rows_plane);
  }
}

// Rows that one fp32 sum of dW runs over, up to half as many again, six products for each.  Error of dW relative to its norm, 64 elements over 300 tokens: of 8192 rows in one sum 1.0e-6,
// of 12288 in one 1.2e-6 and in two 0.7e-6, of 16384 1.4e-6 and 0.8e-6, of 131072 5.0e-6 and 0.5e-6 (the library's product of 32-bit dz: 1.5e-6 to 1.9e-6); the last two calls take
// 850 -> 462 us and 7830 -> 854.  A part but the first costs room for its tiles, written and read once: 8193 rows of 1024 over 32000 tokens in two parts 8.9 ms for 8.6, 16384 of 4096 over
// 20000 36.7 for 37.0.  bf16 sums are six times as short, and their dz is rounded.
constexpr int kSummed = 8192;
__host__ __device__ __forceinline__ int sums_of(int rows) { return rows < kSummed ? 1 : (rows + kSummed / 2) / kSummed; }

// ---- products --------------------------------------------------------------------------------------------------------------------------

// Workgroup -> tile, or quarter of a tile.
S1F_DEV void own_tile(const LossArgs &a, int &tm, int &tn) {
  if (!a.quarters) return decode_tile(a.tiles_m, a.tiles_n, a.tile0 + blockIdx.x, tm, tn);
  decode_tile(a.tiles_m, a.tiles_n, a.tile0 + (blockIdx.x >> 2), tm, tn);
  tm = 2 * tm + ((blockIdx.x >> 1) & 1);
  tn = 2 * tn + (blockIdx.x & 1);
}

S1F_DEV Matrix weight_matrix(const LossArgs &a) {
  return a.direct ? Matrix{reinterpret_cast<const bf16_t *>(a.weight) + a.first * a.weight_stride, a.weight_stride, 0}
                  : Matrix{a.packed, a.width, a.packed_plane};
}

// fp32 scores that the products of planes cannot give: where an operand is not finite, or a score or one of its terms passes the largest float, there is a NaN or an infinity
// among them.  A wave computes the 16 rows' blocks in which that happens again, from the operands in memory, with the fp32 matrix instructions: what fp32 arithmetic gives, in which a score
// of minus infinity has weight zero and leaves its row's others alone.  What is finite pays one instruction per score; one weight of minus infinity in 20011 rows of 1280: loss of 682 rows 234 -> 880 us, an infinity in each of
// 4099 rows of 1024 over 20000 tokens 832 -> 3736.  slot0, col0: of the wave's first block; lanes
// as in the epilogue below.
template <int MB, int NB> S1F_DEV void scores_plain(f32x4 (&acc)[MB][NB], const LossArgs &a, int count, int slot0, int col0) {
  typedef Piece<float, false> P;
  const int lane = lane_id(), n = lane & 15, j = lane >> 4;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) {
    float bad = 0.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) bad = add_if_not_finite(acc[mb][nb], bad);
    if (!any_not_finite(bad)) continue;
    const int slot = slot0 + 16 * mb + n;
    const float *x = reinterpret_cast<const float *>(a.x) + a.xs.offset(a.row_of[slot < count ? slot : count - 1]), *w[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int v = col0 + 16 * nb + n;
      w[nb] = reinterpret_cast<const float *>(a.weight) + (a.first + (v < a.piece ? v : a.piece - 1)) * a.weight_stride;
      acc[mb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // four steps of four at a time, of which lane (n, j) holds elements 4j .. 4j+3: in either operand, so that any order does
#pragma unroll 1
    for (int k0 = 0; k0 < a.hidden; k0 += 16) {
      const int k = k0 + 4 * j;
      const f32x4 fx = P::get(x + k, a.hidden - k);
      f32x4 fw[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) fw[nb] = P::get(w[nb] + k, a.hidden - k);
      bool numbers = false;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mb][nb] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[nb][e], fx[e], acc[mb][nb], 0, 0, 0);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) numbers = numbers || acc[mb][nb][e] == acc[mb][nb][e];
      if (__builtin_amdgcn_ballot_w64(numbers) == 0) break;   // (NaN throughout, and stays so)
    }
  }
}

// Exponentials of scores relative to a maximum.  The difference is taken first: exact or small, then its product with log2 e rounded; and a maximum times log2 e is
// infinite from 2.36e38 on, where masks of the type's lowest value lie.  Where there is no score above -infinity, relative to 0: all of them 0.
S1F_DEV float above(float most) { return most == -INFINITY ? 0.f : most; }
S1F_DEV float exp_of(float x) { return exp2_fast(x * kLog2e); }

// Scores of a tile of rows and vocabulary: STATS: maximum and sum of exponentials of each row (forward); else dz (backward).  Bound by the matrix units, at the
// clock that power leaves them, and by the beginning and end of a tile, about 6 us in which they wait: 4099 rows of 4096 bf16 elements over 50021 tokens 1.30 ms,
// 1.3 PFLOP/s, the library's product alone 1.27; gradient of 5530 rows of 7168 over 100003 tokens 6.3 ms, 1.25 PFLOP/s, the product alone 5.5.
template <typename T, int BM, int BN, int WM, int WN, bool STATS>
__global__ void __launch_bounds__(64 * WM * WN, 2) loss_scores_kernel(const LossArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int PAIRS = sizeof(T) == 4 ? 6 : 1;
  typedef Product<BM, BN, WM, WN, false, false, PAIRS> P;
  const int count = *a.count;
  int tm, tn;
  own_tile(a, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  if (m0 >= count || n0 >= a.piece) return;
  f32x4 acc[P::MB][P::NB];
  const Matrix rows = {a.rows, a.width, a.rows_plane};
  if constexpr (PAIRS == 6 && BM == 64) P::run_planes(acc, rows, weight_matrix(a), m0, count, n0, a.piece, a.width, to_lds_addr(smem));
  else P::run(acc, rows, weight_matrix(a), m0, count, n0, a.piece, a.width, 0, (a.width + kDepth - 1) / kDepth * PAIRS, to_lds_addr(smem));
  const int lane = lane_id(), n = lane & 15, j = lane >> 4, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
  if constexpr (sizeof(T) == 4) scores_plain(acc, a, count, m0 + 16 * wm * P::MB, n0 + 16 * wn * P::NB);
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
      const float from = above(most);
      float sum = 0.f;
#pragma unroll
      for (int nb = 0; nb < P::NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += exp_of(acc[mb][nb][e] - from);
      sum = sum_over_rows(sum);
      if (j == 0) {
        red[2 * (wn * BM + in_tile)] = most;
        red[2 * (wn * BM + in_tile) + 1] = sum;
      }
    }
    __syncthreads();
    // statistics are kept for every 128 columns, whatever tile they come from
    constexpr int PER = BN / 128, WAVES = WN / PER;
    for (int r = threadIdx.x; r < BM * PER; r += P::THREADS) {
      const int row = r % BM, part = r / BM;
      if (m0 + row >= count || n0 + 128 * part >= a.piece) continue;
      const float *in = red + 2 * (part * WAVES * BM + row);
      float most = in[0], sum = 0.f;
#pragma unroll
      for (int w = 1; w < WAVES; ++w) most = fmaxf(most, in[2 * w * BM]);
      const float from = above(most);
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += in[2 * w * BM + 1] * exp_of(in[2 * w * BM] - from);
      float *to = a.stats + 2 * ((int64_t)((a.first + n0) / 128 + part) * a.n + m0 + row);
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
#pragma unroll
      for (int nb = 0; nb < P::NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mb][nb][e] = exp_of(acc[mb][nb][e] - lse[mb]);
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
          const Planes q = split3(d * kUp, f32x4{0.f, 0.f, 0.f, 0.f});
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

// The forward's statistics of each row joined: 16 rows per workgroup, for each of which 64 lanes share the vocabulary's tiles.  Bound by latency: 4 lanes to a
// row took 28 us for 4099 rows and 196 tiles, 16 lanes 15.
__global__ void __launch_bounds__(1024) loss_join_kernel(const LossArgs a) {
  constexpr int SHARES = 64;
  __shared__ float red[SHARES][16][2];
  const int in = threadIdx.x & 15, share = threadIdx.x >> 4, slot = blockIdx.x * 16 + in, count = *a.count;
  if ((int)blockIdx.x * 16 >= count) return;
  float most = -INFINITY, sum = 0.f;
  if (slot < count)
    for (int t = share; t < a.parts; t += SHARES * 4) {   // four at a time, asked for together
      float m[4], x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool is = t + SHARES * u < a.parts;
        const float *s = a.stats + 2 * ((int64_t)(is ? t + SHARES * u : t) * a.n + slot);
        m[u] = s[0];
        x[u] = is ? s[1] : 0.f;
      }
      const float now = fmaxf(fmaxf(most, fmaxf(m[0], m[1])), fmaxf(m[2], m[3])), from = above(now);
      sum *= exp_of(most - from);
#pragma unroll
      for (int u = 0; u < 4; ++u) sum += x[u] * exp_of(m[u] - from);
      most = now;
    }
  red[share][in][0] = most;
  red[share][in][1] = sum;
  for (int half = SHARES / 2; half > 0; half /= 2) {
    __syncthreads();
    if (share < half) {
      const float m = red[share + half][in][0], now = fmaxf(most, m), from = above(now);
      sum = sum * exp_of(most - from) + red[share + half][in][1] * exp_of(m - from);
      most = now;
      red[share][in][0] = most;
      red[share][in][1] = sum;
    }
  }
  if (share > 0 || slot >= count) return;
  const int row = a.row_of[slot];
  const float lse = most + logf(sum);
  a.lse[row] = lse;
  a.loss[row] = lse - a.target_score[slot];
}

// How dx's tiles are cut.  The host plans for all rows; where it cuts every tile and fewer count, the workgroups and the room for parts that the plan has are shared
// out among the tiles that there are (the same in every launch of a call): gradient of half of 1024 rows of 2048 bf16 elements over 32000 tokens 397 -> 366 us, of
// 0.6 * 2048 rows of 2560 over 50021 1176 -> 1096, of 0.7 * 682 rows of 1280 fp32 elements over 20011 587 -> 575.
struct DxParts {
  int tiles_m, whole, rest, splits;
  S1F_DEV DxParts(const LossArgs &a, int count, int tile) {
    tiles_m = a.tiles_m;
    whole = a.whole;
    rest = a.rest;
    splits = a.splits;
    const int there = (count + tile - 1) / tile;
    if (whole == 0 && splits > 1 && there < tiles_m && there > 0) {
      const int planned = rest * (splits - 1);   // parts that there is room for behind every tile's first
      tiles_m = there;
      rest = there * a.tiles_n;
      splits = planned / rest + 1 < a.most_splits ? planned / rest + 1 : a.most_splits;
    }
  }
};

// fp32 dz are split 2^16 times as large as they are, and what comes of them divided: most tokens have next to no probability, and the last plane of a value below 2^-110
// would lie under the smallest bf16 number (see kUp).
template <int PAIRS> constexpr float kOfDz = PAIRS == 6 ? 1.f / kUp : 1.f;

// dx = dz W over a piece of the vocabulary.  Tiles that do not fill a round of workgroups are cut along the vocabulary.  5530 rows of 7168 bf16 elements over
// 100003 tokens: 6.2 ms, 1.28 PFLOP/s, the library's product 7.9.
template <int PAIRS, int BM, int BN, int WM, int WN> __global__ void __launch_bounds__(64 * WM * WN, 2) loss_dx_kernel(const LossArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  typedef Product<BM, BN, WM, WN, false, true, PAIRS> P;
  const int count = *a.count;
  const DxParts cut(a, count, BM);
  int tile = blockIdx.x, part = 0, parts = 1, tm, tn;
  if (tile >= cut.whole) {
    part = (tile - cut.whole) / cut.rest;
    tile -= part * cut.rest;
    parts = cut.splits;
  }
  if (part >= parts) return;
  decode_tile(cut.tiles_m, a.tiles_n, tile, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  if (m0 >= count) return;
  const int64_t stages = (int64_t)((a.piece + kDepth - 1) / kDepth) * PAIRS;
  f32x4 acc[P::MB][P::NB];
  P::run(acc, Matrix{a.dz, a.dz_ld, a.dz_plane}, weight_matrix(a), m0, count, n0, a.width, a.piece, (int)(stages * part / parts),
         (int)(stages * (part + 1) / parts), to_lds_addr(smem));
  const int lane = lane_id(), n = lane & 15, j = lane >> 4, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
  float *to = part == 0 ? a.sum + (int64_t)m0 * a.width + n0 : a.part + ((int64_t)(part - 1) * cut.rest + tile - cut.whole) * (BM * BN);
  const int stride = part == 0 ? a.width : BN;
#pragma unroll
  for (int mb = 0; mb < P::MB; ++mb) {
    const int row = 16 * (wm * P::MB + mb) + n;
    if (m0 + row >= count) continue;
#pragma unroll
    for (int nb = 0; nb < P::NB; ++nb) {
      const int col = 16 * (wn * P::NB + nb) + 4 * j;
      if (n0 + col >= a.width) continue;
      f32x4 *at = reinterpret_cast<f32x4 *>(to + (int64_t)row * stride + col);
      const f32x4 d = acc[mb][nb] * kOfDz<PAIRS>;
      *at = a.add ? *at + d : d;
    }
  }
}

// dx rounded and put where the rows of x lie, parts of cut tiles (of TILE x TILE) added up in their order; zeros for rows without a target.  Bound by memory:
// 6144 rows of 7168 elements, 247 MB, and parts: 57 us.
template <typename T, bool WIDE, int TILE> __global__ void __launch_bounds__(256) loss_dx_join_kernel(const LossArgs a) {
  typedef Piece<T, WIDE> P;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per_row = (a.hidden + P::N - 1) / P::N;
  const int64_t row = id / per_row;
  const int col = (int)(id - row * per_row) * P::N;
  if (row >= a.n) return;
  const int slot = a.slot_of[row];
  float v[P::N], more[P::N];
#pragma unroll
  for (int e = 0; e < P::N; ++e) v[e] = 0.f;
  if (slot >= 0) {
    load_f32<P::N, true>(a.sum + (int64_t)slot * a.width + col, P::N, v);
    if (a.splits > 1) {
      const DxParts cut(a, *a.count, TILE);
      const int tile = encode_tile(cut.tiles_m, a.tiles_n, slot / TILE, col / TILE);
      if (tile >= cut.whole)
        for (int p = 0; p + 1 < cut.splits; ++p) {
          load_f32<P::N, true>(a.part + (((int64_t)p * cut.rest + tile - cut.whole) * TILE + slot % TILE) * TILE + col % TILE, P::N, more);
#pragma unroll
          for (int e = 0; e < P::N; ++e) v[e] += more[e];
        }
    }
  }
  P::store(reinterpret_cast<T *>(a.dx) + a.xs.offset((int)row) + col, a.hidden - col, v);
}

// dW of a piece of the vocabulary: added into fp32 accumulators (ADD), or written in bf16.  No atomics: a workgroup has all rows of its tile, or in fp32, whose six products make a sum
// over as many rows six times as long, those of a part (see kSummed).  5530 rows of 7168 bf16 elements over 100003 tokens: 6.4 ms, 1.24 PFLOP/s, the library's product 6.9.
template <int PAIRS, int BM, int BN, int WM, int WN, bool ADD> __global__ void __launch_bounds__(64 * WM * WN, 2) loss_dw_kernel(const LossArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  typedef Product<BM, BN, WM, WN, true, true, PAIRS> P;
  int tm, tn, part = 0;
  if (PAIRS == 1 || a.dw_parts == 1) {
    own_tile(a, tm, tn);
  } else {
    part = blockIdx.x / (a.tiles_m * a.tiles_n);
    decode_tile(a.tiles_m, a.tiles_n, blockIdx.x - part * (a.tiles_m * a.tiles_n), tm, tn);
  }
  const int m0 = tm * BM, n0 = tn * BN, count = *a.count;
  if (m0 >= a.piece || n0 >= a.width) return;
  int begin = 0, end = (count + kDepth - 1) / kDepth;
  if (PAIRS == 6 && a.dw_parts > 1) {
    const int parts = sums_of(count);
    if (part >= parts) return;
    begin = (int)((int64_t)end * part / parts);
    end = (int)((int64_t)end * (part + 1) / parts);
  }
  f32x4 acc[P::MB][P::NB];
  P::run(acc, Matrix{a.dz, a.dz_ld, a.dz_plane}, Matrix{a.rows, a.width, a.rows_plane}, m0, a.dz_ld, n0, a.width, count, begin * PAIRS, end * PAIRS,
         to_lds_addr(smem));
  const int lane = lane_id(), n = lane & 15, j = lane >> 4, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
  if (PAIRS == 6 && part > 0) {
    float *to = a.dw_part + ((int64_t)(part - 1) * a.tiles_m * a.tiles_n + tm * a.tiles_n + tn) * (BM * BN);
#pragma unroll
    for (int mb = 0; mb < P::MB; ++mb)
#pragma unroll
      for (int nb = 0; nb < P::NB; ++nb)
        *reinterpret_cast<f32x4 *>(to + (16 * (wm * P::MB + mb) + n) * BN + 16 * (wn * P::NB + nb) + 4 * j) = acc[mb][nb] * kOfDz<PAIRS>;
    return;
  }
#pragma unroll
  for (int mb = 0; mb < P::MB; ++mb) {
    const int v = m0 + 16 * (wm * P::MB + mb) + n;
    if (v >= a.piece) continue;
#pragma unroll
    for (int nb = 0; nb < P::NB; ++nb) {
      const int col = n0 + 16 * (wn * P::NB + nb) + 4 * j;
      const int64_t at = (a.first + v) * a.dweight_stride + col;
      const f32x4 d = acc[mb][nb] * kOfDz<PAIRS>;
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

// The parts of dW behind the first (of tiles of TILE x TILE), added up in their order.  Bound by memory.
template <int TILE> __global__ void __launch_bounds__(256) loss_dw_join_kernel(const LossArgs a) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per_row = (a.hidden + 3) / 4;
  const int64_t v = id / per_row;
  const int col = (int)(id - v * per_row) * 4, parts = sums_of(*a.count);
  if (v >= a.piece || parts == 1) return;
  const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
  const float *from = a.dw_part + (v / TILE * a.tiles_n + col / TILE) * (TILE * TILE) + (v % TILE) * TILE + col % TILE;
  f32x4 sum = *reinterpret_cast<const f32x4 *>(from);
  for (int p = 2; p < parts; ++p) sum += *reinterpret_cast<const f32x4 *>(from + (p - 1) * tiles * (TILE * TILE));
  float *to = reinterpret_cast<float *>(a.dweight) + (a.first + v) * a.dweight_stride + col;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (col + e < a.hidden) to[e] += sum[e];
}

// ---- host ------------------------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostLossRows = int64_t(1) << 20, kMostLossVocab = int64_t(1) << 24, kMostWeightStride = int64_t(1) << 22;
constexpr int64_t kMostElements = int64_t(1) << 33;                             // of x: threads of the launch that writes dx
// bytes of a piece of the weight, and of its dz (of more, up to 1.5 GiB, where 2^30 bytes hold less than 256 tokens: fp32 calls of more than 699050 rows)
constexpr int64_t kMostPacked = int64_t(1) << 28, kMostDz = int64_t(1) << 30;

struct LossPlan {
  int64_t n, width, planes, piece;
  bool direct;
  Cut scores, dw;
  DxCut dx;
  int dw_parts;
  int64_t count, row_of, slot_of, target_of, target_score, of_row, stats, rows, packed, dz, sum, part, dw_part, bytes;   // offsets
};

int check_loss(const s1f_rows *d, int64_t vocab, int64_t weight_stride) {
  const int rc = check_rows(d, true, false);
  if (rc != S1F_OK) return rc;
  if (vocab < 1 || weight_stride < d->hidden) return S1F_EINVAL;
  const int64_t n = d->batch * d->rows;
  if (vocab > kMostLossVocab || weight_stride >= kMostWeightStride || n > kMostLossRows || n * d->hidden > kMostElements) return S1F_EUNSUPPORTED;
  return S1F_OK;
}

LossPlan plan_of(const s1f_rows *d, int64_t vocab, int64_t weight_stride, bool backward) {
  LossPlan p = {};
  p.n = d->batch * d->rows;
  p.width = up_to(d->hidden, 8);
  p.planes = d->dtype == S1F_F32 ? 3 : 1;
  p.direct = d->dtype == S1F_BF16 && d->hidden % 8 == 0 && weight_stride % 8 == 0;
  // (of either product over the vocabulary a launch holds fewer than 2^32 threads: up to 512 for 64 x 128 scores, 256 for 128 x 128 of dW)
  int64_t piece = std::min({vocab, (int64_t(1) << 35) / p.n, (int64_t(1) << 36) / p.width});
  if (!p.direct) piece = std::min(piece, kMostPacked / (p.planes * 2 * p.width));
  if (backward) piece = std::min(piece, kMostDz / (p.planes * 2 * p.n));
  // (and never longer than the vocabulary: with enough rows `piece` is below 256, and a vocabulary may lie between)
  p.piece = std::min(vocab, piece < vocab ? std::max<int64_t>(256, piece / 256 * 256) : vocab);
  int64_t at = 0;
  auto take = [&at](int64_t bytes) { const int64_t was = at; at += up_to(bytes, 256); return was; };
  p.count = take(4);
  p.row_of = take(4 * p.n);
  p.slot_of = take(4 * p.n);
  p.target_of = take(4 * p.n);
  p.rows = take(p.planes * 2 * p.n * p.width);
  if (!p.direct) p.packed = take(p.planes * 2 * p.piece * p.width);
  const int64_t pairs = p.planes == 3 ? 6 : 1, stages = (p.width + kDepth - 1) / kDepth * pairs;
  p.scores = cut_for(p.n, p.piece, stages, true);
  if (backward) {
    p.dx = dx_cut_for(p.n, p.width, (p.piece + kDepth - 1) / kDepth * pairs);
    p.dw = cut_for(p.piece, p.width, (p.n + kDepth - 1) / kDepth * pairs, false);
    p.dw_parts = p.planes == 3 ? sums_of((int)p.n) : 1;
    if (p.dw_parts > 1) {   // of whole tiles
      const int64_t big = grid_of(p.piece, p.width, 256, 256), middle = grid_of(p.piece, p.width, 128, 128);
      const double stages = (double)(kSummed / kDepth * pairs);
      p.dw = tiles_us(kBig, big * p.dw_parts, stages) < tiles_us(kMiddle, middle * p.dw_parts, stages) ? Cut{kBig, big} : Cut{kMiddle, 0};
    }
    const int64_t side = p.dx.tile == kBig ? 256 : 128, dw_side = p.dw.tile == kBig ? 256 : 128;
    p.of_row = take(8 * p.n);
    p.dz = take(p.planes * 2 * p.n * up_to(p.piece, 64));
    p.sum = take(4 * p.n * p.width);
    p.part = take(4 * (p.dx.splits - 1) * p.dx.rest * side * side);
    p.dw_part = take(4 * (p.dw_parts - 1) * grid_of(p.piece, p.width, (int)dw_side, (int)dw_side) * dw_side * dw_side);
  } else {
    p.target_score = take(4 * p.n);
    p.stats = take(8 * p.n * ((vocab + 127) / 128));
  }
  p.bytes = at;
  return p;
}

void tiles_of(LossArgs &a, int64_t m, int64_t n, int bm, int bn) {
  a.tiles_m = (int32_t)((m + bm - 1) / bm);
  a.tiles_n = (int32_t)((n + bn - 1) / bn);
}

template <typename T> int pack_weight_piece(const LossArgs &a, bool wide, hipStream_t st) {
  const int64_t grid = ((int64_t)a.piece * (a.width / 8) + 255) / 256;
  return launch_rows_kernel(wide ? &loss_pack_kernel<T, true, false> : &loss_pack_kernel<T, false, false>, grid, 256, a, st);
}
// Counts, numbers and packs the rows, and packs the first piece of the weight unless the products read it as it is.  In one launch, every workgroup of which
// reads the targets of the rows in front of its own, or in two or three: forward of 256 x 256 over 5003 tokens, fp32, 27.0 and 32.6 us, of 1000 x 1024 over 10007,
// bf16, 38.3 and 41.2, of 4099 x 1024 over 20000 176 and 171, of 32768 x 512 over 8000 334 and 304.
constexpr int64_t kMostPrepared = 2048;
template <typename T, bool FWD> int prepare_rows(LossArgs a, bool wide_rows, bool wide_weight, hipStream_t st) {
  if (a.n > kMostPrepared) {
    int e = launch_rows_kernel(&loss_rows_kernel<FWD>, 1, 1024, a, st);
    const int64_t grid = ((int64_t)a.n * (a.width / 8) + 255) / 256;
    if (e == S1F_OK) e = launch_rows_kernel(wide_rows ? &loss_pack_kernel<T, true, true> : &loss_pack_kernel<T, false, true>, grid, 256, a, st);
    if (e == S1F_OK && !a.direct) e = pack_weight_piece<T>(a, wide_weight, st);
    return e;
  }
  a.row_groups = (a.n + kRowsPerGroup - 1) / kRowsPerGroup;
  const int64_t grid = a.row_groups + (a.direct ? 0 : ((int64_t)a.piece * (a.width / 8) + 1023) / 1024);
  if (wide_rows)
    return launch_rows_kernel(wide_weight ? &loss_prepare_kernel<T, true, true, FWD> : &loss_prepare_kernel<T, true, false, FWD>, grid, 1024, a, st);
  return launch_rows_kernel(wide_weight ? &loss_prepare_kernel<T, false, true, FWD> : &loss_prepare_kernel<T, false, false, FWD>, grid, 1024, a, st);
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
  a.sum = reinterpret_cast<float *>(ws + p.sum);
  a.part = reinterpret_cast<float *>(ws + p.part);
  a.dw_part = reinterpret_cast<float *>(ws + p.dw_part);
  a.dw_parts = p.dw_parts;
  a.direct = p.direct;
  a.whole = (int32_t)p.dx.whole;
  a.rest = (int32_t)p.dx.rest;
  a.splits = p.dx.splits;
  a.most_splits = p.dx.most_splits;
  return a;
}
bool wide_weight(const s1f_rows *d, int64_t stride) { return d->hidden % 8 == 0 && stride % elements_of_16_bytes(d->dtype) == 0; }
bool wide_x(const s1f_rows *d, const void *p) { return on16(p) && d->hidden % 8 == 0 && wide_rows(d, d->x_stride_b, d->x_stride_s); }

// Launches `kernel`, made for the tile size that it is given, over the tiles of a product [m, n] as `cut` says.  KERNELS<tile>: the kernel, its LDS and threads.
template <template <Tile> class KERNELS> int launch_cut(const Cut &cut, int64_t m, int64_t n, LossArgs a, hipStream_t st) {
  auto go = [&](auto kernels, int64_t grid) {
    typedef decltype(kernels) K;
    return launch_tiles<K::kernel>(K::LDS_BYTES, K::P::THREADS, grid, a, st);
  };
  if (cut.tile == kMiddle) {
    tiles_of(a, m, n, 128, 128);
    return go(KERNELS<kMiddle>{}, (int64_t)a.tiles_m * a.tiles_n);
  }
  if (cut.tile == kLow) {
    tiles_of(a, m, n, 64, 128);
    return go(KERNELS<kLow>{}, (int64_t)a.tiles_m * a.tiles_n);
  }
  tiles_of(a, m, n, 256, 256);
  const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n, whole = std::min(cut.whole, tiles);   // (the last piece may have fewer)
  const int e = go(KERNELS<kBig>{}, whole);
  if (e != S1F_OK || whole == tiles) return e;
  a.tile0 = (int32_t)whole;
  a.quarters = 1;
  return go(KERNELS<kMiddle>{}, 4 * (tiles - whole));
}
// (sizes of a product do not depend on its number of planes)
template <typename T, bool STATS> struct Scores {
  template <Tile TILE> struct Of : TileShape<TILE> {
    typedef TileShape<TILE> S;
    static constexpr int WM = sizeof(T) == 4 && TILE == kLow ? 2 : S::WM;   // (one workgroup to a unit)
    typedef Product<S::BM, S::BN, WM, S::WN, false, false, 1> P;
    static constexpr int LDS_BYTES = sizeof(T) == 4 && TILE == kLow ? P::PLANES_LDS_BYTES : P::LDS_BYTES;
    static constexpr auto kernel = &loss_scores_kernel<T, S::BM, S::BN, WM, S::WN, STATS>;
  };
};
template <int PAIRS, bool ADD> struct Dw {
  template <Tile TILE> struct Of : TileShape<TILE == kLow ? kMiddle : TILE> {
    typedef TileShape<TILE == kLow ? kMiddle : TILE> S;
    typedef Product<S::BM, S::BN, S::WM, S::WN, true, true, 1> P;
    static constexpr int LDS_BYTES = P::LDS_BYTES;
    static constexpr auto kernel = &loss_dw_kernel<PAIRS, S::BM, S::BN, S::WM, S::WN, ADD>;
  };
};
template <int PAIRS, Tile TILE> int launch_dx(const LossPlan &p, LossArgs a, hipStream_t st) {
  typedef TileShape<TILE> S;
  typedef Product<S::BM, S::BN, S::WM, S::WN, false, true, 1> P;
  tiles_of(a, p.n, a.width, S::BM, S::BN);
  return launch_tiles<&loss_dx_kernel<PAIRS, S::BM, S::BN, S::WM, S::WN>>(P::LDS_BYTES, P::THREADS, a.whole + (int64_t)a.rest * a.splits, a, st);
}

// dW in parts, and their join.
template <Tile TILE> int launch_dw_parts(const LossPlan &p, LossArgs a, hipStream_t st) {
  typedef typename Dw<6, true>::template Of<TILE> K;
  constexpr int SIDE = TILE == kBig ? 256 : 128;
  tiles_of(a, a.piece, a.width, SIDE, SIDE);
  const int e = launch_tiles<K::kernel>(K::LDS_BYTES, K::P::THREADS, (int64_t)a.tiles_m * a.tiles_n * p.dw_parts, a, st);
  if (e != S1F_OK) return e;
  return launch_rows_kernel(&loss_dw_join_kernel<SIDE>, ((int64_t)a.piece * ((a.hidden + 3) / 4) + 255) / 256, 256, a, st);
}

template <typename T> int forward(const s1f_rows *d, LossArgs a, const LossPlan &p, hipStream_t st) {
  const bool wide_w = wide_weight(d, a.weight_stride);
  a.piece = (int32_t)p.piece;
  int e = prepare_rows<T, true>(a, wide_x(d, a.x), wide_w, st);
  for (int64_t at = 0; at < a.vocab && e == S1F_OK; at += p.piece) {
    a.first = (int32_t)at;
    a.piece = (int32_t)std::min(p.piece, a.vocab - at);
    if (!p.direct && at > 0) e = pack_weight_piece<T>(a, wide_w, st);
    if (e == S1F_OK) e = launch_cut<Scores<T, true>::template Of>(p.scores, p.n, a.piece, a, st);
  }
  if (e != S1F_OK) return e;
  a.parts = (a.vocab + 127) / 128;
  return launch_rows_kernel(&loss_join_kernel, (p.n + 15) / 16, 1024, a, st);
}

template <typename T, bool ADD> int backward(const s1f_rows *d, LossArgs a, const LossPlan &p, hipStream_t st) {
  constexpr int PAIRS = sizeof(T) == 4 ? 6 : 1;
  const bool wide_w = wide_weight(d, a.weight_stride);
  a.piece = (int32_t)p.piece;
  int e = prepare_rows<T, false>(a, wide_x(d, a.x), wide_w, st);
  a.wide = on16(a.dweight) && a.dweight_stride % 4 == 0;
  for (int64_t at = 0; at < a.vocab && e == S1F_OK; at += p.piece) {
    a.first = (int32_t)at;
    a.piece = (int32_t)std::min(p.piece, a.vocab - at);
    a.add = at > 0;
    if (!p.direct && at > 0) e = pack_weight_piece<T>(a, wide_w, st);
    if (e == S1F_OK) e = launch_cut<Scores<T, false>::template Of>(p.scores, p.n, a.piece, a, st);
    if (e == S1F_OK) e = p.dx.tile == kBig ? launch_dx<PAIRS, kBig>(p, a, st) : launch_dx<PAIRS, kMiddle>(p, a, st);
    if (e != S1F_OK) continue;
    if (PAIRS == 1 || p.dw_parts == 1) e = launch_cut<Dw<PAIRS, ADD>::template Of>(p.dw, a.piece, a.width, a, st);
    else e = p.dw.tile == kBig ? launch_dw_parts<kBig>(p, a, st) : launch_dw_parts<kMiddle>(p, a, st);
  }
  if (e != S1F_OK) return e;
  const int side = p.dx.tile == kBig ? 256 : 128;
  tiles_of(a, p.n, a.width, side, side);
  const bool wide = wide_x(d, a.dx);
  const int64_t per_row = (d->hidden + elements_of_16_bytes(d->dtype) - 1) / elements_of_16_bytes(d->dtype), grid = (p.n * per_row + 255) / 256;
  if (side == 256) return launch_rows_kernel(wide ? &loss_dx_join_kernel<T, true, 256> : &loss_dx_join_kernel<T, false, 256>, grid, 256, a, st);
  return launch_rows_kernel(wide ? &loss_dx_join_kernel<T, true, 128> : &loss_dx_join_kernel<T, false, 128>, grid, 256, a, st);
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
