// The gated feed-forward block of a layer on the rows of a segment, and its gradient.  n rows of `hidden` elements, `inner` between the projections.
//
//   forward    [g | u] = x W_in^T,  h = act(g) * u,  y = h W_out^T
//   backward   dh = dy W_out,  dg = dh * u * act'(g),  du = dh * act(g);  dx = [dg | du] W_in,  dW_in += [dg | du]^T x,  dW_out += dy^T h
//
// Bound by the matrix units, at the clock that power leaves them: 6 n hidden inner operations and 12.  Forward of 4099 x 4096 x 11008 bf16 921 to 955 us, 1.16 to 1.2 PFLOP/s (a library product of
// 16384^3 of random operands: 1.33); gradient of 4897 x 7168 x 19200 6.55 to 6.64 ms, 1.22 to 1.23.  Few rows: the weights.  Nothing of it is a pass over memory of its own: a tile of x W_in^T holds the same columns of
// both halves, in the same lanes, so that h is what its results leave in memory (and g and u, rounded, if the caller keeps them); dh stays in registers, and the tile
// that computes it reads g and u and leaves dg, du and h.  h, dg and du are bf16 in memory, rounded once, as the attention kernels round their probabilities and score
// gradients; fp32 calls: three bf16 planes that hold them whole, and fp32 operands are split into such planes first.
#include <cmath>

#include "product_launch.hpp"

namespace s1f {
namespace {

// One operand laid out anew: rows of `hidden` elements as rows of `width` bf16 ones, zeros behind the end; fp32 ones as three planes.
struct PackJob {
  const void *from;
  RowsOf rows;
  int64_t n, plane;
  bf16_t *to;
  int32_t hidden, width, wide, up;   // up: times kUp
  int64_t first_block;
};
constexpr int kMostJobs = 4;

struct FfnArgs {
  Matrix a, b;                    // operands of the launch
  int32_t m, n, k;                // rows and columns of its product, and its contraction
  int32_t m_limit, n_limit;       // what there is of either operand (columns: whole pieces of 8)
  int32_t inner, act;
  // where results go: h and [dg | du], planes of [.][ld]; rows of the call's tensors
  bf16_t *h, *dz;
  int64_t h_ld, h_plane, dz_ld, dz_plane;
  void *gate_up;                  // [.][2 * inner]
  void *out;
  RowsOf out_rows;
  float scale;                    // of the results (see kUp)
  // tiles (see Cuts)
  int32_t tiles_m, tiles_n, tile0, quarters, whole, rest, splits;
  float *part;                    // [part][tile][row][column]
  PackJob jobs[kMostJobs];
  int32_t n_jobs;
  // the weight as it lies in memory, for kernels that read it there; few rows: the rows, too (h: rows of inner_width elements)
  const void *weight, *rows;
  int64_t weight_stride;
  RowsOf rows_at;
};

// ---- operands --------------------------------------------------------------------------------------------------------------------------

// Bound by memory.  All of a call's operands in one launch.
template <typename T> __global__ void __launch_bounds__(256) ffn_pack_kernel(const FfnArgs a) {
  int j = 0;
  while (j + 1 < a.n_jobs && (int64_t)blockIdx.x >= a.jobs[j + 1].first_block) ++j;
  const PackJob &p = a.jobs[j];
  const int64_t id = ((int64_t)blockIdx.x - p.first_block) * 256 + threadIdx.x;
  const int per_row = p.width / 8;
  const int64_t row = id / per_row;
  const int c = (int)(id - row * per_row);
  if (row >= p.n) return;
  const T *from = reinterpret_cast<const T *>(p.from) + p.rows.offset((int)row);
  bf16_t *to = p.to + row * p.width + 8 * c;
  if (sizeof(T) == 4 && p.up) {
    f32x4 v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = Piece<float, false>::get(reinterpret_cast<const float *>(from) + 8 * c + 4 * i, p.hidden - 8 * c - 4 * i) * kUp;
    const Planes q = split3(v[0], v[1]);
#pragma unroll
    for (int i = 0; i < 3; ++i) *reinterpret_cast<bf16x8 *>(to + i * p.plane) = q.p[i];
  } else if (p.wide) {
    pack_eight<T, true>(from, p.hidden, c, to, p.plane);
  } else {
    pack_eight<T, false>(from, p.hidden, c, to, p.plane);
  }
}

// ---- activations -----------------------------------------------------------------------------------------------------------------------

// 1 / (1 + exp(-x)).  bf16 calls: the unit's exponential and reciprocal, 2^-22 off or so.
template <typename T> S1F_DEV float sigmoid(float x) {
  if constexpr (sizeof(T) == 4) return 1.f / (1.f + expf(-x));
  else return __builtin_amdgcn_rcpf(1.f + exp2_fast(x * -kLog2e));
}
// act(g), and act'(g).  The tanh form is g * sigmoid(g (c0 + c1 g^2)), (1 + tanh(t)) / 2 being the sigmoid of 2t, which keeps its digits where 1 + tanh would lose them, as erfc does
// where 1 + erf would (erfcf and expf per element: forward of 4099 x 4096 x 11008 bf16 964 us where the others take 928 to 933, gradient 1936 and 1874 to 1887).
template <typename T, int ACT> struct Activation {
  static constexpr float c0 = 1.5957691216f, c1 = c0 * 0.044715f;
  // (past 2^60 squares are left where they are, and no sigmoid changes any more)
  S1F_DEV static float square(float g) { return fminf(g * g, 0x1p120f); }
  S1F_DEV static float value(float g) {
    if constexpr (ACT == S1F_GELU) return g * (0.5f * erfcf(g * -0.70710678f));
    else return g * sigmoid<T>(ACT == S1F_SILU ? g : g * fmaf(c1, square(g), c0));
  }
  S1F_DEV static void both(float g, float &a, float &slope) {
    if constexpr (ACT == S1F_GELU) {
      const float p = 0.5f * erfcf(g * -0.70710678f);
      a = g * p;
      slope = fmaf(g * 0.39894228f, expf(-0.5f * g * g), p);
    } else {
      const float q = square(g), s = sigmoid<T>(ACT == S1F_SILU ? g : g * fmaf(c1, q, c0));
      a = g * s;
      const float rest = a * (1.f - s);   // (0 far out, whatever the square is)
      slope = ACT == S1F_SILU ? rest + s : fmaf(rest, fmaf(3.f * c1, q, c0), s);
    }
  }
};
// f(Int<act>{})
template <typename F> S1F_DEV void with_activation(int act, F &&f) {
  if (act == S1F_SILU) f(Int<S1F_SILU>{});
  else if (act == S1F_GELU) f(Int<S1F_GELU>{});
  else f(Int<S1F_GELU_TANH>{});
}

// ---- products --------------------------------------------------------------------------------------------------------------------------

// Workgroup -> tile, or quarter of a tile; and which part of its contraction.
S1F_DEV void ffn_tile(const FfnArgs &a, int &tm, int &tn, int &tile, int &part, int &parts) {
  part = 0;
  parts = 1;
  if (a.quarters) {
    tile = a.tile0 + (blockIdx.x >> 2);
    decode_tile(a.tiles_m, a.tiles_n, tile, tm, tn);
    tm = 2 * tm + ((blockIdx.x >> 1) & 1);
    tn = 2 * tn + (blockIdx.x & 1);
    return;
  }
  tile = blockIdx.x;
  if (tile >= a.whole) {
    part = (tile - a.whole) / a.rest;
    tile -= part * a.rest;
    parts = a.splits;
  }
  decode_tile(a.tiles_m, a.tiles_n, tile, tm, tn);
}

// fp32 products in low tiles read the weight as it lies in memory, and have all planes of two stages in LDS: one workgroup to a unit.  So do middle tiles with planes that were laid out, and have
// five thirds of a stage there.
template <int PAIRS, int BM> constexpr bool kAllPlanes = PAIRS == 6 && BM == 64;
template <int PAIRS, int BM> constexpr bool kTogether = PAIRS == 6 && BM == 128;
template <typename P, int PAIRS, int BM>
S1F_DEV void ffn_product(f32x4 (&acc)[P::MB][P::NB], const FfnArgs &a, int m0, int n0, int part, int parts, lds_addr lds, int64_t b_apart = 0) {
  const int64_t stages = (a.k + kDepth - 1) / kDepth * (kAllPlanes<PAIRS, BM> || kTogether<PAIRS, BM> ? 1 : PAIRS);
  const int begin = (int)(stages * part / parts), end = (int)(stages * (part + 1) / parts);
  if constexpr (kAllPlanes<PAIRS, BM>)
    P::run_raw(acc, a.a, reinterpret_cast<const float *>(a.weight), a.weight_stride, m0, a.m_limit, n0, a.n, a.k, begin, end, lds, b_apart);
  else if constexpr (kTogether<PAIRS, BM>) P::run_together(acc, a.a, a.b, m0, a.m_limit, n0, a.n_limit, a.k, begin, end, lds, b_apart);
  else P::run(acc, a.a, a.b, m0, a.m_limit, n0, a.n_limit, a.k, begin, end, lds, b_apart);
}

// Eight values of a row of a bf16 matrix, or of its three planes, on any element; the first `there` of them.
template <int PAIRS> S1F_DEV void put8(bf16_t *to, int64_t plane, const float (&v)[8], int there) {
  typedef Piece<bf16_t, false> P;
  if constexpr (PAIRS == 6) {
    const Planes q = split3(f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]});
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if (there >= 8) {
        *reinterpret_cast<P::Loose *>(to + i * plane) = q.p[i];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < there) to[i * plane + e] = q.p[i][e];
      }
    }
  } else {
    P::store(to, there, v);
  }
}
template <typename T> S1F_DEV void get8(const T *from, int there, float (&v)[8]) {
  typedef Piece<T, false> P;
#pragma unroll
  for (int i = 0; i < 8; i += P::N) {
    typename P::Values p;
    P::load(from + i, there - i, p);
#pragma unroll
    for (int e = 0; e < P::N; ++e) v[i + e] = p[e];
  }
}
template <typename T> S1F_DEV void set8(T *to, int there, const float (&v)[8]) {
  typedef Piece<T, false> P;
#pragma unroll
  for (int i = 0; i < 8; i += P::N) {
    typename P::Values p;
#pragma unroll
    for (int e = 0; e < P::N; ++e) p[e] = v[i + e];
    P::store(to + i, there - i, p);
  }
}
// Four values of a row, on any element; the first `there` of them.  (One access also where rows do not start on 16 bytes: gradient of 100 x 1280 x 3413 fp32 196 -> 182 us, of 1000 x 1001 x 2003 bf16 88 -> 80.)
template <typename T> using LooseFour = T __attribute__((ext_vector_type(4), aligned(sizeof(T))));
template <typename T> S1F_DEV void put_values(T *to, f32x4 v, int there) {
  if (there >= 4) {
    *reinterpret_cast<LooseFour<T> *>(to) = __builtin_convertvector(v, LooseFour<T>);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < there) to[e] = (T)v[e];
  }
}
template <typename T> S1F_DEV f32x4 get_values(const T *from, int there) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (there >= 4) {
    v = __builtin_convertvector(*reinterpret_cast<const LooseFour<T> *>(from), f32x4);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < there) v[e] = (float)from[e];
  }
  return v;
}

// What a wave's lanes have written to LDS before is what they read there behind it.
S1F_DEV void between_lanes() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// A wave's results on their way to memory: through LDS of its own, 16 * GM rows at a time, from where a lane takes eight neighbours of a row, so that memory sees whole lines and a
// lane's work on them is a loop.  (From the registers of the matrix instructions, four elements to a lane: the loop over 32 blocks of a 256 x 256 tile was
// not unrolled, its accumulators went to memory, and dh of 4897 x 7168 x 19200 took 19.7 ms.)
template <typename P> struct Staged {
  static constexpr int GM = P::MB < 4 ? P::MB : 4, LD = 16 * P::NB + 4, BYTES = 16 * GM * LD * 4;
  float *base;
  S1F_DEV explicit Staged(char *smem) : base(reinterpret_cast<float *>(smem + (threadIdx.x >> 6) * BYTES)) {}
  S1F_DEV void put(const f32x4 (&acc)[P::MB][P::NB], int mb0) {
    const int lane = lane_id(), n = lane & 15, j = lane >> 4;
#pragma unroll
    for (int mb = 0; mb < GM; ++mb)
#pragma unroll
      for (int nb = 0; nb < P::NB; ++nb) *reinterpret_cast<f32x4 *>(base + (16 * mb + n) * LD + 16 * nb + 4 * j) = acc[mb0 + mb][nb];
    between_lanes();
  }
  S1F_DEV void get(int row, int col, float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4 *>(base + row * LD + col + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = x[e];
    }
  }
};

// Zeros behind the end of a row.
S1F_DEV void clear_behind(float (&v)[8], int there) {
  if (there >= 8) return;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e >= there) v[e] = 0.f;
}

// h = act(g) * u of a tile of BM rows and BN / 2 columns.  4099 x 4096 x 2 x 11008 bf16, g and u kept: 637 us, 1.16 PFLOP/s, matrix units 62 % busy; 17 rows of tiles for 16.01, and 6 rounds of them
// for 5.7, are 8 % of it.  m0: first row of the wave's blocks, n0: its first column.
template <typename T, int ACT, typename P> S1F_DEV void up_results(const f32x4 (&acc)[P::MB][P::NB], const FfnArgs &a, int m0, int n0, char *smem) {
  constexpr int PAIRS = sizeof(T) == 4 ? 6 : 1, LANES = P::NB, ROWS = 64 / LANES;   // lanes to a row of 8 NB columns
  Staged<P> staged(smem);
  // blocks of g and u take turns
  const int lane = lane_id(), at = 8 * (lane % LANES), from = (at >> 4 << 5) + (at & 15), col = n0 + at, there = a.inner - col;
#pragma unroll
  for (int mb = 0; mb < P::MB; mb += Staged<P>::GM) {
    staged.put(acc, mb);
#pragma unroll 1
    for (int r = lane / LANES; r < 16 * Staged<P>::GM; r += ROWS) {
      const int row = m0 + 16 * mb + r;
      float g[8], u[8], h[8];
      staged.get(r, from, g);
      staged.get(r, from + 16, u);
      if (row >= a.m || col >= a.h_ld) continue;
      if (a.gate_up) {
        T *to = reinterpret_cast<T *>(a.gate_up) + (int64_t)row * 2 * a.inner + col;
        set8<T>(to, there, g);
        set8<T>(to + a.inner, there, u);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = Activation<T, ACT>::value(g[e]) * u[e];
      clear_behind(h, there);
      put8<PAIRS>(a.h + (int64_t)row * a.h_ld + col, a.h_plane, h, 8);
    }
    between_lanes();
  }
}
template <typename T, int BM, int BN, int WM, int WN> __global__ void __launch_bounds__(64 * WM * WN, 2) ffn_up_kernel(const FfnArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int PAIRS = sizeof(T) == 4 ? 6 : 1;
  typedef Product<BM, BN, WM, WN, false, false, PAIRS> P;
  int tm, tn, tile, part, parts;
  ffn_tile(a, tm, tn, tile, part, parts);
  const int m0 = tm * BM, n0 = tn * (BN / 2);
  if (m0 >= a.m || n0 >= a.n) return;
  f32x4 acc[P::MB][P::NB];
  ffn_product<P, PAIRS, BM>(acc, a, m0, n0, 0, 1, to_lds_addr(smem), a.inner);
  const int wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
  with_activation(a.act, [&](auto act) { up_results<T, decltype(act)::value, P>(acc, a, m0 + 16 * P::MB * wm, n0 + 8 * P::NB * wn, smem); });
}

// dh = dy W_out of a tile, and of it [dg | du] and h.  4897 x 7168 x 19200 bf16: 1.14 ms, 1.18 PFLOP/s.  (g and u asked for four rows ahead instead of two: no faster.)
template <typename T, int ACT, typename P> S1F_DEV void dh_results(const f32x4 (&acc)[P::MB][P::NB], const FfnArgs &a, int m0, int n0, char *smem) {
  constexpr int PAIRS = sizeof(T) == 4 ? 6 : 1, LANES = 2 * P::NB, ROWS = 64 / LANES;
  Staged<P> staged(smem);
  const int lane = lane_id(), at = 8 * (lane % LANES), col = n0 + at, there = a.inner - col;
#pragma unroll
  for (int mb = 0; mb < P::MB; mb += Staged<P>::GM) {
    staged.put(acc, mb);
#pragma unroll 2
    for (int r = lane / LANES; r < 16 * Staged<P>::GM; r += ROWS) {
      const int row = m0 + 16 * mb + r;
      if (row >= a.m || col >= a.h_ld) continue;
      const T *from = reinterpret_cast<const T *>(a.gate_up) + (int64_t)row * 2 * a.inner + col;
      float d[8], g[8], u[8], h[8];
      get8<T>(from, there, g);
      get8<T>(from + a.inner, there, u);
      staged.get(r, at, d);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float act, slope;
        Activation<T, ACT>::both(g[e], act, slope);
        h[e] = act * u[e];
        g[e] = d[e] * u[e] * slope;
        u[e] = d[e] * act;
      }
      clear_behind(h, there);
      put8<PAIRS>(a.h + (int64_t)row * a.h_ld + col, a.h_plane, h, 8);
      bf16_t *to = a.dz + (int64_t)row * a.dz_ld + col;
      put8<PAIRS>(to, a.dz_plane, g, there);
      put8<PAIRS>(to + a.inner, a.dz_plane, u, there);
      if (there <= 8)   // zeros behind the end of du, where the products read whole pieces of 8
        for (int c = 2 * a.inner; c < a.dz_ld; ++c)
#pragma unroll
          for (int i = 0; i < (PAIRS == 6 ? 3 : 1); ++i) a.dz[(int64_t)row * a.dz_ld + c + i * a.dz_plane] = (bf16_t)0.f;
    }
    between_lanes();
  }
}
template <typename T, int BM, int BN, int WM, int WN> __global__ void __launch_bounds__(64 * WM * WN, 2) ffn_dh_kernel(const FfnArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int PAIRS = sizeof(T) == 4 ? 6 : 1;
  typedef Product<BM, BN, WM, WN, false, true, PAIRS> P;
  int tm, tn, tile, part, parts;
  ffn_tile(a, tm, tn, tile, part, parts);
  const int m0 = tm * BM, n0 = tn * BN;
  if (m0 >= a.m || n0 >= a.n) return;
  f32x4 acc[P::MB][P::NB];
  ffn_product<P, PAIRS, BM>(acc, a, m0, n0, 0, 1, to_lds_addr(smem));
  const int wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
  with_activation(a.act, [&](auto act) { dh_results<T, decltype(act)::value, P>(acc, a, m0 + 16 * P::MB * wm, n0 + 16 * P::NB * wn, smem); });
}

enum Result { kStoreBf16, kStoreF32, kAddF32 };
template <Result R> S1F_DEV void put_result(const FfnArgs &a, int row, int col, f32x4 v) {
  const int64_t at = a.out_rows.offset(row) + col;
  const int there = a.n - col;
  if constexpr (R == kStoreBf16) {
    put_values<bf16_t>(reinterpret_cast<bf16_t *>(a.out) + at, v, there);
  } else {
    float *to = reinterpret_cast<float *>(a.out) + at;
    if constexpr (R == kAddF32) v += get_values<float>(to, there);
    put_values<float>(to, v, there);
  }
}

// y, dx, dW_in and dW_out.  4897 x 7168 x 19200 bf16: dx 2.06 ms, 1.31 PFLOP/s, dW_out 1.05, 1.29, dW_in 2.15, 1.26 (added into fp32 accumulators, both: 0.37 ms more); fp32, 682 x 1280 x 3413: dx 82 us, dW_in 90, dW_out 48.  The tiles from `whole` on are cut along the contraction: their parts are added up by the join.
template <int PAIRS, int BM, int BN, int WM, int WN, bool TRA, bool TRB, Result R> __global__ void __launch_bounds__(64 * WM * WN, 2) ffn_product_kernel(const FfnArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  typedef Product<BM, BN, WM, WN, TRA, TRB, PAIRS> P;
  int tm, tn, tile, part, parts;
  ffn_tile(a, tm, tn, tile, part, parts);
  const int m0 = tm * BM, n0 = tn * BN;
  if (m0 >= a.m || n0 >= a.n) return;
  f32x4 acc[P::MB][P::NB];
  ffn_product<P, PAIRS, BM>(acc, a, m0, n0, part, parts, to_lds_addr(smem));
  const int lane = lane_id(), n = lane & 15, j = lane >> 4, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
  float *to = a.part + ((int64_t)part * a.rest + tile - a.whole) * (BM * BN);
#pragma unroll
  for (int mb = 0; mb < P::MB; ++mb) {
    const int row = 16 * (wm * P::MB + mb) + n;
    if (m0 + row >= a.m) continue;
#pragma unroll
    for (int nb = 0; nb < P::NB; ++nb) {
      const int col = 16 * (wn * P::NB + nb) + 4 * j;
      if (n0 + col >= a.n) continue;
      const f32x4 v = acc[mb][nb] * a.scale;
      if (parts > 1) *reinterpret_cast<f32x4 *>(to + row * BN + col) = v;
      else put_result<R>(a, m0 + row, n0 + col, v);
    }
  }
}

// The parts of cut tiles of BM x BN added up in their order.  Bound by memory.
template <int BM, int BN, Result R> __global__ void __launch_bounds__(256) ffn_join_kernel(const FfnArgs a) {
  constexpr int PER = BM * BN / 1024;   // workgroups to a tile
  const int in = blockIdx.x / PER, at = (blockIdx.x % PER) * 1024 + threadIdx.x * 4, row = at / BN, col = at % BN;
  int tm, tn;
  decode_tile(a.tiles_m, a.tiles_n, a.whole + in, tm, tn);
  if (tm * BM + row >= a.m || tn * BN + col >= a.n) return;
  const float *from = a.part + (int64_t)in * (BM * BN) + at;
  f32x4 v = *reinterpret_cast<const f32x4 *>(from);
#pragma unroll 4
  for (int p = 1; p < a.splits; ++p) v += *reinterpret_cast<const f32x4 *>(from + (int64_t)p * a.rest * (BM * BN));
  put_result<R>(a, tm * BM + row, tn * BN + col, v);
}

// ---- few rows --------------------------------------------------------------------------------------------------------------------------

// Products of few rows are bound by reading the weights, once.  A workgroup has 16 columns (of gate and up both, or of y), whose rows of the weight its waves read in parts along the
// contraction, straight into the registers of the matrix instructions: each lane 16 bytes of its row at a time, several stages of 64 ahead, no LDS, nothing laid out anew (fp32 is split on
// the way), any strides.  The waves' sums meet in LDS.  16 x 4096 x 11008 bf16: 180 MB of W_in in 36 us, 5.0 TB/s, 90 MB of W_out in 22, 4.0; the rows, which every workgroup reads, cost 12 of both
// (one row: 52 us in all).  Two blocks of columns to a workgroup share them, but leave fewer loads in flight: 65 -> 74.
template <typename T, int BLOCKS> struct Ahead {   // elements of a stage of one operand: 16 rows a block, lane (n, j) has 8j .. 8j+7 of either half of row n
  typedef Piece<T, false> P;
  static constexpr int PER = 8 / P::N;
  typename P::Raw raw[BLOCKS][2][PER];
  // k: the lane's first element
  template <bool WHOLE> S1F_DEV void load(const T *const (&row)[BLOCKS], int64_t k, int64_t end) {
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int64_t at = k + 32 * h + P::N * i;
          if constexpr (WHOLE) raw[b][h][i] = *reinterpret_cast<const typename P::Loose *>(row[b] + at);
          else raw[b][h][i] = P::get(row[b] + at, at < end ? (int)(end - at) : 0);
        }
  }
  S1F_DEV auto operand(int b, int h) const {
    if constexpr (sizeof(T) == 4) return split3(raw[b][h][0], raw[b][h][1]);
    else return raw[b][h][0];
  }
};
template <typename T, int MB, int NB, int WAVES, int DEPTH, bool UP> __global__ void __launch_bounds__(64 * WAVES) ffn_few_kernel(const FfnArgs a) {
  __shared__ __attribute__((aligned(16))) f32x4 sums[WAVES][MB * NB][64];
  const int lane = lane_id(), n = lane & 15, j = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col0 = blockIdx.x * (UP ? 8 * NB : 16 * NB);   // (UP: blocks of gate and up take turns)
  const T *rows[MB], *weight[NB];
#pragma unroll
  for (int b = 0; b < MB; ++b) rows[b] = reinterpret_cast<const T *>(a.rows) + a.rows_at.offset(16 * b + n < a.m ? 16 * b + n : a.m - 1);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int c = col0 + 16 * (UP ? b / 2 : b) + n, known = c < a.n ? c : a.n - 1;
    weight[b] = reinterpret_cast<const T *>(a.weight) + (int64_t)(known + (UP && b % 2 ? a.inner : 0)) * a.weight_stride;
  }
  f32x4 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int whole = a.k / kDepth, begin = whole * wave / WAVES, end = whole * (wave + 1) / WAVES;
  Ahead<T, MB> x[DEPTH];
  Ahead<T, NB> w[DEPTH];
  auto product = [&](const Ahead<T, MB> &xs, const Ahead<T, NB> &ws) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      decltype(xs.operand(0, 0)) fx[MB], fw[NB];
#pragma unroll
      for (int i = 0; i < MB; ++i) fx[i] = xs.operand(i, h);
#pragma unroll
      for (int b = 0; b < NB; ++b) fw[b] = ws.operand(b, h);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[i][b] = mma16(fw[b], fx[i], acc[i][b]);
    }
  };
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (begin + d < end) {
      w[d].template load<true>(weight, (int64_t)(begin + d) * kDepth + 8 * j, 0);
      x[d].template load<true>(rows, (int64_t)(begin + d) * kDepth + 8 * j, 0);
    }
#pragma unroll 1
  for (int t = begin; t < end; t += DEPTH)
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      if (t + d >= end) break;
      product(x[d], w[d]);
      if (t + d + DEPTH < end) {
        w[d].template load<true>(weight, (int64_t)(t + d + DEPTH) * kDepth + 8 * j, 0);
        x[d].template load<true>(rows, (int64_t)(t + d + DEPTH) * kDepth + 8 * j, 0);
      }
    }
  if (wave == WAVES - 1 && whole * kDepth < a.k) {
    w[0].template load<false>(weight, (int64_t)whole * kDepth + 8 * j, a.k);
    x[0].template load<false>(rows, (int64_t)whole * kDepth + 8 * j, a.k);
    product(x[0], w[0]);
  }
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) sums[wave][i * NB + b][lane] = acc[i][b];
  __syncthreads();
  auto sum = [&](int block) {
    f32x4 v = sums[0][block][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += sums[w][block][lane];
    return v;
  };
  // a wave takes a block of 16 x 16, or of gate and up
#pragma unroll
  for (int i = 0; i < (UP ? MB * NB / 2 : MB * NB); ++i) {
    if (i % WAVES != wave) continue;
    constexpr int COLS = UP ? NB / 2 : NB;
    const int row = 16 * (i / COLS) + n, col = col0 + 16 * (i % COLS) + 4 * j, there = a.n - col;
    if (row >= a.m) continue;
    if constexpr (UP) {
      const f32x4 g = sum(2 * i), u = sum(2 * i + 1);
      T *h = reinterpret_cast<T *>(a.h) + (int64_t)row * a.h_ld + col, *kept = reinterpret_cast<T *>(a.gate_up) + (int64_t)row * 2 * a.inner + col;
      with_activation(a.act, [&](auto act) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < there) h[e] = (T)(Activation<T, decltype(act)::value>::value(g[e]) * u[e]);
      });
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (a.gate_up && e < there) {
          kept[e] = (T)g[e];
          kept[a.inner + e] = (T)u[e];
        }
    } else {
      put_result<sizeof(T) == 4 ? kStoreF32 : kStoreBf16>(a, row, col, sum(i));
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostInner = int64_t(1) << 17, kMostStride = int64_t(1) << 22, kMostApart = int64_t(1) << 29, kMostElements = int64_t(1) << 33;
constexpr int64_t kMostFfnRows = int64_t(1) << 20;

// How the tiles of a product are taken: big ones up to `whole` and the rest in quarters (Cut); or those from `whole` on in parts along the contraction.
struct Cuts {
  Tile tile;
  int64_t whole, rest;
  int splits;
  bool quarters;
};
constexpr int tile_m(Tile t) { return t == kBig ? 256 : t == kMiddle ? 128 : 64; }
constexpr int tile_n(Tile t) { return t == kBig ? 256 : 128; }
// Predicted microseconds of `tiles` tiles of so many stages: as tiles_us has them, but that few rounds of smaller tiles count whole, too (540 tiles of 128 x 128 and 66 stages: 130 us, 512 of them
// 65), and that smaller tiles of fp32 work on all planes of a stage at once and have a unit to themselves (low ones 1.6 us for the six products of a stage, 1.9 where an operand lies by columns; middle
// ones 2.5, a single round up to 3.1: priced so, a gradient of 2048 x 1024 x 2816 takes big tiles and 473 us instead of 458).  fp32 dh, us, middle and low: 682 x 3413 of 1280 74 and 120; 256 x 11008 of 4096 211 and 253, with planes to be laid
// out first; 1500 x 5632 of 2048 280 and 311 (big 307).
// Smaller bf16 tiles alone on a unit wait longer for operands that come from memory than the loss's do: priced like those, 1000 rows of 2048 x 5632 took 123 us forward in 256 low tiles of 88 stages instead of
// 101 in middle ones cut in two, the gradient 219 instead of 203, 512 of 4096 x 11008 183 instead of 173, the gradient of 2048 of 1024 x 2816 143 instead of 132.
enum Operand { kBf16, kPlanes, kPlanesByColumns };
double round_us(Tile tile, int64_t tiles, double stages, Operand operand) {
  if (tile == kLow && operand != kBf16) return (double)((tiles + kUnits - 1) / kUnits) * (5.5 + (operand == kPlanes ? 0.265 : 0.32) * stages);
  if (tile == kMiddle && operand != kBf16) return (double)((tiles + kUnits - 1) / kUnits) * (6.0 + 0.42 * stages);
  if (tile != kBig && tiles <= kUnits) return tile == kMiddle ? 5.0 + 0.61 * stages : 4.5 + 0.50 * stages;
  if (tile == kBig || tiles > 6 * kUnits) return tiles_us(tile, tiles, stages);
  const int64_t rounds = tiles / (2 * kUnits), rest = tiles - rounds * 2 * kUnits;
  return (rounds ? (double)rounds * tiles_us(tile, 2 * kUnits, stages) / 1.25 : 0.0) + (rest ? tiles_us(tile, rest, stages) : 0.0);
}
// low: whether there are kernels for low tiles; split: whether a sum may be cut along its contraction; laid_out: microseconds for a weight's planes, which low tiles do without
Cuts cuts_for(int64_t m, int64_t n, int64_t stages, Operand operand, bool low, bool split, double laid_out = 0.0) {
  Cuts best = {};
  double best_us = 1e30;
  auto offer = [&](const Cuts &c, double us) {
    if (c.tile != kLow) us += laid_out;
    if (us < 0.98 * best_us) {
      best_us = us;
      best = c;
    }
  };
  for (Tile tile : {kBig, kMiddle, kLow}) {
    if (tile == kLow && !low) continue;
    auto time = [&](int64_t tiles, double of) { return tiles ? round_us(tile, tiles, of, operand) : 0.0; };
    const int64_t tiles = grid_of(m, n, tile_m(tile), tile_n(tile)), round = tile == kBig || operand != kBf16 ? kUnits : 2 * kUnits, full = tiles / round * round;
    offer(Cuts{tile, tiles, 0, 1, false}, time(tiles, (double)stages));
    if (tile == kBig && full > 0 && full < tiles)
      offer(Cuts{tile, full, tiles - full, 1, true}, time(full, (double)stages) + 3.0 + round_us(kMiddle, 4 * (tiles - full), (double)stages, operand));
    if (!split) continue;
    for (const int64_t whole : {full, int64_t(0)}) {
      const int64_t rest = tiles - whole;
      if (rest == 0 || (whole == 0 && tile == kBig && full > 0)) continue;
      for (int splits = 2; splits <= 32 && stages / splits >= 4 && rest * splits <= 4 * kUnits; ++splits)
        offer(Cuts{tile, whole, rest, splits, false}, time(whole, (double)stages) + time(rest * splits, (double)stages / splits) + 3.0 +
                                                          (double)splits * rest * tile_m(tile) * tile_n(tile) * 8 / 4e6);
      if (full == 0) break;
    }
  }
  return best;
}
int64_t part_bytes(const Cuts &c) { return c.splits > 1 ? 4 * c.splits * c.rest * tile_m(c.tile) * tile_n(c.tile) : 0; }

struct FfnPlan {
  int64_t n, planes, width, inner_width, dz_ld, turns, per_turn;   // dW's rows are taken per_turn at a time
  int64_t y_terms, dx_terms;      // of the sums that make y and dx, likewise
  bool direct_in, direct_out;     // weights as they are
  bool few;
  Cuts up, down, dh, dx, dw_in, dw_out;
  int64_t x, dy, w_in, w_out, h, dz, part, bytes;   // offsets
};

int check_ffn(const s1f_rows *d, int64_t inner, int64_t in_stride, int64_t out_stride) {
  const int rc = check_rows(d, true, true);
  if (rc != S1F_OK) return rc;
  if (inner < 1 || in_stride < d->hidden || (d->hidden > 1 && out_stride < inner)) return S1F_EINVAL;
  const int64_t n = d->batch * d->rows;
  if (inner > kMostInner || in_stride >= kMostStride || out_stride >= kMostStride || inner * in_stride > kMostApart || n > kMostFfnRows || n * d->hidden > kMostElements ||
      n * 2 * inner > kMostElements)
    return S1F_EUNSUPPORTED;
  return S1F_OK;
}

// Terms that one fp32 sum runs over, up to half as many again, six products for each: longer sums would be off by more than fp32 products are (the token
// loss's weight gradient, of 64 elements over 300 tokens: 8192 rows 1.0e-6 of the norm, 16384 1.4e-6, 131072 5.0e-6; dx of 2048 x 2048 x 131072 6.0e-6, a library product 4.4e-6).  More rows of a weight's gradient take turns, and
// so does what lies between the projections for y and dx where tiles are not cut as short anyway: each turn adds to what the one before it has left.  (Sums over hidden end in an activation: one of 16384 2.1e-6, a library product 2.3e-6.)
constexpr int64_t kSummed = 8192;
int64_t turns_of(int64_t n, int64_t planes) { return planes == 1 || n < kSummed + kSummed / 2 ? 1 : (n + kSummed / 2) / kSummed; }

// Forwards that the kernel of few rows takes: up to 16 rows, and up to 64 where the call is small.  It reads the rows once for every 16 columns, where a tile has 64 at a time; a tile waits for
// its beginning and end.  us, few and tiles: 4096 x 11008, bf16 1 row 52 and 82, 16 65 and 83, 32 84 and 84, 64 128 and 89; fp32 1 row 113 and 157, 16 128 and 161, 32 165 and 161, 64 253 and 175;
// bf16 32 x 1024 x 2816 16 and 19, 64 24 and 20, 64 x 256 x 688 11.3 and 12.9; fp32 32 x 1024 x 2816 31 and 41, 64 x 512 x 1376 27 and 31, 64 x 2048 x 5632 106 and 82.
bool few_rows(int64_t n, int64_t hidden, int64_t inner) {
  return n <= 16 || (n <= 64 && n * hidden * inner <= int64_t(1) << 27);
}

FfnPlan plan_of(const s1f_rows *d, int64_t inner, int64_t in_stride, int64_t out_stride, bool backward) {
  FfnPlan p = {};
  const int64_t h = d->hidden;
  p.n = d->batch * d->rows;
  p.planes = d->dtype == S1F_F32 ? 3 : 1;
  p.width = up_to(h, 8);
  p.inner_width = up_to(inner, 8);
  p.dz_ld = up_to(2 * inner, 8);
  p.direct_in = d->dtype == S1F_BF16 && h % 8 == 0 && in_stride % 8 == 0;
  p.direct_out = d->dtype == S1F_BF16 && inner % 8 == 0 && out_stride % 8 == 0;
  int64_t at = 0;
  auto take = [&at](int64_t bytes) { const int64_t was = at; at += up_to(bytes, 256); return was; };
  p.few = !backward && few_rows(p.n, h, inner);
  if (p.few) {
    p.h = take(p.planes * 2 * p.n * p.inner_width);
    p.bytes = at;
    return p;
  }
  const bool f32 = p.planes == 3;
  const int64_t pairs = f32 ? 6 : 1;
  auto stages = [&](int64_t k) { return (k + kDepth - 1) / kDepth * pairs; };
  const Operand rows = f32 ? kPlanes : kBf16, columns = f32 ? kPlanesByColumns : kBf16;
  // planes of a weight: 4 bytes read and 6 written, and a share of a launch
  auto laid_out = [&](int64_t elements) { return f32 ? 3.0 + (double)elements * 10 / 4.4e6 : 0.0; };
  // cuts of a product whose sums are not ended by an activation, and how many of its terms a turn takes
  auto in_turns = [&](Cuts &c, int64_t n, int64_t terms, Operand operand, double laid) {
    for (int64_t turns = 1;;) {
      const int64_t per = turns == 1 ? terms : up_to((terms + turns - 1) / turns, kDepth);
      c = cuts_for(p.n, n, stages(per), operand, true, true, laid / (double)turns);
      const int64_t needed = turns_of(c.whole > 0 || c.splits == 1 ? per : (per + c.splits - 1) / c.splits, p.planes);
      if (needed == 1) return per;
      turns = std::max(turns + 1, turns * needed);
    }
  };
  int64_t part = 0;
  if (!backward) {
    // (tiles of [g | u]: as many columns of either)
    p.up = cuts_for(p.n, 2 * up_to(inner, 16), stages(h), rows, true, false, laid_out(2 * inner * h));
    p.y_terms = in_turns(p.down, h, inner, rows, laid_out(inner * h));
    part = part_bytes(p.down);
    p.direct_in |= f32 && p.up.tile == kLow;
    p.direct_out |= f32 && p.down.tile == kLow;
  } else {
    p.turns = turns_of(p.n, p.planes);
    p.per_turn = up_to((p.n + p.turns - 1) / p.turns, kDepth);
    p.dh = cuts_for(p.n, inner, stages(h), columns, true, false, laid_out(inner * h));
    p.dx_terms = in_turns(p.dx, h, 2 * inner, columns, laid_out(2 * inner * h));
    p.dw_in = cuts_for(2 * inner, h, stages(p.per_turn), columns, false, true);
    p.dw_out = cuts_for(h, inner, stages(p.per_turn), columns, false, true);
    for (const Cuts &c : {p.dx, p.dw_in, p.dw_out}) part = std::max(part, part_bytes(c));
    p.direct_in |= f32 && p.dx.tile == kLow;
    p.direct_out |= f32 && p.dh.tile == kLow;
  }
  p.x = take(p.planes * 2 * p.n * p.width);
  if (!p.direct_in) p.w_in = take(p.planes * 2 * 2 * inner * p.width);
  if (!p.direct_out) p.w_out = take(p.planes * 2 * h * p.inner_width);
  p.h = take(p.planes * 2 * p.n * p.inner_width);
  if (backward) {
    p.dy = take(p.planes * 2 * p.n * p.width);
    p.dz = take(p.planes * 2 * p.n * p.dz_ld);
  }
  p.part = take(part);
  p.bytes = at;
  return p;
}

// Launches a product of `m` x `n` as `cuts` says.  KERNELS<tile>: the kernel, its LDS and threads, and the join of its parts.
template <template <Tile> class KERNELS> int launch_product(const Cuts &cuts, FfnArgs a, int64_t columns, hipStream_t st) {
  auto go = [&](auto kernels, int64_t grid) {
    typedef decltype(kernels) K;
    return launch_tiles<K::kernel>(K::LDS_BYTES, K::P::THREADS, grid, a, st);
  };
  auto tiles = [&](Tile t) {
    a.tiles_m = (int32_t)((a.m + tile_m(t) - 1) / tile_m(t));
    a.tiles_n = (int32_t)((columns + tile_n(t) - 1) / tile_n(t));
    a.whole = (int32_t)cuts.whole;
    a.rest = (int32_t)std::max<int64_t>(cuts.rest, 1);
    a.splits = cuts.splits;
  };
  const int64_t grid = cuts.whole + (cuts.quarters ? 0 : cuts.rest * cuts.splits);
  tiles(cuts.tile);
  int e = S1F_OK;
  if (cuts.tile == kBig) {
    if (grid > 0) e = go(KERNELS<kBig>{}, grid);
    if (e != S1F_OK) return e;
    if (cuts.quarters) {
      a.tile0 = (int32_t)cuts.whole;
      a.quarters = 1;
      return go(KERNELS<kMiddle>{}, 4 * cuts.rest);
    }
  } else {
    e = cuts.tile == kMiddle ? go(KERNELS<kMiddle>{}, grid) : go(KERNELS<kLow>{}, grid);
  }
  if (e != S1F_OK || cuts.splits == 1) return e;
  const int64_t joins = cuts.rest * (tile_m(cuts.tile) * tile_n(cuts.tile) / 1024);
  return launch_rows_kernel(cuts.tile == kBig ? KERNELS<kBig>::join : cuts.tile == kMiddle ? KERNELS<kMiddle>::join : KERNELS<kLow>::join, joins, 256, a, st);
}
template <typename T, Tile TILE, bool TRA, bool TRB> struct FfnShape : TileShape<TILE> {
  typedef TileShape<TILE> S;
  static constexpr bool ALL = kAllPlanes<sizeof(T) == 4 ? 6 : 1, S::BM>, TOGETHER = kTogether<sizeof(T) == 4 ? 6 : 1, S::BM>;
  static constexpr int WM = ALL ? 2 : S::WM, WN = TOGETHER ? 4 : S::WN;   // (one workgroup to a unit)
  typedef Product<S::BM, S::BN, WM, WN, TRA, TRB, 1> P;
  static constexpr int LDS_BYTES = ALL ? P::PLANES_LDS_BYTES : TOGETHER ? P::TOGETHER_LDS_BYTES : P::LDS_BYTES;
  static_assert(Staged<P>::BYTES * P::NW <= LDS_BYTES, "results pass through the operands' places");
  static constexpr void (*join)(FfnArgs) = nullptr;
};
template <typename T> struct Up {
  template <Tile TILE> struct Of : FfnShape<T, TILE, false, false> {
    typedef FfnShape<T, TILE, false, false> S;
    static constexpr auto kernel = &ffn_up_kernel<T, S::BM, S::BN, S::WM, S::WN>;
  };
};
template <typename T> struct Dh {
  template <Tile TILE> struct Of : FfnShape<T, TILE, false, true> {
    typedef FfnShape<T, TILE, false, true> S;
    static constexpr auto kernel = &ffn_dh_kernel<T, S::BM, S::BN, S::WM, S::WN>;
  };
};
template <typename T, bool TRA, bool TRB, Result R> struct Of3 {
  template <Tile TILE> struct Of : FfnShape<T, TRA && TILE == kLow ? kMiddle : TILE, TRA, TRB> {
    typedef FfnShape<T, TRA && TILE == kLow ? kMiddle : TILE, TRA, TRB> S;
    static constexpr auto kernel = &ffn_product_kernel<sizeof(T) == 4 ? 6 : 1, S::BM, S::BN, S::WM, S::WN, TRA, TRB, R>;
    static constexpr void (*join)(FfnArgs) = &ffn_join_kernel<S::BM, S::BN, R>;
  };
};

// An operand of the call: as it is, or laid out anew by the launch that is collected in `a`.
struct Operands {
  FfnArgs &a;
  const s1f_rows *d;
  int64_t planes, blocks = 0;
  Matrix add(const void *from, RowsOf rows, int64_t n, int64_t hidden, int64_t width, bool as_it_is, int64_t ld, bool wide, bool up, char *room) {
    if (as_it_is) return Matrix{reinterpret_cast<const bf16_t *>(from), ld, 0};
    PackJob &j = a.jobs[a.n_jobs++];
    j = PackJob{from, rows, n, n * width, reinterpret_cast<bf16_t *>(room), (int32_t)hidden, (int32_t)width, wide, up, blocks};
    blocks += (n * (width / 8) + 255) / 256;
    return Matrix{j.to, width, j.plane};
  }
  // x or dy
  Matrix rows(const void *from, int64_t sb, int64_t ss, bool up, int64_t width, char *room) {
    const int64_t n = d->batch * d->rows;
    const int64_t ld = d->rows > 1 ? ss : sb;   // (one row to a batch entry: its rows are the batch's)
    const bool even = d->batch == 1 || d->rows == 1 || sb == d->rows * ss, wide = on16(from) && d->hidden % 8 == 0 && wide_rows(d, sb, ss);
    const bool as_it_is = d->dtype == S1F_BF16 && wide && even && ld < kMostStride;
    return add(from, RowsOf{sb, ss, Divisor::of(d->rows)}, n, d->hidden, width, as_it_is, n == 1 ? d->hidden : ld, wide, up, room);
  }
  Matrix weight(const void *from, int64_t n, int64_t hidden, int64_t stride, int64_t width, bool direct, char *room) {
    const bool wide = hidden % 8 == 0 && stride % elements_of_16_bytes(d->dtype) == 0;
    return add(from, RowsOf{0, stride, Divisor::of(n)}, n, hidden, width, direct, stride, wide, false, room);
  }
  int pack(hipStream_t st) {
    if (a.n_jobs == 0) return S1F_OK;
    return launch_rows_kernel(d->dtype == S1F_F32 ? &ffn_pack_kernel<float> : &ffn_pack_kernel<bf16_t>, blocks, 256, a, st);
  }
};

void set_weight(FfnArgs &a, const void *weight, int64_t stride) {
  a.weight = weight; a.weight_stride = stride;
}
void set_product(FfnArgs &a, const Matrix &ma, const Matrix &mb, int64_t m, int64_t m_limit, int64_t n, int64_t n_limit, int64_t k) {
  a.a = ma; a.b = mb;
  a.m = (int32_t)m; a.m_limit = (int32_t)m_limit; a.n = (int32_t)n; a.n_limit = (int32_t)n_limit; a.k = (int32_t)k;
}
void set_out(FfnArgs &a, void *out, RowsOf rows, float scale) {
  a.out = out; a.out_rows = rows; a.scale = scale;
}

FfnArgs args_of(const FfnPlan &p, int64_t inner, int32_t act, const void *gate_up, char *ws) {
  FfnArgs a = {};
  a.inner = (int32_t)inner; a.act = act;
  a.h = reinterpret_cast<bf16_t *>(ws + p.h);
  a.h_ld = p.inner_width; a.h_plane = p.n * p.inner_width;
  a.dz = reinterpret_cast<bf16_t *>(ws + p.dz);
  a.dz_ld = p.dz_ld; a.dz_plane = p.n * p.dz_ld;
  a.gate_up = const_cast<void *>(gate_up);
  a.part = reinterpret_cast<float *>(ws + p.part);
  return a;
}

template <typename T, int MB, int NB, int WAVES, int DEPTH, bool UP> int launch_few(const FfnArgs &a, hipStream_t st) {
  constexpr int COLS = UP ? 8 * NB : 16 * NB;
  const int64_t grid = (a.n + COLS - 1) / COLS;
  return launch_rows_kernel(&ffn_few_kernel<T, MB, NB, WAVES, DEPTH, UP>, grid, 64 * WAVES, a, st);
}
template <typename T>
int forward_few(const s1f_rows *d, FfnArgs a, const void *x, const void *w_in, int64_t in_stride, const void *w_out, int64_t out_stride, void *y, hipStream_t st) {
  constexpr bool F32 = sizeof(T) == 4;
  const int64_t n = d->batch * d->rows;
  a.m = (int32_t)n; a.n = a.inner; a.k = d->hidden;
  a.rows = x; a.rows_at = x_rows(d);
  a.weight = w_in; a.weight_stride = in_stride;
  int e = n <= 16 ? launch_few<T, 1, 2, 4, F32 ? 2 : 4, true>(a, st) : n <= 32 ? launch_few<T, 2, 2, 4, F32 ? 1 : 3, true>(a, st)
                                                                             : launch_few<T, 4, 2, 8, F32 ? 1 : 2, true>(a, st);
  if (e != S1F_OK) return e;
  a.n = d->hidden; a.k = a.inner;
  a.rows = a.h; a.rows_at = RowsOf{0, a.h_ld, Divisor::of(n)};
  a.weight = w_out; a.weight_stride = out_stride;
  set_out(a, y, y_rows(d), 1.f);
  return n <= 16 ? launch_few<T, 1, 1, 8, F32 ? 2 : 8, false>(a, st) : n <= 32 ? launch_few<T, 2, 1, F32 ? 8 : 16, F32 ? 2 : 4, false>(a, st)
                                                                               : launch_few<T, 4, 1, F32 ? 8 : 16, F32 ? 1 : 2, false>(a, st);
}

// What a turn behind the first does with its sums (bf16 has no such turns).
template <typename T> constexpr Result kNext = sizeof(T) == 4 ? kAddF32 : kStoreBf16;
template <typename T>
int forward(const s1f_rows *d, const FfnPlan &p, const void *x, const void *w_in, int64_t in_stride, const void *w_out, int64_t out_stride, int64_t inner, int32_t act,
            void *y, void *gate_up, char *ws, hipStream_t st) {
  constexpr Result R = sizeof(T) == 4 ? kStoreF32 : kStoreBf16;
  FfnArgs a = args_of(p, inner, act, gate_up, ws);
  if (p.few) return forward_few<T>(d, a, x, w_in, in_stride, w_out, out_stride, y, st);
  Operands ops{a, d, p.planes};
  const Matrix mx = ops.rows(x, d->x_stride_b, d->x_stride_s, false, p.width, ws + p.x);
  const Matrix mi = ops.weight(w_in, 2 * inner, d->hidden, in_stride, p.width, p.direct_in, ws + p.w_in);
  const Matrix mo = ops.weight(w_out, d->hidden, inner, out_stride, p.inner_width, p.direct_out, ws + p.w_out);
  int e = ops.pack(st);
  if (e != S1F_OK) return e;
  set_product(a, mx, mi, p.n, p.n, inner, inner, d->hidden);
  set_weight(a, w_in, in_stride);
  e = launch_product<Up<T>::template Of>(p.up, a, 2 * up_to(inner, 16), st);
  if (e != S1F_OK) return e;
  set_out(a, y, y_rows(d), 1.f);
  for (int64_t at = 0; at < inner && e == S1F_OK; at += p.y_terms) {
    set_product(a, Matrix{a.h + at, a.h_ld, a.h_plane}, Matrix{mo.data + at, mo.ld, mo.plane}, p.n, p.n, d->hidden, d->hidden, std::min(p.y_terms, inner - at));
    set_weight(a, reinterpret_cast<const T *>(w_out) + at, out_stride);
    e = at == 0 ? launch_product<Of3<T, false, false, R>::template Of>(p.down, a, d->hidden, st) : launch_product<Of3<T, false, false, kNext<T>>::template Of>(p.down, a, d->hidden, st);
  }
  return e;
}

template <typename T, Result W>
int backward(const s1f_rows *d, const FfnPlan &p, const void *dy, const void *x, const void *w_in, int64_t in_stride, const void *w_out, int64_t out_stride, int64_t inner,
             int32_t act, const void *gate_up, void *dx, void *dw_in, int64_t dw_in_stride, void *dw_out, int64_t dw_out_stride, char *ws, hipStream_t st) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr Result R = F32 ? kStoreF32 : kStoreBf16;
  constexpr float kDown = F32 ? 1.f / kUp : 1.f;   // dy's planes, and those of what comes of it, are kUp times as large
  FfnArgs a = args_of(p, inner, act, gate_up, ws);
  Operands ops{a, d, p.planes};
  const Matrix mdy = ops.rows(dy, d->y_stride_b, d->y_stride_s, F32, p.width, ws + p.dy);
  const Matrix mx = ops.rows(x, d->x_stride_b, d->x_stride_s, false, p.width, ws + p.x);
  const Matrix mi = ops.weight(w_in, 2 * inner, d->hidden, in_stride, p.width, p.direct_in, ws + p.w_in);
  const Matrix mo = ops.weight(w_out, d->hidden, inner, out_stride, p.inner_width, p.direct_out, ws + p.w_out);
  int e = ops.pack(st);
  if (e != S1F_OK) return e;
  const int64_t h = d->hidden, n = p.n;
  const Matrix mdz = {a.dz, a.dz_ld, a.dz_plane}, mh = {a.h, a.h_ld, a.h_plane};
  set_product(a, mdy, mo, n, n, inner, p.inner_width, h);
  set_weight(a, w_out, out_stride);
  e = launch_product<Dh<T>::template Of>(p.dh, a, inner, st);
  if (e != S1F_OK) return e;
  auto from = [](Matrix m, int64_t row) { return Matrix{m.data + row * m.ld, m.ld, m.plane}; };
  for (int64_t at = 0; at < n && e == S1F_OK; at += p.per_turn) {
    const int64_t rows = std::min(p.per_turn, n - at);
    set_product(a, from(mdz, at), from(mx, at), 2 * inner, p.dz_ld, h, p.width, rows);
    set_out(a, dw_in, RowsOf{0, dw_in_stride, Divisor::of(2 * inner)}, kDown);
    e = launch_product<Of3<T, true, true, W>::template Of>(p.dw_in, a, h, st);
    if (e != S1F_OK) return e;
    set_product(a, from(mdy, at), from(mh, at), h, p.width, inner, p.inner_width, rows);
    set_out(a, dw_out, RowsOf{0, dw_out_stride, Divisor::of(h)}, kDown);
    e = launch_product<Of3<T, true, true, W>::template Of>(p.dw_out, a, inner, st);
  }
  if (e != S1F_OK) return e;
  // (last, when nobody reads dy, x and gate_up any more: it may lie in their place)
  set_out(a, dx, x_rows(d), kDown);
  for (int64_t at = 0; at < 2 * inner && e == S1F_OK; at += p.dx_terms) {
    set_product(a, Matrix{mdz.data + at, mdz.ld, mdz.plane}, from(mi, at), n, n, h, p.width, std::min(p.dx_terms, 2 * inner - at));
    set_weight(a, reinterpret_cast<const T *>(w_in) + at * in_stride, in_stride);
    e = at == 0 ? launch_product<Of3<T, false, true, R>::template Of>(p.dx, a, h, st) : launch_product<Of3<T, false, true, kNext<T>>::template Of>(p.dx, a, h, st);
  }
  return e;
}

}  // namespace
}  // namespace s1f

using namespace s1f;

extern "C" size_t s1f_gated_ffn_fwd_workspace_bytes(const s1f_rows *desc, int64_t inner, int64_t w_in_stride, int64_t w_out_stride) {
  return check_ffn(desc, inner, w_in_stride, w_out_stride) == S1F_OK ? (size_t)plan_of(desc, inner, w_in_stride, w_out_stride, false).bytes : 0;
}
extern "C" size_t s1f_gated_ffn_bwd_workspace_bytes(const s1f_rows *desc, int64_t inner, int64_t w_in_stride, int64_t w_out_stride) {
  return check_ffn(desc, inner, w_in_stride, w_out_stride) == S1F_OK ? (size_t)plan_of(desc, inner, w_in_stride, w_out_stride, true).bytes : 0;
}

extern "C" int s1f_gated_ffn_fwd(const s1f_rows *desc, const void *x, const void *w_in, int64_t w_in_stride, const void *w_out, int64_t w_out_stride,
                                 int64_t inner, int32_t act, void *y, void *gate_up, void *workspace, size_t workspace_bytes, void *hip_stream) {
  const int rc = check_ffn(desc, inner, w_in_stride, w_out_stride);
  if (rc != S1F_OK) return rc;
  if (act < S1F_SILU || act > S1F_GELU_TANH) return S1F_EINVAL;
  if (!x || !w_in || !w_out || !y || !workspace || !on_element(x, desc->dtype) || !on_element(y, desc->dtype) || !on_element(gate_up, desc->dtype) || !on16(w_in) ||
      !on16(w_out) || !on16(workspace))
    return S1F_EINVAL;
  const FfnPlan p = plan_of(desc, inner, w_in_stride, w_out_stride, false);
  if (workspace_bytes < (size_t)p.bytes) return S1F_EINVAL;
  char *ws = reinterpret_cast<char *>(workspace);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  return desc->dtype == S1F_BF16 ? forward<bf16_t>(desc, p, x, w_in, w_in_stride, w_out, w_out_stride, inner, act, y, gate_up, ws, st)
                                 : forward<float>(desc, p, x, w_in, w_in_stride, w_out, w_out_stride, inner, act, y, gate_up, ws, st);
}

extern "C" int s1f_gated_ffn_bwd(const s1f_rows *desc, const void *dy, const void *x, const void *w_in, int64_t w_in_stride, const void *w_out,
                                 int64_t w_out_stride, int64_t inner, int32_t act, const void *gate_up, void *dx, void *dw_in, int64_t dw_in_stride, void *dw_out,
                                 int64_t dw_out_stride, int32_t dweight_dtype, void *workspace, size_t workspace_bytes, void *hip_stream) {
  const int rc = check_ffn(desc, inner, w_in_stride, w_out_stride);
  if (rc != S1F_OK) return rc;
  if (dweight_dtype != S1F_F32 && !(dweight_dtype == S1F_BF16 && desc->dtype == S1F_BF16)) return S1F_EUNSUPPORTED;
  if (act < S1F_SILU || act > S1F_GELU_TANH || dw_in_stride < desc->hidden || (desc->hidden > 1 && dw_out_stride < inner)) return S1F_EINVAL;
  for (const void *p : {dy, x, gate_up, (const void *)dx})
    if (!p || !on_element(p, desc->dtype)) return S1F_EINVAL;
  if (!w_in || !w_out || !dw_in || !dw_out || !workspace || !on16(w_in) || !on16(w_out) || !on16(workspace) || !on_element(dw_in, dweight_dtype) ||
      !on_element(dw_out, dweight_dtype))
    return S1F_EINVAL;
  const FfnPlan p = plan_of(desc, inner, w_in_stride, w_out_stride, true);
  if (workspace_bytes < (size_t)p.bytes) return S1F_EINVAL;
  char *ws = reinterpret_cast<char *>(workspace);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  auto go = [&](auto call) { return call(desc, p, dy, x, w_in, w_in_stride, w_out, w_out_stride, inner, act, gate_up, dx, dw_in, dw_in_stride, dw_out, dw_out_stride, ws, st); };
  if (desc->dtype == S1F_F32) return go(&backward<float, kAddF32>);
  return dweight_dtype == S1F_F32 ? go(&backward<bf16_t, kAddF32>) : go(&backward<bf16_t, kStoreBf16>);
}
