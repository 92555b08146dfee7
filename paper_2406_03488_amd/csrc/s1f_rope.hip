// Queries and keys of a segment turned by their positions, on the way from a projection into the attention (queries) and the K/V cache
// (keys; values go along as they are), with or without a norm of every head in front, and the way back.
//
//   forward    y = x, or with the norm y = x * rstd * gain,  rstd = 1 / sqrt(sum(x^2) / d + eps)
//              pair i of the rotary_dim / 2 that are turned, as a complex number:  out_i = m * e^(i p f_i) * y_i;  p position, m magnitude
//   backward   dy_i = m * e^(-i p f_i) * dout_i;  with the norm  xhat = x * rstd,  dgain += sum over rows and heads of dy * xhat,
//              g = dy * gain,  dx = rstd * (g - xhat * sum(g * xhat) / d)
//
// Bound by memory: each element is read and written once, between which a row's angles, computed once for all heads that a lane takes, are next to nothing.  A row of a head lies in
// the registers of a few lanes, 16 bytes of the wider type to each, and mostly both elements of a pair in one lane.  4097 tokens of 64 and 2 x 8 heads of 128, bf16: 168 MB, 39.9 us, 4.2 TB/s
// (a large copy: 4.65); their gradient for 4096 tokens of 3 x 32 heads, 268 MB, 58.5 us, 4.6 TB/s; norms and rotation of 4897 tokens of 3 x 56 heads, 421 MB, 90.0 us, 4.7 TB/s; the gradient of 8774
// tokens of 64 and 2 x 8 heads, 557 MB, 126 us, 4.4 TB/s, 0.6 of which the vector units are busy.  One token of 64 + 16 heads 4.4 us, a launch.
// Angles are products in 64 bits: at position 2^20 one in 32 bits is off by 2^-4.  The norm's sums are fp32, as is everything between load and store; results are rounded once.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <initializer_list>
#include <type_traits>

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
  // Units of work: 2^log_rows rows of up to `unit_heads` heads of one of the tensors; units_q, units_k, units_v to a block of rows, all blocks one behind the other,
  // `per_group` consecutive ones (the remainder one more each) to a workgroup
  int32_t log_rows, at_once, unit_heads, units_q, units_k, units_v;   // at_once: heads of a lane in a unit
  Divisor by_units;
  int32_t step;                         // between units of a block that follow one another (see cut_units)
  int32_t units, per_group, remainder;
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
  S1F_DEV static void store(T *p, const float *x) {
    typedef float Floats __attribute__((ext_vector_type(PIECE)));
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      Floats f;
#pragma unroll
      for (int e = 0; e < PIECE; ++e) f[e] = x[i * PIECE + e];
      reinterpret_cast<Vec *>(p)[i] = __builtin_convertvector(f, Vec);
    }
  }
};

// cos and sin of a 64-bit angle: the quarter turn and the rest in 64 bits (pi/2 as two numbers; a fused product takes off the first exactly), the rest's
// series in 32, to 2^-25 of the result.  FAR: angles from kFar on, the number of whose quarter turns is not whole to a fraction of one any more: what is left of them is reduced once again, up to 2^79.
constexpr double kFar = 0x1p48;
template <bool FAR> S1F_DEV void cos_sin(double angle, float &c, float &s) {
  constexpr double kPerQuarter = 0.63661977236758134308;
  const auto less = [](double x, double n) { return fma(-n, 6.123233995736766036e-17, fma(-n, 1.5707963267948965580, x)); };
  double turns = rint(angle * kPerQuarter), rest = less(angle, turns);
  if (FAR && fabs(angle) > kFar) {
    const double more = rint(rest * kPerQuarter);
    rest = less(rest, more);
    turns = turns - 4.0 * floor(turns * 0.25) + more;
  }
  const float x = (float)rest;
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

// How a row's elements and its pairs are dealt out to lanes, PW pairs or 2 PW elements to each share.
//   kHalves  pairs (i, i + half), where half is whole shares: a share has both elements of its pairs
//   kPairs   pairs (2i, 2i + 1): likewise, and its elements are neighbours
//   kAny     pairs (i, i + half), half whatever it is: a share is 2 PW neighbours, and the other elements of their pairs come through LDS (2 x 1357 rows of 3 x 32 heads of 80, 20 of them
//            turned, gradient with norms 54 us; shares of two pairs, 4 bytes of bf16 to a load, 63)
enum Layout { kHalves, kPairs, kAny };
// The lane's elements of a row: [at[0], +PW) and [at[1], +PW).
template <int PW, Layout LAYOUT> struct Share {
  int at[2];
  S1F_DEV Share(const RopeArgs &a, int item) {
    if (LAYOUT != kHalves || item * PW >= a.half) {
      at[0] = LAYOUT != kHalves ? 2 * PW * item : a.rotary + 2 * (item * PW - a.half);
      at[1] = at[0] + PW;
    } else {
      at[0] = item * PW;
      at[1] = at[0] + a.half;
    }
  }
  // where element e < 2 PW lies.  (Not at[e / PW]: an array that is indexed by what is not a constant makes the compiler read the size of the workgroup out of the launch's packet, in the host's
  // memory, one workgroup after the other: norms and rotation of 385 tokens of 32 + 2 x 8 heads of 64, fp32, 17.7 us instead of 4.9, their gradient 23.3 instead of 11.7.)
  S1F_DEV int of(int e) const { return e < PW ? at[0] + e : at[1] + e - PW; }
  // which of the lane's elements e < 2 PW is the first, the second of its pair i
  S1F_DEV static constexpr int first(int i) { return LAYOUT == kPairs ? 2 * i : i; }
  S1F_DEV static constexpr int second(int i) { return LAYOUT == kPairs ? 2 * i + 1 : PW + i; }
};
// What a wave's lanes have written to LDS before is what they read there behind it.
S1F_DEV void between_lanes() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A lane's elements of a head as they lie in memory: fp32, or bf16 in half as many words.
template <int PW, int IT> struct Raw {
  uint32_t w[IT][2][PW];
  template <typename S> S1F_DEV void load(const S *p, const int (&at)[IT][2]) {
    typedef Run<S, PW> R;
#pragma unroll
    for (int t = 0; t < IT; ++t)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        R r;
        r.load(p + at[t][k]);
        if constexpr (sizeof(S) == 2 && PW == 1) w[t][k][0] = __builtin_bit_cast(uint16_t, r.v[0][0]);
        else __builtin_memcpy(w[t][k], r.v, sizeof(S) * PW);
      }
  }
  template <typename S> S1F_DEV float get(int t, int k, int e) const {
    if constexpr (sizeof(S) == 4) return __builtin_bit_cast(float, w[t][k][e]);
    else return __builtin_bit_cast(float, e & 1 ? w[t][k][e / 2] & 0xffff0000u : w[t][k][e / 2] << 16);
  }
};

enum Kind { kQ, kK, kV };
struct Unit {
  int block, kind, head;   // block of rows; tensor; first head
};
S1F_DEV Unit unit_of(const RopeArgs &a, int unit) {
  int block, u, unused;
  div_mod(unit, a.by_units, block, u);
  div_mod(u * a.step, a.by_units, unused, u);
  const int kind = u < a.units_q ? kQ : u < a.units_q + a.units_k ? kK : kV;
  return Unit{block, kind, (u - (kind == kQ ? 0 : kind == kK ? a.units_q : a.units_q + a.units_k)) * a.unit_heads};
}

// T: type of the tensors, K: of the keys' and values' source (fp32 accumulators in the backward).  L lanes to a row, IT shares to a lane, U heads to a lane and unit.  BACK: turn back.
// The groups of L lanes that a workgroup has beyond its 2^log_rows rows share the heads of a unit.  A head of the next unit is asked for as soon as this one's has become numbers, and
// the first unit before the angles are computed.  Lanes without a share, a row or a head of their own work on another's and leave nothing behind.  (Units of one tensor, four heads to a lane and 16 bytes of
// fp32 to a load, instead of a lane walking all heads: gqa segment 50 -> 40 us, 7b gradient 72 -> 58.  Where a lane's row lies kept in registers instead of multiplied out for each head: 8 % fewer
// vector instructions, one wave less to a unit, gradient with norms 131 -> 145.  Heads behind a tensor's last passed over: ragged gradient with norms 54 -> 59, of 5 + 1 heads no faster.)
template <typename T, typename K, int PW, int L, int IT, int U, Layout LAYOUT, bool NORM, bool BACK> __global__ void __launch_bounds__(256) rope_kernel(const RopeArgs a) {
  constexpr int E = 2 * PW, GAIN_COLS = L * IT * E, ANGLES = LAYOUT == kAny ? E : PW;   // ANGLES: of pairs, or (kAny) of elements
  static_assert(LAYOUT != kAny || IT == 1, "one share to a lane");
  constexpr bool GAINS = NORM && BACK;
  __shared__ __attribute__((aligned(16))) float gains[NORM ? 2 * GAIN_COLS : 1];
  const int lane = threadIdx.x % L, group = threadIdx.x / L, in_row = group & ((1 << a.log_rows) - 1), slot = group >> a.log_rows, slots = (256 / L) >> a.log_rows;
  const int g = blockIdx.x, first = g * a.per_group + (g < a.remainder ? g : a.remainder), last = first + a.per_group + (g < a.remainder ? 1 : 0);
  bool has[IT];
  int at[IT][2], straight[IT][2];   // the lane's elements of a row, and of values, which are not turned
#pragma unroll
  for (int t = 0; t < IT; ++t) {
    const int item = lane + t * L, known = item < a.items ? item : 0;
    const Share<PW, LAYOUT> share(a, known);
    has[t] = item < a.items;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      at[t][k] = share.at[k];
      straight[t][k] = known * E + k * PW;
    }
  }
  int b, r;
  bool row_is;
  auto go_to = [&](int block) {
    const int row = (block << a.log_rows) + in_row;
    row_is = row < a.n;
    div_mod(row_is ? row : a.n - 1, a.by_rows, b, r);
  };
  auto heads_of = [&](const Unit &u) { return u.kind == kQ ? a.n_q : a.n_k; };
  auto head_of = [&](const Unit &u, int i) { return u.head + slot + i * slots; };
  Raw<PW, IT> in[U], x[GAINS ? U : 1];
  auto ask = [&](const Unit &u, int i) {
    if (i >= a.at_once) return;
    const int heads = heads_of(u), own = head_of(u, i), h = own < heads ? own : heads - 1;
    const HeadStrides &ss = u.kind == kQ ? a.src_qs : a.src_ks, &xs = u.kind == kQ ? a.dst_qs : a.dst_ks;
    const int64_t from = b * ss.sb + r * ss.ss + h * ss.sh;
    if (u.kind == kQ) in[i].load(reinterpret_cast<const T *>(a.src_q) + from, at);
    else if (u.kind == kK) in[i].load(reinterpret_cast<const K *>(a.src_k) + from, at);
    else in[i].load(reinterpret_cast<const K *>(a.src_v) + from, straight);
    if constexpr (GAINS)
      if (u.kind != kV) x[i].load(reinterpret_cast<const T *>(u.kind == kQ ? a.x_q : a.x_k) + b * xs.sb + r * xs.ss + h * xs.sh, at);
  };
  Unit next = unit_of(a, first);
  go_to(next.block);
#pragma unroll
  for (int i = 0; i < U; ++i) ask(next, i);
  // kAny: elements of the wave's rows, element e of a lane at 64 e + lane, so that neither writes nor reads meet in a bank; where the lane's elements' partners are
  __shared__ float exchange[LAYOUT == kAny ? 4 : 1][LAYOUT == kAny ? 64 * E : 1];
  int partner[LAYOUT == kAny ? E : 1];
  if constexpr (LAYOUT == kAny) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = lane * E + e, other = i < a.half ? i + a.half : i < a.rotary ? i - a.half : i;
      partner[e] = other % E * 64 + other / E + ((int)threadIdx.x & 63) - lane;
    }
  }
  float c[IT][ANGLES], s[IT][ANGLES];
  auto angles = [&]() {
    const int64_t position = a.positions ? a.positions[b * a.positions_sb + r] : a.first_position + r;
    bool far = false;
    auto turn = [&](auto again) {
#pragma unroll
      for (int t = 0; t < IT; ++t)
#pragma unroll
        for (int i = 0; i < ANGLES; ++i) {
          const int of = (lane + t * L) * ANGLES + i;
          const bool second = LAYOUT == kAny && of >= a.half;
          const int pair = second ? of - a.half : of;
          c[t][i] = 1.f;
          s[t][i] = 0.f;
          if (pair < a.half) {
            const double angle = (double)position * a.freqs[pair];
            far = far || fabs(angle) > kFar;
            cos_sin<decltype(again)::value>(angle, c[t][i], s[t][i]);
            c[t][i] *= a.magnitude;
            s[t][i] *= BACK != second ? -a.magnitude : a.magnitude;
          }
        }
    };
    turn(std::false_type{});
    if (__builtin_expect(__any(far), 0)) turn(std::true_type{});
  };
  int angles_of = -1;
  if constexpr (NORM) {   // (under the angles' latencies)
    constexpr int PER = (2 * GAIN_COLS + 255) / 256;
    float gain[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int i = threadIdx.x + 256 * p, side = i / GAIN_COLS, col = i % GAIN_COLS, item = col / E, e = col % E;
      const Share<PW, LAYOUT> share(a, item);
      gain[p] = side < 2 && item < a.items ? (float)reinterpret_cast<const T *>(side ? a.gain_k : a.gain_q)[share.of(e)] : 0.f;
    }
    if (next.kind != kV) {
      angles();
      angles_of = next.block;
    }
#pragma unroll
    for (int p = 0; p < PER; ++p)
      if (threadIdx.x + 256 * p < 2 * GAIN_COLS) gains[threadIdx.x + 256 * p] = gain[p];
    __syncthreads();
  }
  float dg[2][IT][E];
  if constexpr (GAINS) {
#pragma unroll
    for (int t = 0; t < IT; ++t)
#pragma unroll
      for (int e = 0; e < E; ++e) dg[0][t][e] = dg[1][t][e] = 0.f;
  }
#pragma unroll 1
  for (int unit = first; unit < last; ++unit) {
    const Unit u = next;
    if (u.kind != kV && angles_of != u.block) {
      angles_of = u.block;
      angles();
    }
    const bool is = row_is, more = unit + 1 < last;
    const int heads = heads_of(u);
    const HeadStrides &ds = u.kind == kQ ? a.dst_qs : a.dst_ks;
    T *to = reinterpret_cast<T *>(u.kind == kQ ? a.dst_q : u.kind == kK ? a.dst_k : a.dst_v) + b * ds.sb + r * ds.ss;
    if (more) {
      next = unit_of(a, unit + 1);
      if (next.block != u.block) go_to(next.block);
    }
    float of_unit[IT][E];
#pragma unroll
    for (int t = 0; t < IT; ++t)
#pragma unroll
      for (int e = 0; e < E; ++e) of_unit[t][e] = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (i >= a.at_once) break;
      const int h = head_of(u, i);
      const bool mine = is && h < heads;
      float v[IT][E], w[IT][E];
#pragma unroll
      for (int t = 0; t < IT; ++t)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (sizeof(T) != sizeof(K) && u.kind != kQ) v[t][e] = in[i].template get<K>(t, e / PW, e % PW);
          else v[t][e] = in[i].template get<T>(t, e / PW, e % PW);
          if constexpr (GAINS) w[t][e] = x[i].template get<T>(t, e / PW, e % PW);
        }
      if (more) ask(next, i);
      if (u.kind != kV) {
        const float *gain = gains + (NORM ? (u.kind == kQ ? 0 : GAIN_COLS) + lane * E : 0);
        // sum of squares of a row, and one over the root of their mean
        auto rstd_of = [&](const float (&y)[IT][E]) {
          float sum = 0.f;
#pragma unroll
          for (int t = 0; t < IT; ++t) {
            float part = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) part = fmaf(y[t][e], y[t][e], part);
            sum += has[t] ? part : 0.f;
          }
          return __builtin_amdgcn_rsqf(fmaf(sum_of<L>(sum), a.inv_dim, a.eps));
        };
        if constexpr (NORM && !BACK) {
          const float rstd = rstd_of(v);
#pragma unroll
          for (int t = 0; t < IT; ++t)
#pragma unroll
            for (int e = 0; e < E; ++e) v[t][e] = v[t][e] * rstd * gain[t * L * E + e];
        }
        if constexpr (LAYOUT == kAny) {
          float *of_wave = exchange[threadIdx.x >> 6];
#pragma unroll
          for (int e = 0; e < E; ++e) of_wave[64 * e + (threadIdx.x & 63)] = v[0][e];
          between_lanes();
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float other = of_wave[partner[e]];
            v[0][e] = lane * E + e < a.rotary ? v[0][e] * c[0][e] - other * s[0][e] : v[0][e];
          }
          between_lanes();
        } else {
#pragma unroll
          for (int t = 0; t < IT; ++t)
#pragma unroll
            for (int p = 0; p < PW; ++p) {
              constexpr auto F = &Share<PW, LAYOUT>::first, G = &Share<PW, LAYOUT>::second;
              float &re = v[t][F(p)], &im = v[t][G(p)];
              const bool turned = (lane + t * L) * PW + p < a.half;   // (the others stay what they are, infinities too)
              const float was = re;
              re = turned ? was * c[t][p] - im * s[t][p] : was;
              im = turned ? im * c[t][p] + was * s[t][p] : im;
            }
        }
        if constexpr (GAINS) {
          const float rstd = rstd_of(w);
          float along = 0.f;
#pragma unroll
          for (int t = 0; t < IT; ++t) {
            const float by = mine && has[t] ? rstd : 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
              w[t][e] *= by;
              of_unit[t][e] = fmaf(mine ? v[t][e] : 0.f, w[t][e], of_unit[t][e]);   // (another's may be infinite)
              v[t][e] *= gain[t * L * E + e];
              along = fmaf(v[t][e], w[t][e], along);
            }
          }
          along = sum_of<L>(along) * a.inv_dim;
#pragma unroll
          for (int t = 0; t < IT; ++t)
#pragma unroll
            for (int e = 0; e < E; ++e) v[t][e] = rstd * (v[t][e] - w[t][e] * along);
        }
      }
#pragma unroll
      for (int t = 0; t < IT; ++t)
        if (has[t] && mine) {
#pragma unroll
          for (int k = 0; k < 2; ++k) Run<T, PW>::store(to + h * ds.sh + (u.kind == kV ? straight[t][k] : at[t][k]), &v[t][k * PW]);
        }
    }
    if constexpr (GAINS) {
#pragma unroll
      for (int t = 0; t < IT; ++t)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (u.kind == kQ) dg[0][t][e] += of_unit[t][e];
          else if (u.kind == kK) dg[1][t][e] += of_unit[t][e];
        }
    }
  }
  if constexpr (GAINS) {   // the groups' sums of q, then of k, in their order; columns [item][element]
    constexpr int GROUPS = 256 / L, COLS = L * IT * E;
    __shared__ float sums[GROUPS][COLS + 1];
    float *part = a.part + (int64_t)blockIdx.x * 2 * a.dim;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      __syncthreads();
#pragma unroll
      for (int t = 0; t < IT; ++t)
#pragma unroll
        for (int e = 0; e < E; ++e) sums[group][(t * E + e) * L + lane] = dg[side][t][e];
      __syncthreads();
      for (int col = threadIdx.x; col < COLS; col += 256) {
        const int item = col % L + col / (L * E) * L, e = col / L % E;
        if (item >= a.items) continue;
        float sum = 0.f;
        for (int g = 0; g < GROUPS; ++g) sum += sums[g][col];
        const Share<PW, LAYOUT> share(a, item);
        part[side * a.dim + share.of(e)] = sum;
      }
    }
  }
}

// Adds the workgroups' sums: 16 columns of [q, k][dim] per workgroup, 64 shares of the parts (16 shares of 64 columns: chains of loads, 5.0 us for 768 parts of 160).
__global__ void __launch_bounds__(1024) rope_join_kernel(const RopeArgs a) {
  constexpr int SHARES = 64;
  __shared__ float of_share[SHARES][16];
  const int in = threadIdx.x & 15, share = threadIdx.x >> 4, width = 2 * a.dim, col = blockIdx.x * 16 + in;
  float sum = 0.f;
  if (col < width) {
    const int begin = a.parts * share / SHARES, end = a.parts * (share + 1) / SHARES;
#pragma unroll 8
    for (int p = begin; p < end; ++p) sum += a.part[(int64_t)p * width + col];
  }
  of_share[share][in] = sum;
  __syncthreads();
  if (share > 0 || col >= width) return;
  sum = 0.f;
#pragma unroll 16
  for (int w = 0; w < SHARES; ++w) sum += of_share[w][in];
  float *to = col < a.dim ? a.dgain_q + col : a.dgain_k + col - a.dim;
  *to += sum;
}

// ---- host ------------------------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostTokens = int64_t(1) << 26;
constexpr int32_t kMostHeads = 1 << 16, kMostDim = 256;
// Workgroups of a backward with the norm, each of which leaves sums: as many as the device holds at once, each an equal share of the units (gqa segment: 1024 where it holds 768 at once 154 us, 768
// 128).  Of the other calls: about as many as keep memory busy, several units to each only where there are more.
constexpr int kMostParts = 2048;
constexpr int64_t kMostGroups = 4096;
constexpr int64_t kFew = int64_t(1) << 22;   // elements
constexpr int64_t kMostTokenHeads = int64_t(1) << 31;   // (units of work are numbered in 32 bits)

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
  if (d->batch * d->rows * (d->n_q_heads + 2 * (int64_t)d->n_kv_heads) > kMostTokenHeads) return S1F_EUNSUPPORTED;
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

// How a call's rows are dealt out, and pairs to a share: 8 or 4 (16 bytes) where addresses allow it, else 1.
struct Dealt {
  Layout layout;
  int pairs;
};
Dealt deal(const s1f_heads *d, int most, const Alignment &typed, const Alignment &wide, int64_t esz) {
  for (int pw = most; pw >= 4; pw /= 2) {
    if (d->head_dim % (2 * pw) != 0 || !typed.at_least(pw * esz) || !wide.at_least(pw * 4)) continue;
    if (d->interleaved) return {kPairs, pw};
    if (d->rotary_dim / 2 % pw == 0) return {kHalves, pw};
    if (pw == 4) return {kAny, pw};
  }
  return {d->interleaved ? kPairs : kHalves, 1};
}

// Workgroups of a kernel that the device holds at once, asked once per device.
template <auto KERNEL> int held_at_once() {
  static std::atomic<int> known[64];
  int dev = 0, per_unit = 0, units = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 512;
  const bool cached = dev >= 0 && dev < 64;
  if (cached && known[dev].load(std::memory_order_acquire) > 0) return known[dev].load(std::memory_order_acquire);
  if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_unit, reinterpret_cast<const void *>(KERNEL), 256, 0) != hipSuccess ||
      hipDeviceGetAttribute(&units, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || per_unit < 1 || units < 1) {
    (void)hipGetLastError();
    return 512;
  }
  if (cached) known[dev].store(per_unit * units, std::memory_order_release);
  return per_unit * units;
}
struct Instance {
  void (*kernel)(RopeArgs);
  int (*held)();
  int lanes, heads;   // to a row; of a lane at once
};
template <typename T, typename K, Layout LAYOUT, bool NORM, bool BACK> Instance instance_of(int pw, int items) {
#define S1F_ROPE_INSTANCE(PW, L, IT, U) Instance{&rope_kernel<T, K, PW, L, IT, U, LAYOUT, NORM, BACK>, &held_at_once<&rope_kernel<T, K, PW, L, IT, U, LAYOUT, NORM, BACK>>, L, U}
  if constexpr (sizeof(T) == 2 && !BACK && LAYOUT != kAny) {
    if (pw == 8) return items <= 4 ? S1F_ROPE_INSTANCE(8, 4, 1, 4) : items <= 8 ? S1F_ROPE_INSTANCE(8, 8, 1, 4) : S1F_ROPE_INSTANCE(8, 16, 1, 4);
  }
  constexpr int U = NORM && BACK ? 2 : 4;
  if constexpr (LAYOUT != kAny) {
    if (pw == 1) return items <= 32 ? S1F_ROPE_INSTANCE(1, 8, 4, 2) : items <= 64 ? S1F_ROPE_INSTANCE(1, 16, 4, 2) : S1F_ROPE_INSTANCE(1, 32, 4, 2);
  }
  return items <= 8 ? S1F_ROPE_INSTANCE(4, 8, 1, U) : items <= 16 ? S1F_ROPE_INSTANCE(4, 16, 1, U) : S1F_ROPE_INSTANCE(4, 32, 1, U);
#undef S1F_ROPE_INSTANCE
}
static_assert(kMostDim / 2 <= 32 * 4 && kMostDim / 8 <= 32 && kMostDim / 16 <= 16, "a row has a place in the lanes");

// Units of work, and workgroups.
int64_t cut_units(RopeArgs &a, const Instance &in, bool gains) {
  const int groups = 256 / in.lanes;
  a.log_rows = 0;
  while ((2 << a.log_rows) <= groups && (int64_t(1) << a.log_rows) < a.n) ++a.log_rows;
  const int64_t blocks = ((int64_t)a.n + (int64_t(1) << a.log_rows) - 1) >> a.log_rows;
  int64_t per_block = 0;
  // (fewer heads to a unit where there would not be one for every compute unit)
  for (a.at_once = in.heads; ; a.at_once /= 2) {
    a.unit_heads = (groups >> a.log_rows) * a.at_once;
    auto units = [&](int heads) { return (heads + a.unit_heads - 1) / a.unit_heads; };
    a.units_q = units(a.n_q);
    a.units_k = units(a.n_k);
    a.units_v = units(a.n_v);
    per_block = a.units_q + a.units_k + a.units_v;
    if (a.at_once == 1 || blocks * per_block >= 256) break;
  }
  const int64_t all = blocks * per_block;
  a.by_units = Divisor::of(per_block);
  // Consecutive units take the tensors in turn: values are less work than the others, and a workgroup's share of some ten units would be of one kind: gradient of 2 x 1357 rows of
  // 3 x 32 heads of 80 64.4 -> 62.8 us.
  auto common = [](int64_t x, int64_t y) {
    while (y) std::swap(x %= y, y);
    return x;
  };
  a.step = 1;
  if (gains && per_block > 2 && per_block < 32768)
    for (a.step = (int32_t)(per_block * 0.618); common(per_block, a.step) != 1; ++a.step) {}
  a.units = (int32_t)all;
  int64_t grid = gains ? std::min<int64_t>({all, in.held(), kMostParts}) : all;
  if (!gains && all > kMostGroups) grid = (all + (all + kMostGroups - 1) / kMostGroups - 1) / ((all + kMostGroups - 1) / kMostGroups);
  a.per_group = (int32_t)(all / grid);
  a.remainder = (int32_t)(all % grid);
  a.parts = (int32_t)grid;
  return grid;
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
  // (16 bytes of either type to a lane, but for few elements, where twice the lanes compute half as many angles each: 200 tokens of 32 + 2 x 8 heads of 128 4.8 -> 4.5 us, 600 5.8 -> 5.5)
  const int64_t elements = (int64_t)a.n * (a.n_q + a.n_k + a.n_v) * a.dim;
  const Dealt dealt = deal(d, esz == 2 && !BACK && elements > kFew ? 8 : 4, typed, wide, esz);
  a.items = d->head_dim / (2 * dealt.pairs);
  auto pick = [&](auto t) {
    typedef decltype(t) T;
    typedef std::conditional_t<BACK, float, T> K;
    if (dealt.layout == kPairs) return instance_of<T, K, kPairs, NORM, BACK>(dealt.pairs, a.items);
    if (dealt.layout == kAny) return instance_of<T, K, kAny, NORM, BACK>(dealt.pairs, a.items);
    return instance_of<T, K, kHalves, NORM, BACK>(dealt.pairs, a.items);
  };
  const Instance in = d->dtype == S1F_F32 ? pick(float{}) : pick(bf16_t{});
  const int64_t grid = cut_units(a, in, NORM && BACK);
  const int e = launch_rows_kernel(in.kernel, grid, 256, a, st);
  if (e != S1F_OK || !(NORM && BACK)) return e;
  return launch_rows_kernel(&rope_join_kernel, (2 * a.dim + 15) / 16, 1024, a, st);
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
  // (each accumulator is added to by lanes of its own)
  if (dq_gain_acc < dk_gain_acc + desc->head_dim && dk_gain_acc < dq_gain_acc + desc->head_dim) return S1F_EINVAL;
  if (!tensors_ok(desc->dtype, {q, k, q_gain, k_gain}) || !(eps >= 0.f) || !dq_gain_acc || !dk_gain_acc || !on4(dq_gain_acc) || !on4(dk_gain_acc) ||
      !workspace || !on16(workspace) || workspace_bytes < s1f_qk_norm_rope_bwd_workspace_bytes(desc))
    return S1F_EINVAL;
  RopeArgs a = args_of(desc, freqs, magnitude, positions, positions_stride_b, first_position);
  a.x_q = q; a.x_k = k; a.gain_q = q_gain; a.gain_k = k_gain; a.eps = eps;
  a.dgain_q = dq_gain_acc; a.dgain_k = dk_gain_acc; a.part = reinterpret_cast<float *>(workspace);
  return backward<true>(desc, dq_rot, dk_prefix_acc, dv_prefix_acc, a, seg_off, dq, dk, dv, reinterpret_cast<hipStream_t>(hip_stream));
}
