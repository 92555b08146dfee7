// Matrix products of the token loss and of the gated feed-forward block (gfx950): C[m][n] = sum over k of A(m, k) * B(n, k), both operands bf16, sums fp32.
//
// A workgroup owns a BM x BN tile of C and walks k in stages of 64, which travel from memory to LDS by asynchronous copies and from
// there into the registers of the matrix instructions.  An operand is stored either way around:
//   rows     element (m, k) at base + m * ld + k: k runs along a row, as in products of rows with rows of the weight
//   columns  element (m, k) at base + k * ld + m: the contraction runs over rows; LDS reads that transpose hand the matrix instructions
//            what they need, and nothing is ever laid out anew in memory
//
// LDS layout of one operand and stage: pieces of 1 KiB, each filled by one copy instruction of a wave, lane l at byte 16 * l.
//   rows     8 rows of 128 bytes.  Chunk c (16 bytes) of row r lies in slot c ^ (r / 2 mod 8): the 16 lanes that a 128-bit read serves
//            together (0-3 with 12-15, 20-23 and 24-27, and so on) take 16 different slots.
//   columns  rows of 2 * BM bytes.  Unit u (32 bytes, 16 columns) of row k lies in slot u ^ h(k): a transposing read takes the same unit of rows
//            8j .. 8j+3 and 8j+8 .. 8j+11 together, which h spreads over all banks.
// Both keep a wave's 64 lanes on whole lines of memory.
//
// Bound by power and LDS: a round of 256 x 256 tiles of 256 stages (4096 rows of 16384 elements over 4096 tokens) takes 385 us, 1.43 PFLOP/s, matrix units 65 % busy at 2.09 GHz, of which
// a stage is 1.42 us (the difference to 128 stages), 1.52 PFLOP/s; in launches of milliseconds power leaves 1.8 GHz (4099 rows of 4096 over 50021 tokens: 70 % busy, 1.3 PFLOP/s).  Operands that
// are constant take 15 % less.  Eight waves of 128 x 64 read 192 KiB of operands per stage out of LDS, which takes about as long
// as their products; four waves of 128 x 128 read 128 KiB but have nobody to take turns with on their unit's four matrix pipes: no faster.
#pragma once
#include <type_traits>

#include "attn_tile.hpp"

namespace s1f {

constexpr int kDepth = 64;   // contraction per stage

template <int N> struct Int {
  static constexpr int value = N;
};
template <int N, int I = 0, typename F> S1F_DEV void for_each(F &&f) {   // f(Int<0>{}) .. f(Int<N - 1>{})
  if constexpr (I < N) {
    f(Int<I>{});
    for_each<N, I + 1>(f);
  }
}
S1F_DEV const char *uniform_pointer(const char *p) {
  const uint64_t bits = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const char *>(((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(bits >> 32)) << 32) |
                                        (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)bits));
}

// R: rows of C (or columns of C, for the other operand) in the tile; TR: stored by columns; NW: waves that copy.
template <int R, bool TR, int NW> struct Side {
  static constexpr int BYTES = R * kDepth * 2, PIECES = BYTES / 1024, PER_WAVE = PIECES / NW;
  static_assert(PIECES % NW == 0 && PER_WAVE <= 4, "a wave's pieces share one M0: the offset of a copy instruction reaches four");
  static_assert(!TR || R >= 128, "a unit has eight slots");
  static constexpr int ROW = TR ? 2 * R : 128, CHUNKS = ROW / 16, RPP = 1024 / ROW;   // bytes and chunks of a row, rows per piece
  S1F_DEV static int h(int k) { return (k & 3) | ((k >> 3) & 1) << 2; }

  static constexpr int BIAS = 1024 * (PER_WAVE - 1);
  const char *next;         // of the stage that is copied next, less BIAS (uniform)
  int64_t step;             // bytes to the next stage
  unsigned voff[PER_WAVE];  // of the lane's chunk in each of the wave's pieces
  int row_bytes;

  // The lane's slot in piece p: row within the stage's image and chunk of that row.
  S1F_DEV static void slot(int p, int lane, int &row, int &chunk) {
    row = p * RPP + lane / CHUNKS;
    const int c = lane % CHUNKS;
    chunk = TR ? ((((c >> 1) ^ h(row)) << 1) | (c & 1)) : (c ^ ((row >> 1) & 7));
  }
  // m0: first row (column) of the tile; limit: rows (columns) that there are; those behind are copies of the last (columns: first).
  // apart: 0, or (rows) the tile's blocks of 16 are taken in turn from the rows from m0 on, R / 2 of them, and from those `apart` rows behind them: what belongs together
  // of two products then lies in one wave's registers.
  S1F_DEV void init(const bf16_t *data, int64_t ld, int64_t m0, int64_t limit, int64_t apart, int k_stage, int wave, int lane) {
    row_bytes = (int)(ld * 2);
    step = TR ? kDepth * ld * 2 : kDepth * 2;
    next = reinterpret_cast<const char *>(TR ? data + m0 : data + m0 * ld) + k_stage * step - BIAS;
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      int r, c;
      slot(wave * PER_WAVE + i, lane, r, c);
      if (TR) {
        if (m0 + 8 * c >= limit) c = 0;
      } else {
        const int second = apart ? (r >> 4) & 1 : 0;
        if (apart) r = (r >> 5 << 4) + (r & 15);
        if (m0 + r >= limit) r = (int)(limit - 1 - m0);
        r += second ? (int)apart : 0;
      }
      // (the immediate offset of a copy instruction counts for its address in memory as well as in LDS)
      voff[i] = (unsigned)(r * row_bytes + 16 * c) + (unsigned)(BIAS - 1024 * i);
    }
  }
  // From here on stages hold `left` of their contraction: what is behind is read from the stage's beginning, and cleared by clear_tail.
  S1F_DEV void shorten(int left, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      int r, c;
      slot(wave * PER_WAVE + i, lane, r, c);
      if (TR) {
        if (r >= left) voff[i] -= (unsigned)(r * row_bytes);
      } else {
        if (8 * c >= left) voff[i] -= (unsigned)(16 * c);
      }
    }
  }
  // Copies piece I of the wave's pieces of a stage at `from` (uniform) to LDS address `dst` (of the wave's first piece; uniform).
  template <int I> S1F_DEV void copy(const char *from, unsigned dst) const {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3"
                 : : "s"(dst), "v"(voff[I]), "s"(from), "n"(1024 * I) : "m0");
  }
  // Zeros in the wave's own slots behind the end of the contraction, once its copies have landed.
  S1F_DEV void clear_tail(lds_addr at, int left, int wave, int lane) const {
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      int r, c;
      slot(wave * PER_WAVE + i, lane, r, c);
      if (TR ? r >= left : 8 * c >= left)
        *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>((uintptr_t)(at + (unsigned)((wave * PER_WAVE + i) * 1024 + 16 * lane))) = u32x4{0, 0, 0, 0};
    }
  }
  // Operand of one matrix instruction: rows (columns) 16 * block .. +15 of the tile, contraction 32 * half .. +31; of the latter
  // lane (n, j) holds 8j .. 8j+7, whichever way the operand is stored.
  // at(): the lane's address for the wave's first block; operand(): its block number `block`.
  S1F_DEV static lds_addr at(int first_block, int lane) {
    const int n = lane & 15, j = lane >> 4;
    if constexpr (TR) {
      const int k = 8 * j + (n >> 2);
      return (unsigned)(k * ROW + (n & 3) * 8) + ((unsigned)(h(k) * 32) ^ (unsigned)(first_block * 32));
    } else {
      return (unsigned)(first_block * 2048 + n * 128 + 16 * (j ^ ((n >> 1) & 7)));
    }
  }
  // (what has to be added to the address of a stage's half is a constant; see opaque)
  S1F_DEV static lds_addr half_of(lds_addr a, int half) { return opaque(TR ? a : a ^ (unsigned)(half * 64)); }
  S1F_DEV static bf16x8 operand(lds_addr a, int block, int half) {
    if constexpr (TR) {
      const lds_addr p = a ^ (unsigned)(block * 32);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          reinterpret_cast<__attribute__((address_space(3))) s16x4 *>((uintptr_t)(p + (unsigned)(half * 32 * ROW))));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          reinterpret_cast<__attribute__((address_space(3))) s16x4 *>((uintptr_t)(p + (unsigned)(half * 32 * ROW + 4 * ROW))));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      s16x8 r = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf16x8, r);
    } else {
      return lds_load<bf16x8>(a + (unsigned)(block * 2048));
    }
  }
};

// Operands of a product in memory.  planes: 1, or 3 for fp32 operands as three bf16 planes (see Planes), `plane` elements apart; the product
// is then the six products of planes that fp32 resolves, each a stage of its own.
struct Matrix {
  const bf16_t *data;
  int64_t ld, plane;
};

// The main loop: acc[mb][nb] = the block of rows 16 * (MB * wave_m + mb) and columns 16 * (NB * wave_n + nb), as the matrix
// instruction leaves it with the operands in this order: lane (n, j) holds row n, columns 4j .. 4j+3 of the block.
// PAIRS: 1, or 6 products of planes for each.
template <int BM, int BN, int WM, int WN, bool TRA, bool TRB, int PAIRS> struct Product {
  static constexpr int NW = WM * WN, THREADS = 64 * NW, MB = BM / WM / 16, NB = BN / WN / 16;
  typedef Side<BM, TRA, NW> SA;
  typedef Side<BN, TRB, NW> SB;
  static constexpr int LDS_BYTES = 3 * SA::BYTES + 2 * SB::BYTES;

  // k: contraction; stages [begin, end) of it, counted in stages of a product of planes, the PAIRS of each one after the other
  // b_apart: see Side::init
  S1F_DEV static void run(f32x4 (&acc)[MB][NB], const Matrix &a, const Matrix &b, int64_t m0, int64_t m_limit, int64_t n0, int64_t n_limit,
                          int64_t k, int begin, int end, lds_addr lds, int64_t b_apart = 0) {
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (begin >= end) return;
    SA sa;
    SB sb;
    sa.init(a.data, a.ld, m0, m_limit, 0, begin / PAIRS, wave, lane);
    sb.init(b.data, b.ld, n0, n_limit, b_apart, begin / PAIRS, wave, lane);
    const int left = (int)((k - 1) % kDepth) + 1;   // contraction of the last stage
    const int tail = left < kDepth ? (int)((k - 1) / kDepth) * PAIRS : 0x7fffffff;   // first stage that is not whole
    // Where a side's stage t is copied from, and to.  Calls are for consecutive stages.
    const char *from_a, *from_b;
    unsigned to_a, to_b;
    int pair_a = begin % PAIRS, pair_b = pair_a;
    auto begin_copy = [&](auto &side, const Matrix &m, unsigned order, int &pair, const char *&from, unsigned &to, int t, lds_addr dst) {
      if (t == tail || (t == begin && t > tail)) side.shorten(left, wave, lane);
      from = side.next;
      if constexpr (PAIRS == 6) from += (int64_t)((order >> (4 * pair)) & 3u) * m.plane * 2;
      from = uniform_pointer(from);
      to = __builtin_amdgcn_readfirstlane(dst + (unsigned)(wave * side.PER_WAVE * 1024));
      if (PAIRS == 1 || ++pair == PAIRS) {
        pair = 0;
        side.next += side.step;
      }
    };
    // planes of the pairs: (2,0) (0,2) (1,1) (1,0) (0,1) (0,0), smallest products first
    auto begin_a = [&](int t, lds_addr dst) { begin_copy(sa, a, 0x001102u, pair_a, from_a, to_a, t, dst); };
    auto begin_b = [&](int t, lds_addr dst) { begin_copy(sb, b, 0x010120u, pair_b, from_b, to_b, t, dst); };
    auto piece_a = [&](auto i) { sa.template copy<decltype(i)::value>(from_a, to_a); };
    auto piece_b = [&](auto i) { sb.template copy<decltype(i)::value>(from_b, to_b); };
    constexpr int PA = SA::PER_WAVE, PB = SB::PER_WAVE;
    auto landed = [&](int t, lds_addr at_a, lds_addr at_b) {        // this wave's copies of stage t are there
      if (t >= tail) {
        sa.clear_tail(at_a, left, wave, lane);
        sb.clear_tail(at_b, left, wave, lane);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    };
    // Three places for stages of A, two for those of B: all that LDS holds of 256 x 256 tiles.
    lds_addr a0 = lds, a1 = lds + SA::BYTES, a2 = a1 + SA::BYTES, b0 = a2 + SA::BYTES, b1 = b0 + SB::BYTES;
    begin_a(begin, a0);
    for_each<PA>(piece_a);
    begin_b(begin, b0);
    for_each<PB>(piece_b);
    if (begin + 1 < end) {
      begin_a(begin + 1, a1);
      for_each<PA>(piece_a);
      begin_b(begin + 1, b1);
      for_each<PB>(piece_b);
      wait_async_tiles_but_last<PA + PB>();
    } else {
      wait_async_tiles();
    }
    landed(begin, a0, b0);
    __syncthreads();
    // Operands are read half a stage ahead of the products that take them.  When the products of a stage's first half are through,
    // nobody reads that stage any more: one barrier per stage says so, and that the next one has landed.  Behind it B's stage after the next is
    // copied into the place that has become free, and under the first half of the next stage A's stage after that.
    bf16x8 fa[2][MB], fb[2][NB];
    const lds_addr lane_a = SA::at(wm * MB, lane), lane_b = SB::at(wn * NB, lane);
    constexpr int OPERANDS = MB + NB, PER_SLOT = (OPERANDS * 4 + 3 * MB - 1) / (3 * MB);   // read in the first three quarters of the products
    // Products of one half, and the reads of the operands of the next: a slot for each row of blocks, nothing moves across its end.  The wave's copies
    // are spread over the slots: a wave issues in order, and copies of all waves one right behind the other fill the queues of the memory
    // pipe, in front of which they then wait with their products behind them.
    auto half_stage = [&](bf16x8 (&ra)[MB], bf16x8 (&rb)[NB], const bf16x8 (&xa)[MB], const bf16x8 (&xb)[NB], lds_addr at_a, lds_addr at_b, auto second,
                          auto pieces, auto piece) {
      constexpr int HALF = decltype(second)::value, PIECES = decltype(pieces)::value;
      const lds_addr pa = SA::half_of(at_a + lane_a, HALF), pb = SB::half_of(at_b + lane_b, HALF);
      for_each<MB>([&](auto slot) {
        constexpr int i = decltype(slot)::value;
#pragma unroll
        for (int r = 0; r < PER_SLOT; ++r) {
          const int o = i * PER_SLOT + r;
          if (o < NB) rb[o] = SB::operand(pb, o, HALF);
          else if (o < OPERANDS) ra[o - NB] = SA::operand(pa, o - NB, HALF);
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = mma16(xb[j], xa[i], acc[i][j]);
        constexpr int FIRST = i * PIECES / MB, COUNT = (i + 1) * PIECES / MB - FIRST;
        for_each<COUNT>([&](auto p) { piece(Int<FIRST + decltype(p)::value>{}); });
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    {
      const lds_addr pa = SA::half_of(a0 + lane_a, 0), pb = SB::half_of(b0 + lane_b, 0);
#pragma unroll
      for (int j = 0; j < NB; ++j) fb[0][j] = SB::operand(pb, j, 0);
#pragma unroll
      for (int i = 0; i < MB; ++i) fa[0][i] = SA::operand(pa, i, 0);
    }
    int t = begin;
    auto step = [&](auto copies) {   // copies: whether there is a stage t + 2
      constexpr int C = decltype(copies)::value;
      if constexpr (C) begin_a(t + 2, a2);
      __builtin_amdgcn_sched_barrier(0);
      half_stage(fa[1], fb[1], fa[0], fb[0], a0, b0, Int<1>{}, Int<C * PA>{}, piece_a);
      if constexpr (C) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(PA) : "memory");
      else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      landed(t + 1, a1, b1);   // (behind the last stage: clears what nobody reads)
      __syncthreads();
      if constexpr (C) begin_b(t + 2, b0);
      __builtin_amdgcn_sched_barrier(0);
      half_stage(fa[0], fb[0], fa[1], fb[1], a1, b1, Int<0>{}, Int<C * PB>{}, piece_b);   // (behind the last stage: reads that nothing uses)
      const lds_addr was_a = a0, was_b = b0;
      a0 = a1;
      a1 = a2;
      a2 = was_a;
      b0 = b1;
      b1 = was_b;
      ++t;
    };
    while (t + 2 < end) step(Int<1>{});
    while (t < end) step(Int<0>{});
    __syncthreads();
  }

  // The same for operands of three planes and tiles small enough that LDS holds all planes of two stages: each is copied once for the six products, and read
  // once into registers.  A call of few tiles is a chain of stages, of which there are then a sixth: scores of 256 rows of 256 elements over 5003 tokens 15.1 -> 11.2 us,
  // loss of 64 rows of 4096 over 30000, which reads 740 MB of planes, 865 -> 570.  Eight waves of 32 x 32, two to a SIMD, so that one's reads pass under the other's
  // products: 1.35 us per stage, four of 64 x 32 1.5.
  static constexpr int PLANES_LDS_BYTES = 2 * 3 * (SA::BYTES + SB::BYTES);
  S1F_DEV static void run_planes(f32x4 (&acc)[MB][NB], const Matrix &a, const Matrix &b, int64_t m0, int64_t m_limit, int64_t n0, int64_t n_limit,
                                 int64_t k, lds_addr lds) {
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    SA sa;
    SB sb;
    sa.init(a.data, a.ld, m0, m_limit, 0, 0, wave, lane);
    sb.init(b.data, b.ld, n0, n_limit, 0, 0, wave, lane);
    const int stages = (int)((k + kDepth - 1) / kDepth), left = (int)((k - 1) % kDepth) + 1;
    constexpr int COPIES = 3 * (SA::PER_WAVE + SB::PER_WAVE);
    auto copy_side = [&](auto &side, const Matrix &m, lds_addr at, int bytes) {
      for_each<3>([&](auto plane) {
        constexpr int p = decltype(plane)::value;
        const char *from = uniform_pointer(side.next + p * m.plane * 2);
        const unsigned to = __builtin_amdgcn_readfirstlane(at + (unsigned)(p * bytes + wave * side.PER_WAVE * 1024));
        for_each<std::remove_reference_t<decltype(side)>::PER_WAVE>([&](auto i) { side.template copy<decltype(i)::value>(from, to); });
      });
      side.next += side.step;
    };
    auto copy_stage = [&](int t, lds_addr place) {
      if (t + 1 == stages && left < kDepth) {
        sa.shorten(left, wave, lane);
        sb.shorten(left, wave, lane);
      }
      copy_side(sa, a, place, SA::BYTES);
      copy_side(sb, b, place + 3 * SA::BYTES, SB::BYTES);
    };
    const lds_addr places[2] = {lds, lds + 3 * (SA::BYTES + SB::BYTES)};
    copy_stage(0, places[0]);
    if (stages > 1) copy_stage(1, places[1]);
    const lds_addr lane_a = SA::at(wm * MB, lane), lane_b = SB::at(wn * NB, lane);
    for (int t = 0; t < stages; ++t) {
      const lds_addr at_a = places[t & 1], at_b = at_a + 3 * SA::BYTES;
      if (t + 1 < stages) wait_async_tiles_but_last<COPIES>();
      else wait_async_tiles();
      if (t + 1 == stages && left < kDepth) {
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          sa.clear_tail(at_a + p * SA::BYTES, left, wave, lane);
          sb.clear_tail(at_b + p * SB::BYTES, left, wave, lane);
        }
      }
      __syncthreads();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bf16x8 fa[3][MB], fb[3][NB];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          const lds_addr pa = SA::half_of(at_a + p * SA::BYTES + lane_a, half), pb = SB::half_of(at_b + p * SB::BYTES + lane_b, half);
#pragma unroll
          for (int j = 0; j < NB; ++j) fb[p][j] = SB::operand(pb, j, half);
#pragma unroll
          for (int i = 0; i < MB; ++i) fa[p][i] = SA::operand(pa, i, half);
        }
        for_each<6>([&](auto pair) {   // (as above, smallest products first)
          constexpr int P = decltype(pair)::value, PA = (0x001102 >> (4 * P)) & 3, PB = (0x010120 >> (4 * P)) & 3;
#pragma unroll
          for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = mma16(fb[PB][j], fa[PA][i], acc[i][j]);
        });
      }
      __syncthreads();
      if (t + 2 < stages) copy_stage(t + 2, at_a);
    }
  }

  // The same for tiles of which LDS holds five thirds of a stage: planes 0 and 1 of two stages and planes 2 of one, which arrive under the four products of the others.  stages [begin, end)
  // of k.  128 x 128, eight waves: 2.5 to 3.1 us per stage, where alone on a unit six passes of run take 4.3 and beside another tile 2.7.  What bounds it are the copies, 96 KiB a stage: without the products 2.2
  // to 3.1 us, without the copies 1.8 to 2.4.  (Stages of 32, three of them in LDS and operands read one ahead of the products: the same, half lines of memory cost what the distance gains.)
  static constexpr int TOGETHER_LDS_BYTES = 5 * (SA::BYTES + SB::BYTES);
  S1F_DEV static void run_together(f32x4 (&acc)[MB][NB], const Matrix &a, const Matrix &b, int64_t m0, int64_t m_limit, int64_t n0, int64_t n_limit, int64_t k, int begin, int end,
                                   lds_addr lds, int64_t b_apart = 0) {
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (begin >= end) return;
    SA sa;
    SB sb;
    sa.init(a.data, a.ld, m0, m_limit, 0, begin, wave, lane);
    sb.init(b.data, b.ld, n0, n_limit, b_apart, begin, wave, lane);
    const int left = (int)((k - 1) % kDepth) + 1, ragged = left < kDepth ? (int)((k - 1) / kDepth) : 0x7fffffff;   // first stage that is not whole
    constexpr int BOTH = SA::BYTES + SB::BYTES, COPIES = 2 * (SA::PER_WAVE + SB::PER_WAVE);
    auto copy_plane = [&](const auto &side, const Matrix &m, int plane, lds_addr at) {
      const char *from = uniform_pointer(side.next + plane * m.plane * 2);
      const unsigned to = __builtin_amdgcn_readfirstlane(at + (unsigned)(wave * side.PER_WAVE * 1024));
      for_each<std::remove_reference_t<decltype(side)>::PER_WAVE>([&](auto i) { side.template copy<decltype(i)::value>(from, to); });
    };
    // Places of a stage's planes 0 and 1, each a's and then b's, and behind them of planes 2.
    const lds_addr places[2] = {lds, lds + 2 * BOTH}, at_last = lds + 4 * BOTH;
    auto copy_first = [&](int t, lds_addr at) {
      if (t == ragged) {
        sa.shorten(left, wave, lane);
        sb.shorten(left, wave, lane);
      }
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        copy_plane(sa, a, p, at + p * BOTH);
        copy_plane(sb, b, p, at + p * BOTH + SA::BYTES);
      }
    };
    auto clear_plane = [&](lds_addr at) {
      sa.clear_tail(at, left, wave, lane);
      sb.clear_tail(at + SA::BYTES, left, wave, lane);
    };
    const lds_addr lane_a = SA::at(wm * MB, lane), lane_b = SA::BYTES + SB::at(wn * NB, lane);
    auto read = [&](bf16x8 (&xa)[MB], bf16x8 (&xb)[NB], lds_addr at, int half) {
      const lds_addr pa = SA::half_of(at + lane_a, half), pb = SB::half_of(at + lane_b, half);
#pragma unroll
      for (int j = 0; j < NB; ++j) xb[j] = SB::operand(pb, j, half);
#pragma unroll
      for (int i = 0; i < MB; ++i) xa[i] = SA::operand(pa, i, half);
    };
    auto multiply = [&](const bf16x8 (&xa)[MB], const bf16x8 (&xb)[NB]) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = mma16(xb[j], xa[i], acc[i][j]);
    };
    copy_first(begin, places[0]);
#pragma unroll 1
    for (int t = begin; t < end; ++t) {
      const int in = (t - begin) & 1;
      const lds_addr at = places[in];
      wait_async_tiles();
      if (t >= ragged) {
#pragma unroll
        for (int p = 0; p < 2; ++p) clear_plane(at + p * BOTH);
      }
      __syncthreads();
      copy_plane(sa, a, 2, at_last);
      copy_plane(sb, b, 2, at_last + SA::BYTES);
      if (t + 1 < end) {
        sa.next += sa.step;
        sb.next += sb.step;
        copy_first(t + 1, places[1 - in]);
      }
      bf16x8 fa[2][MB], fb[2][NB];   // planes 0 of either half, for the products with planes 2, too
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bf16x8 ga[MB], gb[NB];
        read(fa[half], fb[half], at, half);
        read(ga, gb, at + BOTH, half);
        multiply(ga, gb);
        multiply(fa[half], gb);
        multiply(ga, fb[half]);
        multiply(fa[half], fb[half]);
      }
      if (t + 1 < end) wait_async_tiles_but_last<COPIES>();
      else wait_async_tiles();
      if (t >= ragged) clear_plane(at_last);
      __syncthreads();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bf16x8 ga[MB], gb[NB];
        read(ga, gb, at_last, half);
        multiply(ga, fb[half]);
        multiply(fa[half], gb);
      }
    }
    __syncthreads();
  }

  // The same with B as it lies in fp32 memory, on any element: a weight that few rows are multiplied with is read once, 4 bytes an element, where laying out planes moves 16.  A
  // lane loads the chunks that it would have copied, two stages ahead, and puts their planes where the copies would have gone.  b_ld in fp32 elements; n_limit: rows (columns) that B has; stages
  // [begin, end) of k.  One barrier per stage: behind it nobody reads the other place any more.
  S1F_DEV static void run_raw(f32x4 (&acc)[MB][NB], const Matrix &a, const float *b, int64_t b_ld, int64_t m0, int64_t m_limit, int64_t n0, int64_t n_limit, int64_t k, int begin,
                              int end, lds_addr lds, int64_t b_apart = 0) {
    typedef float Loose4 __attribute__((ext_vector_type(4), aligned(4)));
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (begin >= end) return;
    SA sa;
    sa.init(a.data, a.ld, m0, m_limit, 0, begin, wave, lane);
    const int stages = (int)((k + kDepth - 1) / kDepth), left = (int)((k - 1) % kDepth) + 1;
    constexpr int PB = SB::PER_WAVE;
    const float *from[PB];
    int there[PB], row[PB];   // columns that there are from the chunk on (rows: its first place in the contraction), and its row
    const int64_t step = TRB ? kDepth * b_ld : kDepth;
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      int r, c;
      SB::slot(wave * PB + i, lane, r, c);
      row[i] = r;
      if constexpr (TRB) {
        there[i] = (int)(n_limit - n0) - 8 * c;
        from[i] = b + n0 + 8 * c + (begin * (int64_t)kDepth + r) * b_ld;
      } else {
        there[i] = 8 * c;
        const int second = b_apart ? (r >> 4) & 1 : 0;
        if (b_apart) r = (r >> 5 << 4) + (r & 15);
        if (n0 + r >= n_limit) r = (int)(n_limit - 1 - n0);
        from[i] = b + (n0 + r + (second ? b_apart : 0)) * b_ld + 8 * c + begin * (int64_t)kDepth;
      }
    }
    const bool edge = TRB && n0 + BN > n_limit;
    const int ragged = left < kDepth ? stages - 1 : stages;   // first stage that is not whole
    f32x4 raw[2][PB][2];
    // (fences: the compiler counts neither the copies nor where its loads lie among them; see the wait)
    auto load = [&](f32x4 (&v)[PB][2], int t) {
      asm volatile("" ::: "memory");
      if (!edge && t < ragged) {
#pragma unroll
        for (int i = 0; i < PB; ++i) {
          v[i][0] = *reinterpret_cast<const Loose4 *>(from[i]);
          v[i][1] = *reinterpret_cast<const Loose4 *>(from[i] + 4);
        }
      } else {
        const int rows_left = t < ragged ? kDepth : left;
#pragma unroll
        for (int i = 0; i < PB; ++i) {
          const int n = TRB ? (row[i] < rows_left ? there[i] : 0) : rows_left - there[i];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[i][e / 4][e % 4] = e < n ? from[i][e] : 0.f;
        }
      }
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < PB; ++i) from[i] += step;
    };
    auto put = [&](const f32x4 (&v)[PB][2], lds_addr at_b) {
#pragma unroll
      for (int i = 0; i < PB; ++i) {
        const Planes q = split3(v[i][0], v[i][1]);
#pragma unroll
        for (int p = 0; p < 3; ++p)
          *reinterpret_cast<__attribute__((address_space(3))) bf16x8 *>((uintptr_t)(at_b + (unsigned)(p * SB::BYTES + (wave * PB + i) * 1024 + 16 * lane))) = q.p[p];
      }
    };
    auto copy_a = [&](int t, lds_addr at_a) {
      if (t == ragged) sa.shorten(left, wave, lane);
      for_each<3>([&](auto plane) {
        constexpr int p = decltype(plane)::value;
        const char *at = uniform_pointer(sa.next + p * a.plane * 2);
        const unsigned to = __builtin_amdgcn_readfirstlane(at_a + (unsigned)(p * SA::BYTES + wave * SA::PER_WAVE * 1024));
        for_each<SA::PER_WAVE>([&](auto i) { sa.template copy<decltype(i)::value>(at, to); });
      });
      sa.next += sa.step;
    };
    const lds_addr places[2] = {lds, lds + 3 * (SA::BYTES + SB::BYTES)};
    const lds_addr lane_a = SA::at(wm * MB, lane), lane_b = SB::at(wn * NB, lane);
    load(raw[0], begin);
    if (begin + 1 < end) load(raw[1], begin + 1);
    put(raw[0], places[0] + 3 * SA::BYTES);
    copy_a(begin, places[0]);
    if (begin + 2 < end) load(raw[0], begin + 2);
    auto stage = [&](int t, auto parity) {
      constexpr int Q = decltype(parity)::value;
      const lds_addr at_a = places[Q], at_b = at_a + 3 * SA::BYTES;
      // the copies of A's stage t, behind which only the loads of stage t + 2 have been issued: 2 PB of them, if they are whole
      if (t + 2 < end && t + 2 < ragged && !edge) wait_async_tiles_but_last<2 * PB>();
      else wait_async_tiles();
      if (t >= ragged) {
#pragma unroll
        for (int p = 0; p < 3; ++p) sa.clear_tail(at_a + p * SA::BYTES, left, wave, lane);
      }
      __syncthreads();
      if (t + 1 < end) {
        put(raw[1 - Q], places[1 - Q] + 3 * SA::BYTES);   // (before the copies: the wait for its loads counts from their end)
        copy_a(t + 1, places[1 - Q]);
        if (t + 3 < end) load(raw[1 - Q], t + 3);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bf16x8 fa[3][MB], fb[3][NB];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          const lds_addr pa = SA::half_of(at_a + p * SA::BYTES + lane_a, half), pb = SB::half_of(at_b + p * SB::BYTES + lane_b, half);
#pragma unroll
          for (int j = 0; j < NB; ++j) fb[p][j] = SB::operand(pb, j, half);
#pragma unroll
          for (int i = 0; i < MB; ++i) fa[p][i] = SA::operand(pa, i, half);
        }
        for_each<6>([&](auto pair) {   // (as above, smallest products first)
          constexpr int P = decltype(pair)::value, PA = (0x001102 >> (4 * P)) & 3, PBB = (0x010120 >> (4 * P)) & 3;
#pragma unroll
          for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = mma16(fb[PBB][j], fa[PA][i], acc[i][j]);
        });
      }
    };
#pragma unroll 1
    for (int t = begin; t < end; t += 2) {
      stage(t, Int<0>{});
      if (t + 1 < end) stage(t + 1, Int<1>{});
    }
    __syncthreads();
  }
};

}  // namespace s1f
