// Matrix products of the token loss (gfx950): C[m][n] = sum over k of A(m, k) * B(n, k), both operands bf16, sums fp32.
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
#pragma once
#include "attn_tile.hpp"

namespace s1f {

constexpr int kDepth = 64;   // contraction per stage

// R: rows of C (or columns of C, for the other operand) in the tile; TR: stored by columns; NW: waves that copy.
template <int R, bool TR, int NW> struct Side {
  static constexpr int BYTES = R * kDepth * 2, PIECES = BYTES / 1024, PER_WAVE = PIECES / NW;
  static_assert(PIECES % NW == 0 && PER_WAVE <= 4, "pieces of a wave share one M0");
  static constexpr int ROW = TR ? 2 * R : 128, CHUNKS = ROW / 16, RPP = 1024 / ROW;   // bytes and chunks of a row, rows per piece
  S1F_DEV static int h(int k) { return R >= 128 ? (k & 3) | ((k >> 3) & 1) << 2 : ((k >> 1) & 1) | ((k >> 3) & 1) << 1; }

  const char *base;         // of the stage that is copied next (uniform)
  int64_t step;             // bytes to the next stage
  unsigned voff[PER_WAVE];  // of the lane's chunk in each of the wave's pieces
  int row_bytes;

  // The lane's slot in piece p: row within the stage's image and chunk of that row.
  S1F_DEV static void slot(int p, int lane, int &row, int &chunk) {
    row = p * RPP + lane / CHUNKS;
    const int c = lane % CHUNKS;
    chunk = TR ? ((((c >> 1) ^ h(row)) << 1) | (c & 1)) : (c ^ ((row >> 1) & 7));
  }
  // m0: first row (column) of the tile; limit: rows (columns) that there are; those behind are copies of the last (columns: first)
  S1F_DEV void init(const bf16_t *data, int64_t ld, int64_t m0, int64_t limit, int wave, int lane) {
    row_bytes = (int)(ld * 2);
    base = reinterpret_cast<const char *>(TR ? data + m0 : data + m0 * ld);
    step = TR ? kDepth * ld * 2 : kDepth * 2;
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      int r, c;
      slot(wave * PER_WAVE + i, lane, r, c);
      if (TR) {
        if (m0 + 8 * c >= limit) c = 0;
      } else {
        if (m0 + r >= limit) r = (int)(limit - 1 - m0);
      }
      voff[i] = (unsigned)(r * row_bytes + 16 * c);
    }
  }
  // Copies a stage to LDS address `dst`.  left: contraction that the operand has from this stage on; where it is less than a stage, what
  // is behind is read from the stage's beginning and overwritten by clear_tail.
  S1F_DEV void issue(const char *from, lds_addr dst, int left, int wave, int lane) const {
    unsigned off[PER_WAVE];
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) off[i] = voff[i];
    if (left < kDepth) {
#pragma unroll
      for (int i = 0; i < PER_WAVE; ++i) {
        int r, c;
        slot(wave * PER_WAVE + i, lane, r, c);
        if (TR) {
          if (r >= left) off[i] -= (unsigned)(r * row_bytes);
        } else {
          if (8 * c >= left) off[i] -= (unsigned)(16 * c);
        }
      }
    }
    const uint64_t bits = reinterpret_cast<uint64_t>(from);
    const char *b = reinterpret_cast<const char *>(
        ((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(bits >> 32)) << 32) |
        (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)bits));
    const unsigned to = __builtin_amdgcn_readfirstlane(dst + (unsigned)(wave * PER_WAVE * 1024));
    if constexpr (PER_WAVE == 4)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\t"
                   "global_load_lds_dwordx4 %2, %6 offset:1024\n\t"
                   "global_load_lds_dwordx4 %3, %7 offset:2048\n\t"
                   "global_load_lds_dwordx4 %4, %8 offset:3072"
                   : : "s"(to), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(b), "s"(b - 1024), "s"(b - 2048), "s"(b - 3072)
                   : "m0");
    else if constexpr (PER_WAVE == 2)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
                   "global_load_lds_dwordx4 %2, %4 offset:1024"
                   : : "s"(to), "v"(off[0]), "v"(off[1]), "s"(b), "s"(b - 1024) : "m0");
    else {
      static_assert(PER_WAVE == 1, "one, two or four pieces");
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(off[0]), "s"(b) : "m0");
    }
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
  struct At {
    lds_addr a;
  };
  S1F_DEV static At at(lds_addr stage, int lane) {
    const int n = lane & 15, j = lane >> 4;
    if constexpr (TR) {
      const int k = 8 * j + (n >> 2);
      return At{opaque(stage + (unsigned)(k * ROW + h(k) * 32 + (n & 3) * 8))};
    } else {
      return At{opaque(stage + (unsigned)(n * 128 + 16 * (j ^ ((n >> 1) & 7))))};
    }
  }
  S1F_DEV static bf16x8 operand(At x, int block, int half) {
    if constexpr (TR) {
      const lds_addr p = (x.a ^ (unsigned)((block * 32) & (ROW - 1))) + (unsigned)(half * 32 * ROW);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4 *>((uintptr_t)p));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          reinterpret_cast<__attribute__((address_space(3))) s16x4 *>((uintptr_t)(p + (unsigned)(4 * ROW))));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      s16x8 r = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf16x8, r);
    } else {
      return lds_load<bf16x8>((x.a ^ (unsigned)(half * 64)) + (unsigned)(block * 2048));
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
template <int BM, int BN, int WM, int WN, bool TRA, bool TRB> struct Product {
  static constexpr int NW = WM * WN, THREADS = 64 * NW, MB = BM / WM / 16, NB = BN / WN / 16;
  typedef Side<BM, TRA, NW> SA;
  typedef Side<BN, TRB, NW> SB;
  static constexpr int STAGE = SA::BYTES + SB::BYTES, LDS_BYTES = 2 * STAGE;

  // k: contraction of one product of planes; stages [begin, end) of all of them, counted k-stage by k-stage, plane by plane within
  S1F_DEV static void run(f32x4 (&acc)[MB][NB], const Matrix &a, const Matrix &b, int64_t m0, int64_t m_limit, int64_t n0, int64_t n_limit,
                          int64_t k, int pairs, int begin, int end, lds_addr lds) {
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    SA sa;
    SB sb;
    sa.init(a.data, a.ld, m0, m_limit, wave, lane);
    sb.init(b.data, b.ld, n0, n_limit, wave, lane);
    int pair = begin % pairs;                      // of the stage that is copied next
    int kt = begin / pairs;
    // copies the next stage to `dst`
    auto issue = [&](lds_addr dst) {
      // (2,0) (0,2) (1,1) (1,0) (0,1) (0,0): smallest products first
      const int of_a = pairs == 1 ? 0 : (int)((0x001102u >> (4 * pair)) & 3u), of_b = pairs == 1 ? 0 : (int)((0x010120u >> (4 * pair)) & 3u);
      const int64_t rest = k - (int64_t)kt * kDepth;
      const int left = rest < kDepth ? (int)rest : kDepth;
      sa.issue(sa.base + kt * sa.step + of_a * a.plane * 2, dst, left, wave, lane);
      sb.issue(sb.base + kt * sb.step + of_b * b.plane * 2, dst + SA::BYTES, left, wave, lane);
      if (++pair == pairs) {
        pair = 0;
        ++kt;
      }
    };
    // contraction left from stage t on
    auto left_at = [&](int t) -> int {
      const int64_t rest = k - (int64_t)(t / pairs) * kDepth;
      return rest < kDepth ? (int)rest : kDepth;
    };
    auto landed = [&](lds_addr at, int t) {        // this wave's copies of stage t are there
      const int left = left_at(t);
      if (left < kDepth) {
        sa.clear_tail(at, left, wave, lane);
        sb.clear_tail(at + SA::BYTES, left, wave, lane);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    };
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (begin >= end) return;
    lds_addr cur = lds, next = lds + STAGE;
    issue(cur);
    if (begin + 1 < end) issue(next);
    for (int t = begin; t < end; ++t) {
      if (t + 1 < end) wait_async_tiles_but_last<SA::PER_WAVE + SB::PER_WAVE>();
      else wait_async_tiles();
      landed(cur, t);
      __syncthreads();
      const typename SA::At xa = SA::at(cur, lane);
      const typename SB::At xb = SB::at(cur + SA::BYTES, lane);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bf16x8 fa[MB], fb[NB];
#pragma unroll
        for (int i = 0; i < MB; ++i) fa[i] = SA::operand(xa, wm * MB + i, half);
#pragma unroll
        for (int j = 0; j < NB; ++j) fb[j] = SB::operand(xb, wn * NB + j, half);
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[i][j] = mma16(fb[j], fa[i], acc[i][j]);
      }
      __syncthreads();
      if (t + 2 < end) issue(cur);
      const lds_addr was = cur;
      cur = next;
      next = was;
    }
  }
};

}  // namespace s1f
