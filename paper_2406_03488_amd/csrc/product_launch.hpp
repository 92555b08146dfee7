// What the products of loss_tile.hpp need around them: fp32 operands as planes, the order of tiles, which tiles a launch takes, and the launch.
#pragma once
#include <algorithm>
#include <atomic>

#include "loss_tile.hpp"
#include "rows.hpp"

namespace s1f {

// Planes of fp32 operands, of the largest ones too: past the largest bf16 number the first plane is that number, which rounding would take to infinity, and
// the others have what is left, exactly.  A mask of the type's lowest value has planes, then, and takes no part in a gradient as zero times it is zero.  The planes
// of infinities and NaN are such: see scores_plain.
S1F_DEV Planes planes_of(f32x4 lo, f32x4 hi) {
  constexpr float kMost = 0x1.fep127f;
  f32x4 l, h;
  bool all = true;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    l[e] = __builtin_amdgcn_fmed3f(lo[e], -kMost, kMost);
    h[e] = __builtin_amdgcn_fmed3f(hi[e], -kMost, kMost);
    all = all && l[e] == lo[e] && h[e] == hi[e];
  }
  Planes p = split3(l, h);
  if (!all) {
    const Planes rest = split3(lo - l, hi - h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = e < 4 ? lo[e] : hi[e - 4], c = e < 4 ? l[e] : h[e - 4];
      if (x == c) continue;
      p.p[1][e] = rest.p[0][e];
      p.p[2][e] = rest.p[1][e];
    }
  }
  return p;
}
// Eight elements of a row as the products read them: bf16, zeros behind `hidden`; fp32 ones as three planes, `plane` elements apart.  (Planes not
// 2^16 times as large, see kUp: the largest floats would have none, and what lies below 2^-110 is nothing beside a row's other scores; to gradients of nothing but
// such elements it leaves 8 bits.)
template <typename T, bool WIDE> S1F_DEV void pack_eight(const T *from, int hidden, int c, bf16_t *to, int64_t plane) {
  typedef Piece<T, WIDE> P;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; i += P::N) {
    typename P::Values p;
    P::load(from + 8 * c + i, hidden - 8 * c - i, p);
#pragma unroll
    for (int e = 0; e < P::N; ++e) v[i + e] = p[e];
  }
  if constexpr (sizeof(T) == 4) {
    const Planes p = planes_of(f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]});
#pragma unroll
    for (int i = 0; i < 3; ++i) *reinterpret_cast<bf16x8 *>(to + i * plane) = p.p[i];
  } else {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (bf16_t)v[e];
    *reinterpret_cast<bf16x8 *>(to) = o;
  }
}
// Number of a tile -> its place.  The hardware hands workgroups to the 8 XCDs in turn; each takes consecutive tiles, in blocks of four columns of tiles
// walked down the rows, so that the 32 workgroups that an XCD runs side by side share eight row and four column panels in its L2.
S1F_DEV void decode_tile(int tiles_m, int tiles_n, int tile, int &tm, int &tn) {
  const int per = tiles_m * tiles_n >> 3;
  if (tile < per * 8) tile = (tile & 7) * per + (tile >> 3);
  const int group = tile / (4 * tiles_m), in = tile - group * 4 * tiles_m, left = tiles_n - 4 * group;
  if (left >= 4) {
    tm = in >> 2;
    tn = 4 * group + (in & 3);
  } else {
    tm = in / left;
    tn = 4 * group + in % left;
  }
}
// The number of the tile at a place.
S1F_DEV int encode_tile(int tiles_m, int tiles_n, int tm, int tn) {
  const int per = tiles_m * tiles_n >> 3, group = tn >> 2, left = tiles_n - 4 * group;
  const int tile = 4 * group * tiles_m + tm * (left < 4 ? left : 4) + (tn & 3);
  return tile < per * 8 ? (tile % per) * 8 + tile / per : tile;
}
inline int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// Tiles of 256 x 256 (eight waves, one workgroup to a compute unit), 128 x 128 (four, two to a unit) or 64 x 128 (four, two to a unit; scores in fp32: eight, one to
// a unit, see run_planes).
enum Tile { kBig, kMiddle, kLow };
constexpr int kUnits = 256;   // compute units

// Predicted microseconds of a launch of tiles of so many stages of products, from launches of 1 to 4099 rows over 800 to 50021 tokens with 256 to 4096
// elements: a tile's beginning and end, and its stages: alone on a compute unit, or beside another one.  Rounds of big tiles count whole, those of
// the others overlap.  (fp32 scores in 64 x 128 tiles take less, 5.5 us and 0.23 per stage a round, but are priced like the others.)  Measured for 28 forwards of 1 to 4099 rows of 64 to
// 4096 elements over 4000 to 130000 tokens, of either type, each cut in all ways: in 22 the choice is within 2 % of the best, in 26 within 5 %; farthest 4099 x 256 bf16 over 20000, 79.4 us, in middle
// tiles 73.1.  fp32, 256 x 1024 over 5003: low tiles 42.6 us, middle 64.5, big 126; 300 x 1280 over 20011: middle 149, low 166, big 190; 1000 x 1024 over 10007: big 137, middle 147, low 152.
inline double tiles_us(Tile tile, int64_t tiles, double stages) {
  if (tile == kBig) return (double)((tiles + kUnits - 1) / kUnits) * (8.0 + 1.45 * stages);
  if (tiles <= kUnits) return tile == kMiddle ? 5.0 + 0.55 * stages : 4.5 + 0.40 * stages;
  const double rounds = std::max(1.0, (double)tiles / (2 * kUnits) + 0.25);
  return rounds * (tile == kMiddle ? 6.0 + 0.90 * stages : 5.0 + 0.60 * stages);
}
inline int64_t grid_of(int64_t m, int64_t n, int bm, int bn) { return (m + bm - 1) / bm * ((n + bn - 1) / bn); }

// How the tiles of a product [m, n] are taken: big ones up to `whole`, their rest in quarters (the last round of big tiles may be one of a few: forward of
// 4099 rows over 50021 tokens, 3332 tiles); or all in one of the other sizes.
struct Cut {
  Tile tile;
  int64_t whole;
};
inline Cut cut_for(int64_t m, int64_t n, int64_t stages, bool low) {
  const int64_t big = grid_of(m, n, 256, 256), rounds = big / kUnits * kUnits;
  Cut best = {kBig, big};
  double least = tiles_us(kBig, big, (double)stages);
  auto offer = [&](Cut c, double us) {
    if (us < least) {
      least = us;
      best = c;
    }
  };
  if (rounds > 0 && rounds < big) offer({kBig, rounds}, tiles_us(kBig, rounds, (double)stages) + 3.0 + tiles_us(kMiddle, 4 * (big - rounds), (double)stages));
  offer({kMiddle, 0}, tiles_us(kMiddle, grid_of(m, n, 128, 128), (double)stages));
  if (low) offer({kLow, 0}, tiles_us(kLow, grid_of(m, n, 64, 128), (double)stages));
  return best;
}
// dx: the big tiles behind the last full round, or all middle tiles, cut into parts along the vocabulary, each of which but the first
// is written and read once more (4 TB/s).
struct DxCut {
  Tile tile;
  int64_t whole, rest;
  int splits, most_splits;   // (the most if fewer rows count)
};
inline DxCut dx_cut_for(int64_t m, int64_t n, int64_t stages) {
  DxCut best = {};
  double least = 1e30;
  for (Tile tile : {kBig, kMiddle}) {
    const int side = tile == kBig ? 256 : 128;
    const int64_t tiles = grid_of(m, n, side, side), whole = tile == kBig ? tiles / kUnits * kUnits : 0, rest = tiles - whole;
    for (int splits = 1; splits <= 32 && (splits == 1 || (rest > 0 && stages / splits >= 4 && rest * splits <= 4 * kUnits)); ++splits) {
      const double us = (whole ? tiles_us(tile, whole, (double)stages) : 0.0) + (rest ? tiles_us(tile, rest * splits, (double)stages / splits) : 0.0) +
                        (double)(splits - 1) * rest * side * side * 8 / 4e6;
      if (us < 0.98 * least) {
        least = us;
        best = {tile, whole, rest, splits, (int)std::max<int64_t>(splits, std::min<int64_t>(64, stages / 4))};
      }
    }
  }
  return best;
}

template <Tile TILE> struct TileShape {
  static constexpr int BM = TILE == kBig ? 256 : TILE == kMiddle ? 128 : 64, BN = TILE == kBig ? 256 : 128, WM = TILE == kLow ? 1 : 2,
                       WN = TILE == kMiddle ? 2 : 4;
};

// Kernels that use more than 64 KiB of LDS are told so once per device.
template <auto KERNEL, typename ARGS> int launch_tiles(int lds, int threads, int64_t grid, const ARGS &a, hipStream_t st) {
  static std::atomic<bool> told[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return S1F_EDEVICE;
  const bool known = dev >= 0 && dev < 64;
  if (!known || !told[dev].load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return S1F_EDEVICE;
    if (known) told[dev].store(true, std::memory_order_release);
  }
  return launch_rows_kernel(KERNEL, grid, threads, a, st, lds);
}

}  // namespace s1f
