// Rows of hidden states out of tokens, and the gradient of the table they come from: what the first stage of a pipeline does with a
// segment before its first layer and behind the backward pass of it.
//
//   forward    out[r] = scale * table[id[r]]
//   backward   acc[t] += scale * sum of dout[r] over the rows r with id[r] = t
//
// The forward moves data only.  The backward sums without atomics, in one order whatever the launch: rows are sorted by (token, row), the
// sorted list is cut into chunks of equal length, however often a token occurs, and a workgroup sums the runs of equal tokens in its
// chunk.  A run inside one chunk goes straight into the accumulators; a longer one leaves a partial sum for each chunk, which
// a last kernel adds up in their order.
#include "rows.hpp"

namespace s1f {
namespace {

struct EmbedArgs {
  const int64_t *ids;
  int64_t ids_sb;
  const void *table, *dout;
  int64_t table_stride;
  void *out;
  float *acc;
  int64_t acc_stride;
  RowsOf y;
  int32_t n, hidden, vocab, pieces;     // rows of all batch entries; pieces of a row
  int32_t tpr_log2, chunk, part_ld;     // threads that share a row; sorted rows per chunk of the sums; row length of their partial sums
  float scale;
  // workspace of the backward
  int32_t *row_of, *key_of;             // rows sorted by token, and their tokens (`vocab`: none)
  int32_t *row_from, *key_from, *count; // input of a sorting pass; rows of each tile with each digit
  int32_t *long_runs;                   // number of runs that go on behind a chunk, and the chunks where they start
  float *head, *tail;                   // [chunk][part_ld]: sum of the run that reaches into the chunk, that leaves it
  int32_t tiles, shift, bits, first_pass, scanned;
};

S1F_DEV int key_at(const EmbedArgs &a, int row) {
  int b, r;
  div_mod(row, a.y.by_rows, b, r);
  const int64_t id = a.ids[b * a.ids_sb + r];
  return id >= 0 && id < a.vocab ? (int)id : a.vocab;
}

// 2^tpr_log2 threads per row, each of which takes every 2^tpr_log2-th piece.  Bound by memory: 4897 rows of 7168 bf16 elements, 136 MB with a table row read for
// each, 19 us, of which the caches serve some; 16 rows of 256 fp32 elements 2 us, a chain of two loads and a store.
template <typename T, bool WIDE> __global__ void __launch_bounds__(256) embed_fwd_kernel(const EmbedArgs a) {
  typedef Piece<T, WIDE> P;
  const int row = (blockIdx.x << (8 - a.tpr_log2)) + (threadIdx.x >> a.tpr_log2);
  if (row >= a.n) return;
  const int key = key_at(a, row), step = 1 << a.tpr_log2;
  const T *from = reinterpret_cast<const T *>(a.table) + (key < a.vocab ? key : 0) * a.table_stride;
  T *to = reinterpret_cast<T *>(a.out) + a.y.offset(row);
  for (int p = threadIdx.x & (step - 1); p < a.pieces; p += step) {
    const int left = a.hidden - p * P::N;
    typename P::Values v;
    P::load(from + p * P::N, left, v);
#pragma unroll
    for (int e = 0; e < P::N; ++e) v[e] = key < a.vocab ? v[e] * a.scale : 0.f;
    P::store(to + p * P::N, left, v);
  }
}

// Rows sorted by token by counting, for every row, the rows in front of it: n^2 comparisons, of 64 by one vector instruction, whose
// result a scalar one counts.  A workgroup of 16 waves places 32 rows, two to a wave, out of all tokens in LDS: 5.8 us for 2714 rows (each wave reading them
// from memory as it went 12, a chain of loads), 12 for 8192, 26 for 12000, 34 for 16384, where two sorting passes take 33.
constexpr int32_t kMostRanked = 12288;    // rows up to which counting sorts them
constexpr int kRanked = 32;               // rows per workgroup
__global__ void __launch_bounds__(1024) embed_rank_kernel(const EmbedArgs a) {
  extern __shared__ int tokens[];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first = blockIdx.x * kRanked, blocks = (a.n + 63) >> 6;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.long_runs = 0;
  for (int i = threadIdx.x; i < 64 * blocks; i += 1024) tokens[i] = i < a.n ? key_at(a, i) : 0x7fffffff;
  __syncthreads();
  constexpr int R = kRanked / 16;
  int key[R], before[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    key[i] = __builtin_amdgcn_readfirstlane(tokens[first + R * wave + i]);
    before[i] = 0;
  }
  const int here = first >> 6;
  // rows in front with the same token count, those behind do not
  auto count = [&](int begin, int end, int equal) {
#pragma unroll 4
    for (int c = begin; c < end; ++c) {
      const int x = tokens[64 * c + lane];
#pragma unroll
      for (int i = 0; i < R; ++i) before[i] += __builtin_popcountll(__ballot(x < key[i] + equal));
    }
  };
  count(0, here, 1);
  count(here + 1, blocks, 0);
  const int x = tokens[64 * here + lane];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = first + R * wave + i;
    before[i] += __builtin_popcountll(__ballot(x < key[i] || (x == key[i] && 64 * here + lane < row)));
    if (lane == i && row < a.n) {
      a.row_of[before[i]] = row;
      a.key_of[before[i]] = key[i];
    }
  }
}

// Sorting in passes over digits of at most 9 bits, the lowest first, each of which keeps the order of equal digits: count the digits of
// every tile of 1024 rows, sum the counts of each digit up over the tiles, and place the rows.  Bound by latency: of 32768 rows a pass counts for 4.6 us and
// places for 8.8, with one workgroup to a tile.
constexpr int kTile = 1024, kDigits = 512, kMostSummed = 64;   // (the last: tiles whose counts the placing workgroups sum up)

S1F_DEV int pass_key(const EmbedArgs &a, int i) { return a.first_pass ? key_at(a, i) : a.key_from[i]; }

__global__ void __launch_bounds__(256) embed_count_kernel(const EmbedArgs a) {
  __shared__ int counts[kDigits];
  const int digits = 1 << a.bits;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.long_runs = 0;
  for (int d = threadIdx.x; d < digits; d += 256) counts[d] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kTile / 256; ++u) {
    const int i = blockIdx.x * kTile + 256 * u + threadIdx.x;
    if (i < a.n) atomicAdd(&counts[(pass_key(a, i) >> a.shift) & (digits - 1)], 1);   // (whole numbers: the same in any order)
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += 256) a.count[a.scanned ? d * a.tiles + blockIdx.x : blockIdx.x * digits + d] = counts[d];
}

// Of many tiles: exclusive sums over the tiles of one digit per wave; their total behind them.
__global__ void __launch_bounds__(256) embed_scan_kernel(const EmbedArgs a) {
  const int lane = threadIdx.x & 63, digit = blockIdx.x * 4 + (threadIdx.x >> 6), digits = 1 << a.bits;
  if (digit >= digits) return;
  int *count = a.count + digit * a.tiles, carry = 0;
  for (int at = 0; at < a.tiles; at += 64) {
    const int own = at + lane < a.tiles ? count[at + lane] : 0;
    int x = own;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int y = __shfl_up(x, s);
      if (lane >= s) x += y;
    }
    if (at + lane < a.tiles) count[at + lane] = carry + x - own;
    carry += __shfl(x, 63);
  }
  if (lane == 0) a.count[digits * a.tiles + digit] = carry;
}

// A wave places 256 rows of the tile, 64 at a time.  Of few tiles every workgroup sums the counts up itself: a launch of 5 us less per pass.  next[wave][digit]: where its next row with that digit goes.
__global__ void __launch_bounds__(256) embed_place_kernel(const EmbedArgs a) {
  __shared__ int next[4][kDigits], of_wave[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, digits = 1 << a.bits;
  for (int d = threadIdx.x; d < 4 * kDigits; d += 256) (&next[0][0])[d] = 0;
  __syncthreads();
  constexpr int U = kTile / 256;
  int key[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = blockIdx.x * kTile + 256 * wave + 64 * u + lane;
    key[u] = i < a.n ? pass_key(a, i) : 0;
    if (i < a.n) atomicAdd(&next[wave][(key[u] >> a.shift) & (digits - 1)], 1);
  }
  __syncthreads();
  // rows with smaller digits (2 digits per thread), with this digit in tiles in front, in waves in front
  int total[2], in_front[2], own = 0;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int d = 2 * threadIdx.x + e;
    total[e] = in_front[e] = 0;
    if (d < digits && a.scanned) {
      total[e] = a.count[digits * a.tiles + d];
      in_front[e] = a.count[d * a.tiles + blockIdx.x];
    } else if (d < digits) {
#pragma unroll 8
      for (int t = 0; t < a.tiles; ++t) {
        const int c = a.count[t * digits + d];
        total[e] += c;
        in_front[e] += t < (int)blockIdx.x ? c : 0;
      }
    }
    own += total[e];
  }
  int x = own;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const int y = __shfl_up(x, s);
    if (lane >= s) x += y;
  }
  if (lane == 63) of_wave[wave] = x;
  __syncthreads();
  int before = x - own;
  for (int w = 0; w < wave; ++w) before += of_wave[w];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int d = 2 * threadIdx.x + e;
    if (d < digits) {
      int at = before + in_front[e];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int c = next[w][d];
        next[w][d] = at;
        at += c;
      }
    }
    before += total[e];
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = blockIdx.x * kTile + 256 * wave + 64 * u + lane, digit = (key[u] >> a.shift) & (digits - 1);
    const bool is = i < a.n;
    uint64_t same = __ballot(is);
    for (int b = 0; b < a.bits; ++b) {
      const uint64_t ones = __ballot((digit >> b) & 1);
      same &= (digit >> b) & 1 ? ones : ~ones;
    }
    if (is) {
      const int at = *(volatile int *)&next[wave][digit] + __builtin_popcountll(same & ((uint64_t(1) << lane) - 1));
      a.key_of[at] = key[u];
      a.row_of[at] = a.first_pass ? i : a.row_from[i];
      if ((same >> lane) == 1) *(volatile int *)&next[wave][digit] = at + 1;   // the last lane of its digit
    }
  }
}

// Sums of the runs in one chunk of the sorted rows.  2^tpr_log2 threads share the columns of a row; the others of a workgroup take
// other chunks.  Of eight rows at a time everything is asked for together, the accumulators that their runs end in included.  Bound by memory: 32768 rows of 4096
// bf16 elements over 50021 tokens, 646 MB with the accumulators read and written, 142 to 146 us, 4.5 TB/s (a large copy: 4.8).
template <typename T, bool WIDE> __global__ void __launch_bounds__(256) embed_sum_kernel(const EmbedArgs a) {
  typedef Piece<T, WIDE> P;
  const int tpr = 1 << a.tpr_log2;
  const int chunk = (int)(blockIdx.x << (8 - a.tpr_log2)) + (int)(threadIdx.x >> a.tpr_log2);
  const int piece = blockIdx.y * tpr + (threadIdx.x & (tpr - 1));
  const int begin = chunk * a.chunk, end = begin + a.chunk < a.n ? begin + a.chunk : a.n;
  if (begin >= a.n || piece >= a.pieces) return;
  const T *dout = reinterpret_cast<const T *>(a.dout) + piece * P::N;
  const int64_t part = (int64_t)chunk * a.part_ld + piece * P::N;
  const int left = a.hidden - piece * P::N;
  int key = a.key_of[begin];
  bool into = begin > 0 && a.key_of[begin - 1] == key;   // the run reaches into the chunk from the one before
  float sum[P::N];
#pragma unroll
  for (int e = 0; e < P::N; ++e) sum[e] = 0.f;
  constexpr int U = 8;
  for (int i = begin; i < end && key < a.vocab; i += U) {
    int k[U + 1];
    typename P::Values v[U];
    float was[U][P::N];
#pragma unroll
    for (int u = 0; u <= U; ++u) k[u] = i + u < a.n ? a.key_of[i + u] : a.vocab;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = i + u < end ? i + u : end - 1;
      P::load(dout + a.y.offset(a.row_of[at]), left, v[u]);
      if (k[u] != k[u + 1] && k[u] < a.vocab && i + u < end) load_f32<P::N, WIDE>(a.acc + k[u] * a.acc_stride + piece * P::N, left, was[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= end || k[u] >= a.vocab) break;
#pragma unroll
      for (int e = 0; e < P::N; ++e) sum[e] += v[u][e];
      if (k[u] != k[u + 1]) {   // the run ends
        if (into) {
          store_f32<P::N, true>(a.head + part, P::N, sum);
        } else {
#pragma unroll
          for (int e = 0; e < P::N; ++e) was[u][e] += a.scale * sum[e];
          store_f32<P::N, WIDE>(a.acc + k[u] * a.acc_stride + piece * P::N, left, was[u]);
        }
        into = false;
#pragma unroll
        for (int e = 0; e < P::N; ++e) sum[e] = 0.f;
      } else if (i + u + 1 == end) {   // it goes on behind the chunk
        store_f32<P::N, true>((into ? a.head : a.tail) + part, P::N, sum);
        if (!into && piece == 0) a.long_runs[1 + atomicAdd(a.long_runs, 1)] = chunk;
      }
    }
    key = k[U];
  }
}

// Runs longer than a chunk, which the sums have listed by the chunk in which each starts (in any order: no result depends on it).  A workgroup takes 64
// pieces of the columns of one and adds up what it has left there and in the chunks behind, its waves an eighth of them each.  (One thread one after the
// other: 48 us for the 2100 rows of the most frequent of 50021 tokens; a workgroup for every chunk, most of which end at once: 17 to 60.)
template <int N> __global__ void __launch_bounds__(512) embed_join_kernel(const EmbedArgs a) {
  constexpr int SHARES = 8;
  __shared__ __attribute__((aligned(16))) float meet[SHARES][64 * N];
  const int lane = threadIdx.x & 63, share = threadIdx.x >> 6, blocks = (a.pieces + 63) / 64, units = *a.long_runs * blocks;
  for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int chunk = a.long_runs[1 + unit / blocks], piece = unit % blocks * 64 + lane;
    const int key = a.key_of[(chunk + 1) * a.chunk];
    // last chunk that begins within the run: 64 of them are asked at a time
    const int all = (a.n + a.chunk - 1) / a.chunk;
    int last = chunk;
    for (int more = 64; more == 64; last += more) {
      const int c = last + 1 + lane;
      const uint64_t on = __ballot(c < all && a.key_of[(c < all ? c : 0) * a.chunk] == key);
      more = ~on ? __builtin_ctzll(~on) : 64;
    }
    const int chunks = last - chunk, stop = chunk + 1 + chunks * (share + 1) / SHARES;
    const bool is = piece < a.pieces;
    const float *head = a.head + (is ? piece : 0) * N;
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.f;
    constexpr int U = 4;
    for (int c = chunk + 1 + chunks * share / SHARES; c < stop; c += U) {
      float more[U][N];
#pragma unroll
      for (int u = 0; u < U; ++u) load_f32<N, true>(head + (int64_t)(c + u < stop ? c + u : c) * a.part_ld, N, more[u]);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += c + u < stop ? more[u][e] : 0.f;
    }
    __syncthreads();   // (the sums of the unit before have been read)
    store_f32<N, true>(&meet[share][lane * N], N, sum);
    __syncthreads();
    const int col = (unit % blocks) * 64 * N + threadIdx.x;
    static_assert(64 * N <= 64 * SHARES, "a column to a thread");
    if ((int)threadIdx.x < 64 * N && col < a.hidden) {
      float *to = a.acc + key * a.acc_stride + col, total = a.tail[(int64_t)chunk * a.part_ld + col];
      const float was = *to;
#pragma unroll
      for (int w = 0; w < SHARES; ++w) total += meet[w][threadIdx.x];
      *to = was + a.scale * total;
    }
  }
}

constexpr int32_t kMostVocab = 1 << 26;   // three sorting passes

int threads_per_row_log2(int64_t pieces) {
  int t = 3;
  while (t < 8 && (1 << t) < pieces) ++t;
  return t;
}
int check(const s1f_rows *d, int64_t vocab, int64_t stride) {
  const int rc = check_rows(d, false, true);
  if (rc != S1F_OK) return rc;
  if (vocab < 1 || stride < d->hidden) return S1F_EINVAL;
  return vocab > kMostVocab ? S1F_EUNSUPPORTED : S1F_OK;
}
int64_t up(int64_t x) { return (x + 255) / 256 * 256; }
int64_t part_ld_of(const s1f_rows *d) { return (d->hidden + 7) / 8 * 8; }
int32_t pieces_of(const s1f_rows *d) { return (int32_t)((d->hidden + elements_of_16_bytes(d->dtype) - 1) / elements_of_16_bytes(d->dtype)); }
struct EmbedSpace {
  int64_t rows, keys, rows2, keys2, count, long_runs, head, tail, bytes;
};
// Sorted rows per chunk: a chunk is a chain of a few loads, so that few rows take short ones; a long one leaves fewer partial sums.  us of a call with chunks of 8, 16 and 32,
// for 512 fp32 elements over 9973 tokens / 4096 bf16 over 50021 / 1024 bf16 over 2000:
//   4096 rows   18.9 20.3 25.0 /  35  32  36 / 21.0 22.4 27.3       24576 rows  51.1 47.8 50.1 / 159 146 140 / 57.4 49.9 51.7
//   8191        27.6 27.6 32.4 /  58  54  50 / 30.9 30.0 35.7       32767       61.3 53.1 53.2 / 206 189 185 / 65.6 58.6 55.6
//  12288        45.8 45.2 50.3 /  86  82  78 / 50.1 48.0 52.5       49152       75.2 66.5 60.9 / 285 259 254 / 83.5 70.1 62.1
int chunk_of(int64_t n) { return n < 8192 ? 8 : n < 28672 ? 16 : 32; }
EmbedSpace space_of(const s1f_rows *d) {
  const int64_t n = d->batch * d->rows, chunks = (n + chunk_of(n) - 1) / chunk_of(n);
  EmbedSpace s = {};
  int64_t at = 0;
  auto take = [&at](int64_t bytes) { const int64_t was = at; at += up(bytes); return was; };
  s.rows = take(4 * n);
  s.keys = take(4 * n);
  if (n > kMostRanked) {
    s.rows2 = take(4 * n);
    s.keys2 = take(4 * n);
    s.count = take(4 * kDigits * ((n + kTile - 1) / kTile + 1));
  }
  s.long_runs = take(4 * (chunks + 1));
  if (chunks > 1) {
    s.head = take(4 * chunks * part_ld_of(d));
    s.tail = take(4 * chunks * part_ld_of(d));
  }
  s.bytes = at;
  return s;
}

template <typename T> int sums(const EmbedArgs &a, bool wide, hipStream_t st) {
  const int64_t chunks = (a.n + a.chunk - 1) / a.chunk, groups = 256 >> a.tpr_log2;
  const dim3 grid((unsigned)((chunks + groups - 1) / groups), (a.pieces + (1 << a.tpr_log2) - 1) >> a.tpr_log2);
  EmbedArgs args = a;
  void *params[] = {&args};
  const void *sum = wide ? reinterpret_cast<const void *>(&embed_sum_kernel<T, true>) : reinterpret_cast<const void *>(&embed_sum_kernel<T, false>);
  if (hipLaunchKernel(sum, grid, dim3(256), params, 0, st) != hipSuccess) return S1F_EDEVICE;
  if (chunks == 1) return S1F_OK;
  const void *join = reinterpret_cast<const void *>(&embed_join_kernel<Elem<T>::CE>);
  const int64_t units = chunks * ((a.pieces + 63) / 64);
  return hipLaunchKernel(join, dim3((unsigned)(units < 2048 ? units : 2048)), dim3(512), params, 0, st) == hipSuccess ? S1F_OK : S1F_EDEVICE;
}

}  // namespace
}  // namespace s1f

using namespace s1f;

extern "C" int s1f_embed_fwd(const s1f_rows *desc, const int64_t *ids, int64_t ids_stride_b, const void *table, int64_t table_stride,
                             int64_t vocab, float scale, void *out, void *hip_stream) {
  const int rc = check(desc, vocab, table_stride);
  if (rc != S1F_OK) return rc;
  if (!ids || !table || !out || !on_element(table, desc->dtype) || !on_element(out, desc->dtype) || (reinterpret_cast<uintptr_t>(ids) & 7)) return S1F_EINVAL;
  const bool wide = on16(table) && on16(out) && table_stride % elements_of_16_bytes(desc->dtype) == 0 &&
                    wide_rows(desc, desc->y_stride_b, desc->y_stride_s);
  EmbedArgs a = {};
  a.ids = ids; a.ids_sb = ids_stride_b;
  a.table = table; a.table_stride = table_stride;
  a.out = out; a.y = y_rows(desc);
  a.n = (int32_t)(desc->batch * desc->rows); a.hidden = desc->hidden; a.vocab = (int32_t)vocab; a.scale = scale;
  a.pieces = pieces_of(desc);
  a.tpr_log2 = threads_per_row_log2(a.pieces);
  const int64_t groups = 256 >> a.tpr_log2, grid = (a.n + groups - 1) / groups;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  if (desc->dtype == S1F_BF16) return launch_rows_kernel(wide ? &embed_fwd_kernel<bf16_t, true> : &embed_fwd_kernel<bf16_t, false>, grid, 256, a, st);
  return launch_rows_kernel(wide ? &embed_fwd_kernel<float, true> : &embed_fwd_kernel<float, false>, grid, 256, a, st);
}

extern "C" size_t s1f_embed_bwd_workspace_bytes(const s1f_rows *desc, int64_t vocab) {
  return desc && check(desc, vocab, desc->hidden) == S1F_OK ? (size_t)space_of(desc).bytes : 0;
}

extern "C" int s1f_embed_bwd(const s1f_rows *desc, const int64_t *ids, int64_t ids_stride_b, const void *dout, int64_t vocab, float scale,
                             float *dtable_acc, int64_t acc_stride, void *workspace, size_t workspace_bytes, void *hip_stream) {
  const int rc = check(desc, vocab, acc_stride);
  if (rc != S1F_OK) return rc;
  if (!ids || !dout || !dtable_acc || !workspace || !on_element(dout, desc->dtype) || !on4(dtable_acc) || !on16(workspace) ||
      (reinterpret_cast<uintptr_t>(ids) & 7))
    return S1F_EINVAL;
  const EmbedSpace space = space_of(desc);
  if (workspace_bytes < (size_t)space.bytes) return S1F_EINVAL;
  const bool wide = on16(dout) && on16(dtable_acc) && acc_stride % 4 == 0 && wide_rows(desc, desc->y_stride_b, desc->y_stride_s);
  char *ws = reinterpret_cast<char *>(workspace);
  EmbedArgs a = {};
  a.ids = ids; a.ids_sb = ids_stride_b;
  a.dout = dout; a.y = y_rows(desc);
  a.acc = dtable_acc; a.acc_stride = acc_stride;
  a.n = (int32_t)(desc->batch * desc->rows); a.hidden = desc->hidden; a.vocab = (int32_t)vocab; a.scale = scale;
  a.pieces = pieces_of(desc);
  a.tpr_log2 = threads_per_row_log2(a.pieces);
  a.chunk = chunk_of(a.n);
  a.part_ld = (int32_t)part_ld_of(desc);
  a.row_of = reinterpret_cast<int32_t *>(ws + space.rows);
  a.key_of = reinterpret_cast<int32_t *>(ws + space.keys);
  a.long_runs = reinterpret_cast<int32_t *>(ws + space.long_runs);
  a.head = reinterpret_cast<float *>(ws + space.head);
  a.tail = reinterpret_cast<float *>(ws + space.tail);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  int e = S1F_OK;
  if (a.n <= kMostRanked) {
    e = launch_rows_kernel(&embed_rank_kernel, (a.n + kRanked - 1) / kRanked, 1024, a, st, 4 * 64 * ((a.n + 63) / 64));
  } else {
    int all = 1;
    while ((int64_t(1) << all) <= vocab) ++all;   // bits of 0 .. vocab
    const int passes = (all + 8) / 9;
    a.tiles = (a.n + kTile - 1) / kTile;
    a.count = reinterpret_cast<int32_t *>(ws + space.count);
    a.scanned = a.tiles > kMostSummed;
    int32_t *rows[2] = {a.row_of, reinterpret_cast<int32_t *>(ws + space.rows2)}, *keys[2] = {a.key_of, reinterpret_cast<int32_t *>(ws + space.keys2)};
    for (int p = 0; p < passes && e == S1F_OK; ++p) {
      const int to = (passes - 1 - p) & 1;   // the last pass ends in row_of
      EmbedArgs pass = a;
      pass.row_of = rows[to]; pass.key_of = keys[to];
      pass.row_from = rows[to ^ 1]; pass.key_from = keys[to ^ 1];
      pass.first_pass = p == 0;
      pass.shift = all * p / passes;
      pass.bits = all * (p + 1) / passes - pass.shift;
      e = launch_rows_kernel(&embed_count_kernel, a.tiles, 256, pass, st);
      if (e == S1F_OK && a.scanned) e = launch_rows_kernel(&embed_scan_kernel, ((1 << pass.bits) + 3) / 4, 256, pass, st);
      if (e == S1F_OK) e = launch_rows_kernel(&embed_place_kernel, a.tiles, 256, pass, st);
    }
  }
  if (e != S1F_OK) return e;
  return desc->dtype == S1F_BF16 ? sums<bf16_t>(a, wide, st) : sums<float>(a, wide, st);
}
