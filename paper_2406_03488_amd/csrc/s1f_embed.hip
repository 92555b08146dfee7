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
  int32_t tpr_log2, chunk;              // threads that share a row; sorted rows per workgroup of the sums
  float scale;
  // workspace of the backward
  int32_t *row_of, *key_of;             // rows sorted by token, and their tokens (`vocab`: none)
  int32_t *row_from, *key_from, *count; // input of a sorting pass; rows of each tile with each digit
  float *head, *tail;                   // [chunk][hidden]: sum of the run that reaches into the chunk, that leaves it
  int32_t tiles, shift, bits, first_pass;
};

S1F_DEV int key_at(const EmbedArgs &a, int row) {
  int b, r;
  div_mod(row, a.y.by_rows, b, r);
  const int64_t id = a.ids[b * a.ids_sb + r];
  return id >= 0 && id < a.vocab ? (int)id : a.vocab;
}

// 2^tpr_log2 threads per row, each of which takes every 2^tpr_log2-th piece.
template <typename T, bool WIDE> __global__ void __launch_bounds__(256) embed_fwd_kernel(const EmbedArgs a) {
  typedef Piece<T, WIDE> P;
  const int row = (blockIdx.x << (8 - a.tpr_log2)) + (threadIdx.x >> a.tpr_log2);
  if (row >= a.n) return;
  const int key = key_at(a, row), step = 1 << a.tpr_log2;
  const T *from = reinterpret_cast<const T *>(a.table) + (key < a.vocab ? key : 0) * a.table_stride;
  T *to = reinterpret_cast<T *>(a.out) + a.y.offset(row);
  for (int p = threadIdx.x & (step - 1); p < a.pieces; p += step) {
    typename P::Values v;
    P::load(from + p * P::N, v);
#pragma unroll
    for (int e = 0; e < P::N; ++e) v[e] = key < a.vocab ? v[e] * a.scale : 0.f;
    P::store(to + p * P::N, v);
  }
}

// Rows sorted by token by counting, for every row, the rows in front of it: n^2 comparisons, of 64 by one vector instruction, whose
// result a scalar one counts.  A workgroup places 32 rows; its waves share the rows that they are compared with.
__global__ void __launch_bounds__(256) embed_rank_kernel(const EmbedArgs a) {
  __shared__ int counted[4][32];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first = blockIdx.x * 32;
  const int own_row = first + (lane & 31);
  const int own = own_row < a.n ? key_at(a, own_row) : a.vocab;
  int key[32], before[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    key[i] = __builtin_amdgcn_readlane(own, i);
    before[i] = 0;
  }
  const int blocks = (a.n + 63) >> 6, here = first >> 6;
  for (int c = wave; c < blocks; c += 4) {
    const int row = 64 * c + lane;
    const int x = row < a.n ? key_at(a, row) : 0x7fffffff;
    if (c == here) {
#pragma unroll
      for (int i = 0; i < 32; ++i) before[i] += __builtin_popcountll(__ballot(x < key[i] || (x == key[i] && row < first + i)));
    } else {
      const int equal = c < here ? 1 : 0;   // rows in front with the same token count, those behind do not
#pragma unroll
      for (int i = 0; i < 32; ++i) before[i] += __builtin_popcountll(__ballot(x < key[i] + equal));
    }
  }
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < 32; ++i) counted[wave][i] = before[i];
  }
  __syncthreads();
  if (threadIdx.x < 32 && own_row < a.n) {
    const int at = counted[0][lane] + counted[1][lane] + counted[2][lane] + counted[3][lane];
    a.row_of[at] = own_row;
    a.key_of[at] = own;
  }
}

// Sorting in passes over digits of at most 9 bits, the lowest first, each of which keeps the order of equal digits: count the digits of
// every tile of 1024 rows, sum the counts up, and place the rows.  A wave has a tile to itself.
constexpr int kTile = 1024, kDigits = 512;

S1F_DEV int pass_key(const EmbedArgs &a, int i) { return a.first_pass ? key_at(a, i) : a.key_from[i]; }

__global__ void __launch_bounds__(256) embed_count_kernel(const EmbedArgs a) {
  __shared__ int counts[4][kDigits];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, tile = blockIdx.x * 4 + wave, digits = 1 << a.bits;
  for (int d = lane; d < digits; d += 64) counts[wave][d] = 0;
  __syncthreads();
  for (int i = tile * kTile + lane; i < a.n && i < (tile + 1) * kTile; i += 64)
    atomicAdd(&counts[wave][(pass_key(a, i) >> a.shift) & (digits - 1)], 1);   // (whole numbers: the same in any order)
  __syncthreads();
  if (tile < a.tiles)
    for (int d = lane; d < digits; d += 64) a.count[d * a.tiles + tile] = counts[wave][d];
}

// Exclusive sums of `count` by one workgroup, 4 entries per thread at a time.
__global__ void __launch_bounds__(1024) embed_scan_kernel(const EmbedArgs a) {
  __shared__ int of_wave[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, total = a.tiles << a.bits;
  int carry = 0;
  for (int at = 0; at < total; at += 4096) {
    const int i = at + 4 * threadIdx.x;
    int v[4], own = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = i + e < total ? a.count[i + e] : 0;
      own += v[e];
    }
    int x = own;
    for (int s = 1; s < 64; s *= 2) {
      const int y = __shfl_up(x, s);
      if (lane >= s) x += y;
    }
    if (lane == 63) of_wave[wave] = x;
    __syncthreads();
    int before = carry, all = 0;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before += of_wave[w];
      all += of_wave[w];
    }
    before += x - own;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (i + e < total) a.count[i + e] = before;
      before += v[e];
    }
    carry += all;
    __syncthreads();
  }
}

__global__ void __launch_bounds__(256) embed_place_kernel(const EmbedArgs a) {
  __shared__ int next[4][kDigits];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, tile = blockIdx.x * 4 + wave, digits = 1 << a.bits;
  if (tile < a.tiles)
    for (int d = lane; d < digits; d += 64) next[wave][d] = a.count[d * a.tiles + tile];
  __syncthreads();
  if (tile >= a.tiles) return;   // (no barrier from here on)
  const int end = (tile + 1) * kTile < a.n ? (tile + 1) * kTile : a.n;
  for (int base = tile * kTile; base < end; base += 64) {
    const int i = base + lane;
    const bool is = i < end;
    const int key = is ? pass_key(a, i) : 0, digit = (key >> a.shift) & (digits - 1);
    uint64_t same = __ballot(is);
    for (int b = 0; b < a.bits; ++b) {
      const uint64_t ones = __ballot((digit >> b) & 1);
      same &= (digit >> b) & 1 ? ones : ~ones;
    }
    if (is) {
      const int rank = __builtin_popcountll(same & ((uint64_t(1) << lane) - 1));
      const int at = *(volatile int *)&next[wave][digit] + rank;
      a.key_of[at] = key;
      a.row_of[at] = a.first_pass ? i : a.row_from[i];
      if ((same >> lane) == 1) *(volatile int *)&next[wave][digit] = at + 1;   // the last lane of its digit
    }
  }
}

// Sums of the runs in one chunk of the sorted rows.  2^tpr_log2 threads share the columns of a row; the others of a workgroup take
// other chunks.
template <typename T, bool WIDE> struct RunSum {
  typedef Piece<T, WIDE> P;
  const EmbedArgs &a;
  float sum[P::N];
  int chunk, piece;
  // at the end of a run: whether it reaches into the chunk from the one before, whether it goes on behind it
  S1F_DEV void flush(int key, bool into, bool on) {
    if (key < a.vocab) {
      if (into || on) {
        store_f32<P::N>((into ? a.head : a.tail) + (int64_t)chunk * a.hidden + piece * P::N, sum);
      } else {
        float *to = a.acc + key * a.acc_stride + piece * P::N;
        float was[P::N];
        load_f32<P::N>(to, was);
#pragma unroll
        for (int e = 0; e < P::N; ++e) was[e] += a.scale * sum[e];
        store_f32<P::N>(to, was);
      }
    }
#pragma unroll
    for (int e = 0; e < P::N; ++e) sum[e] = 0.f;
  }
};

template <typename T, bool WIDE> __global__ void __launch_bounds__(256) embed_sum_kernel(const EmbedArgs a) {
  typedef Piece<T, WIDE> P;
  const int tpr = 1 << a.tpr_log2;
  RunSum<T, WIDE> s{a, {}, (int)(blockIdx.x << (8 - a.tpr_log2)) + (int)(threadIdx.x >> a.tpr_log2),
                    (int)(blockIdx.y * tpr + (threadIdx.x & (tpr - 1)))};
  const int begin = s.chunk * a.chunk, end = begin + a.chunk < a.n ? begin + a.chunk : a.n;
  if (begin >= a.n || s.piece >= a.pieces) return;
  const T *dout = reinterpret_cast<const T *>(a.dout) + s.piece * P::N;
  int key = a.key_of[begin];
  bool into = begin > 0 && a.key_of[begin - 1] == key;
  constexpr int U = 8;   // rows asked for together
  for (int i = begin; i < end && key < a.vocab; i += U) {
    int k[U];
    typename P::Values v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = i + u < end ? i + u : end - 1;
      k[u] = a.key_of[at];
      P::load(dout + a.y.offset(a.row_of[at]), v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= end) break;
      if (k[u] != key) {
        s.flush(key, into, false);
        into = false;
        key = k[u];
      }
#pragma unroll
      for (int e = 0; e < P::N; ++e) s.sum[e] += v[u][e];
    }
  }
  s.flush(key, into, end < a.n && a.key_of[end] == key);
}

// Runs longer than a chunk: the threads of the chunk in which one starts add up what it has left there and in the chunks behind.
template <int N> __global__ void __launch_bounds__(256) embed_join_kernel(const EmbedArgs a) {
  const int tpr = 1 << a.tpr_log2;
  const int chunk = (int)(blockIdx.x << (8 - a.tpr_log2)) + (int)(threadIdx.x >> a.tpr_log2);
  const int piece = blockIdx.y * tpr + (threadIdx.x & (tpr - 1));
  const int begin = chunk * a.chunk;
  int end = begin + a.chunk;
  if (end >= a.n || piece >= a.pieces) return;
  const int key = a.key_of[end - 1];
  if (key >= a.vocab || a.key_of[end] != key) return;
  if (begin > 0 && a.key_of[begin - 1] == key) return;   // it has started further in front
  float sum[N], more[N];
  load_f32<N>(a.tail + (int64_t)chunk * a.hidden + piece * N, sum);
  for (int c = chunk + 1;; ++c) {
    load_f32<N>(a.head + (int64_t)c * a.hidden + piece * N, more);
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] += more[e];
    end += a.chunk;
    if (end >= a.n || a.key_of[end] != key || a.key_of[end - 1] != key) break;
  }
  float *to = a.acc + key * a.acc_stride + piece * N;
  load_f32<N>(to, more);
#pragma unroll
  for (int e = 0; e < N; ++e) more[e] += a.scale * sum[e];
  store_f32<N>(to, more);
}

constexpr int32_t kMostVocab = 1 << 26;   // three sorting passes
constexpr int32_t kMostRanked = 16384;    // rows up to which counting sorts them

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
struct EmbedSpace {
  int64_t rows, keys, rows2, keys2, count, head, tail, bytes;
};
constexpr int kChunk = 32;
EmbedSpace space_of(const s1f_rows *d) {
  const int64_t n = d->batch * d->rows, chunks = (n + kChunk - 1) / kChunk;
  EmbedSpace s = {};
  int64_t at = 0;
  auto take = [&at](int64_t bytes) { const int64_t was = at; at += up(bytes); return was; };
  s.rows = take(4 * n);
  s.keys = take(4 * n);
  if (n > kMostRanked) {
    s.rows2 = take(4 * n);
    s.keys2 = take(4 * n);
    s.count = take(4 * kDigits * ((n + kTile - 1) / kTile));
  }
  if (chunks > 1) {
    s.head = take(4 * chunks * d->hidden);
    s.tail = take(4 * chunks * d->hidden);
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
  const void *join = wide ? reinterpret_cast<const void *>(&embed_join_kernel<Elem<T>::CE>) : reinterpret_cast<const void *>(&embed_join_kernel<1>);
  return hipLaunchKernel(join, grid, dim3(256), params, 0, st) == hipSuccess ? S1F_OK : S1F_EDEVICE;
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
  a.pieces = wide ? desc->hidden / (int32_t)elements_of_16_bytes(desc->dtype) : desc->hidden;
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
  a.pieces = wide ? desc->hidden / (int32_t)elements_of_16_bytes(desc->dtype) : desc->hidden;
  a.tpr_log2 = threads_per_row_log2(a.pieces);
  a.chunk = kChunk;
  a.row_of = reinterpret_cast<int32_t *>(ws + space.rows);
  a.key_of = reinterpret_cast<int32_t *>(ws + space.keys);
  a.head = reinterpret_cast<float *>(ws + space.head);
  a.tail = reinterpret_cast<float *>(ws + space.tail);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  int e = S1F_OK;
  if (a.n <= kMostRanked) {
    e = launch_rows_kernel(&embed_rank_kernel, (a.n + 31) / 32, 256, a, st);
  } else {
    int all = 1;
    while ((int64_t(1) << all) <= vocab) ++all;   // bits of 0 .. vocab
    const int passes = (all + 8) / 9;
    a.tiles = (a.n + kTile - 1) / kTile;
    a.count = reinterpret_cast<int32_t *>(ws + space.count);
    int32_t *rows[2] = {a.row_of, reinterpret_cast<int32_t *>(ws + space.rows2)}, *keys[2] = {a.key_of, reinterpret_cast<int32_t *>(ws + space.keys2)};
    for (int p = 0; p < passes && e == S1F_OK; ++p) {
      const int to = (passes - 1 - p) & 1;   // the last pass ends in row_of
      EmbedArgs pass = a;
      pass.row_of = rows[to]; pass.key_of = keys[to];
      pass.row_from = rows[to ^ 1]; pass.key_from = keys[to ^ 1];
      pass.first_pass = p == 0;
      pass.shift = all * p / passes;
      pass.bits = all * (p + 1) / passes - pass.shift;
      e = launch_rows_kernel(&embed_count_kernel, (a.tiles + 3) / 4, 256, pass, st);
      if (e == S1F_OK) e = launch_rows_kernel(&embed_scan_kernel, 1, 1024, pass, st);
      if (e == S1F_OK) e = launch_rows_kernel(&embed_place_kernel, (a.tiles + 3) / 4, 256, pass, st);
    }
  }
  if (e != S1F_OK) return e;
  return desc->dtype == S1F_BF16 ? sums<bf16_t>(a, wide, st) : sums<float>(a, wide, st);
}
