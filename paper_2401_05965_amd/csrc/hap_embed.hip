/*
 * Embedding table: Y[t] = scale * W[id_t], and its gradient dW[v] = scale * sum of dY[t] over the tokens with id v.
 *
 * A lookup is the product of one-hot rows with W, so the sharding rules are those of a linear layer: batch (tokens), feature (columns of W),
 * reduction (rows of W: a device's Y is a partial sum, zeros for the other devices' tokens).
 *
 * Bound: HBM; the gradient's largest part is usually the table itself, written whole.  Its steps:
 *   1  sort the tokens by id (stable counting sort by digits, hap_sort.h); up to kSortAlone tokens one workgroup does it while the other
 *      workgroups of the launch fill the table with zeros.  The sort costs nothing where the fill takes longer: 8192 tokens 19 us, a fill of 125 MB;
 *      16384 tokens 27 us, 180 MB.  A smaller table, and an accumulating pass, which fills nothing, wait for it
 *   2  chunks of the sorted tokens, one wave per chunk and 64 vectors of columns: rows of one id follow each other and are summed in registers;
 *      an id whose tokens all lie in the chunk is finished and stored, one that crosses the chunk's borders leaves a partial row
 *   3  the partial rows of an id are added up by the workgroup of the chunk in which it begins
 * Every sum has a fixed order; no floating-point atomics.
 */
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "hap_internal.h"
#include "hap_lanes.h"
#include "hap_sort.h"

namespace {

using namespace hap_lanes;

constexpr int64_t kSortAlone = 16384;
constexpr int kSortBlocks = 256;

/* Ids of 4 or 8 bytes -> row of the device's part of the table, -1 for an id outside of it (padding, another device's). */
struct Ids {
  const void* p;
  int bytes;
  int64_t lo, n;
};
__device__ __forceinline__ int64_t id_at(const Ids& d, int64_t t) {
  return d.bytes == 8 ? static_cast<const int64_t*>(d.p)[t] : (int64_t) static_cast<const int*>(d.p)[t];
}
__device__ __forceinline__ int64_t row_of(const Ids& d, int64_t id) {
  const uint64_t r = (uint64_t)id - (uint64_t)d.lo;
  return id >= 0 && r < (uint64_t)d.n ? (int64_t)r : -1;
}

/* Rows are the elements [first, cols) of rows that begin on a chunk: a range of columns of whole tensors may begin inside one. */
template <typename T, int V, bool STREAM, bool CUT>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(int64_t tokens, int first, int cols, const Ids ids, const T* W, int64_t ldw, float scale, T* Y, int64_t ldy) {
  constexpr int U = 4, STEP = 64 * V;  // chunks in flight
  const int lane = threadIdx.x & 63, bytes = chunk_bytes<T, V>(cols);
  const int64_t t = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  if (t >= tokens) return;
  const int64_t r = row_of(ids, id_at(ids, t));
  const auto from = row_at(W + (r < 0 ? 0 : r) * ldw, r < 0 ? 0 : bytes), to = row_at(Y + t * ldy, bytes);
  for (int c = lane * V; c - lane * V < cols; c += U * STEP) {
    Pack<T, V> p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) p[u] = row_load<T, V>(from, c + u * STEP);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int v = 0; v < V; ++v) p[u].v[v] = r >= 0 ? (T)(scale * to_f32(p[u].v[v])) : (T)0.0f;
      row_store_part<STREAM, CUT>(to, c + u * STEP, p[u], first, cols);
    }
  }
}

/* ---- sorting: keys are rows of the device's part of the table, `n` (larger than all) for tokens without one */

struct SortArgs {
  int64_t tokens, per_block;
  Ids ids;
  int passes, bits;
  uint32_t *key[2], *token[2];
  int* before;                         // [workgroups][1 << bits]
};

/* f(load, digit_of, place) with the entries of a pass: the ids themselves in the first, keys and tokens as the pass before left them later. */
struct Entry { uint32_t key, token; };
template <typename F> __device__ __forceinline__ void with_entries(const SortArgs& a, int pass, F&& f) {
  const int shift = pass * a.bits;
  const uint32_t mask = (1u << a.bits) - 1;
  uint32_t *key = a.key[pass & 1], *token = a.token[pass & 1];
  if (pass == 0) {
    const auto key_of = [&](int64_t id) {
      const int64_t r = row_of(a.ids, id);
      return (uint32_t)(r < 0 ? a.ids.n : r);
    };
    const auto digit_of = [&](int64_t id) { return (int)(key_of(id) & mask); };
    const auto place = [&](int64_t n, int64_t id, int p) { key[p] = key_of(id); token[p] = (uint32_t)n; };
    // (one branch around all loads: the compiler waits where a branch ends)
    if (a.ids.bytes == 8) f([&](int64_t n) { return static_cast<const int64_t*>(a.ids.p)[n]; }, digit_of, place);
    else f([&](int64_t n) { return (int64_t) static_cast<const int*>(a.ids.p)[n]; }, digit_of, place);
  } else {
    const uint32_t *from = a.key[(pass - 1) & 1], *who = a.token[(pass - 1) & 1];
    f([&](int64_t n) { return Entry{from[n], who[n]}; }, [&](Entry e) { return (int)((e.key >> shift) & mask); },
      [&](int64_t, Entry e, int p) { key[p] = e.key; token[p] = e.token; });
  }
}

/* Sum of v over the threads before this one; all kThreads threads take part. */
__device__ __forceinline__ int before_me(int v, hap_sort::lds_int* scratch) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, s = sum_up_to_lane(v);
  if (lane == 63) scratch[wave] = s;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int w = 0; w < hap_sort::kWaves; ++w) {
    const int x = scratch[w];
    base += w < wave ? x : 0;
  }
  __syncthreads();
  return base + s - v;
}

/* One digit of the range of workgroup b out of nb; `before` holds every workgroup's counts of the digit's values. */
__device__ __forceinline__ void sort_pass(const SortArgs& a, int pass, int b, int nb, hap_sort::lds_int* count, hap_sort::lds_int* scratch) {
  const int values = 1 << a.bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  hap_sort::lds_int *const mine = count + hap_sort::kWaves * values, *const all = mine + values;      // of the workgroups before this one, of all
  for (int d = threadIdx.x; d < 2 * values; d += hap_sort::kThreads) mine[d] = 0;
  const int64_t begin = (int64_t)b * a.per_block, end = begin + a.per_block < a.tokens ? begin + a.per_block : a.tokens;
  with_entries(a, pass, [&](auto load, auto digit_of, auto) { hap_sort::count_keys(count, values, begin, end, load, digit_of); });
  for (int d = lane; d < values; d += 64) {
    int lower = 0, total = 0;
#pragma unroll 4
    for (int i = wave; i < nb; i += hap_sort::kWaves) {
      const int c = a.before[(int64_t)i * values + d];
      total += c;
      lower += i < b ? c : 0;
    }
    __hip_atomic_fetch_add(&all[d], total, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __hip_atomic_fetch_add(&mine[d], lower, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
  __syncthreads();
  const int d = threadIdx.x;            // (at most 512 values: a thread for each)
  const int first = before_me(d < values ? all[d] : 0, scratch);
  if (d < values) hap_sort::first_places(count, values, d, first + mine[d]);
  __syncthreads();
  with_entries(a, pass, [&](auto load, auto digit_of, auto place) { hap_sort::place_keys(count, values, a.bits, begin, end, load, digit_of, place); });
}

/* Non-temporal as long as the one workgroup's sort beside it takes longer or about as long: little waits for the stores then, and the sums that follow find room in the
 * last-level cache.  That is up to 50 MB and 11 KB more for every token (fill_streamed).  Plain / non-temporal, three sets of buffers in turn, gradient alone and with the norm
 * over it behind, which reads all of it, us:
 *   300 tokens of 1024      30 MB 17.7 / 16.9 and 27.5 / 27.1     63 MB 18.6 / 18.2 and 32.8 / 35.2    125 MB 29.6 / 29.9 and 50.7 / 56.3
 *   2000 of 4096            63 MB 27.4 / 25.5 and 41.6 / 40.8     94 MB 34.3 / 29.2 and 53.9 / 53.1    125 MB 35.3 / 34.6 and 59.3 / 63.1
 *   4096 of 2560, bf16      94 MB 38.7 / 30.5 and 59.4 / 58.1    110 MB 39.1 / 33.9 and 61.9 / 62.7    156 MB 43.4 / 42.2 and 71.5 / 78.7
 *   8192 of 1024           125 MB 44.5 / 36.5 and 68.0 / 67.3    140 MB 44.7 / 40.2 and 70.4 / 71.0    156 MB 44.7 / 43.6 and 73.1 / 78.1
 *   8192 of 4096, bf16     125 MB 59.7 / 57.8 and 84.7 / 82.9    156 MB 59.4 / 61.2 and 94.5 / 92.0    200 MB 69.8 / 71.1 and 100.5 / 110.1
 *   16384 of 768           140 MB 60.7 / 51.0 and 86.0 / 85.6    200 MB 60.4 / 56.7 and 96.6 / 98.6    250 MB 66.8 / 65.6 and 105.0 / 116.9
 *   16384 of 4096, bf16    156 MB 99.6 / 93.3 and 125 / 117      200 MB 105 / 95 and 136 / 128         320 MB 118 / 122 and 180 / 181
 * (two sets, which the cache half holds: 8192 of 1024, 125 MB 35.6 / 34.9 and 59.3 / 61.6).  Many workgroups' sort is too short: 32768 of 2048, 63 MB 93.5 / 96.0 and
 * 110 / 111, 200 MB 135 / 143 and 169 / 172. */
struct FillArgs {
  char* p;
  int64_t rows, ld;                    // ld in bytes
  int width, unit;                     // bytes of a row; 4 or 2: what rows begin and end on a multiple of
  int stream;                          // non-temporal
};

/* 16-byte stores between the first and the last boundary of them in a row, units before and behind. */
template <typename U> __device__ __forceinline__ void fill_rows(const FillArgs& f, int64_t first, int64_t step) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const u32x4 zero = {0, 0, 0, 0};
  for (int64_t r = first * hap_sort::kWaves + wave; r < f.rows; r += step * hap_sort::kWaves) {
    char* const row = f.p + r * f.ld;
    const int head = (int)(-(uintptr_t)row & 15) < f.width ? (int)(-(uintptr_t)row & 15) : f.width, chunks = (f.width - head) / 16, tail = head + chunks * 16;
    u32x4* const body = reinterpret_cast<u32x4*>(row + head);
    if (f.stream) {
      for (int c = lane; c < chunks; c += 64) __builtin_nontemporal_store(zero, body + c);
    } else {
      for (int c = lane; c < chunks; c += 64) body[c] = zero;
    }
    if (lane * (int)sizeof(U) < head) reinterpret_cast<U*>(row)[lane] = 0;
    if (tail + lane * (int)sizeof(U) < f.width) reinterpret_cast<U*>(row + tail)[lane] = 0;
  }
}

__device__ __forceinline__ void fill(const FillArgs& f, int64_t first, int64_t step) {
  if (f.unit == 4) fill_rows<uint32_t>(f, first, step);
  else fill_rows<uint16_t>(f, first, step);
}

/* Workgroup 0 sorts, the others fill.  An entry is one word, its key above its token, and stays in a register between a pass's walk and the
 * exchange through LDS (entries scattered to global memory instead: 57 us for 16384 tokens, one compute unit's address path). */
constexpr int kAloneTokenBits = 14;
template <int BITS> __global__ __launch_bounds__(hap_sort::kThreads) void sort_alone_kernel(const SortArgs a, const FillArgs f) {
  using namespace hap_sort;
  extern __shared__ int lds[];
  __shared__ int sums[kWaves];
  if (blockIdx.x > 0) {
    fill(f, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  lds_int *const count = (lds_int*)lds, *const scratch = (lds_int*)sums;
  constexpr int values = 1 << BITS;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  lds_int* const entries = count + kWaves * values;
  int64_t lo, hi;
  part_of(0, a.tokens, &lo, &hi);
  int64_t id[kBatch];
  const auto at = [&](int i) { return lo + i * 64 + lane < hi ? lo + i * 64 + lane : hi - 1; };
  if (lo < hi && a.ids.bytes == 8) {   // (one branch around all loads: the compiler waits where a branch ends)
#pragma unroll
    for (int i = 0; i < kBatch; ++i) id[i] = static_cast<const int64_t*>(a.ids.p)[at(i)];
  } else if (lo < hi) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) id[i] = static_cast<const int*>(a.ids.p)[at(i)];
  }
  uint32_t v[kBatch];
  int rank[kBatch];
#pragma unroll
  for (int i = 0; i < kBatch; ++i) {
    const int64_t r = lo < hi ? row_of(a.ids, id[i]) : -1;
    v[i] = (uint32_t)(r < 0 ? a.ids.n : r) << kAloneTokenBits | (uint32_t)(lo + i * 64 + lane);
  }
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = kAloneTokenBits + pass * BITS;
    for (int i = threadIdx.x; i < kWaves * values; i += kThreads) count[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (lo + i * 64 < hi) rank[i] = take_place<BITS>(count + wave * values, lo + i * 64 + lane < hi ? (int)((v[i] >> shift) & (uint32_t)(values - 1)) : -1, BITS);
    __syncthreads();
    const int total = (int)threadIdx.x < values ? first_places(count, values, threadIdx.x, 0) : 0;
    const int first = before_me(total, scratch);
    if ((int)threadIdx.x < values) entries[threadIdx.x] = first;
    __syncthreads();
    int place[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (lo + i * 64 + lane < hi) {
        const int k = (int)((v[i] >> shift) & (uint32_t)(values - 1));
        place[i] = entries[k] + count[wave * values + k] + rank[i];
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (lo + i * 64 + lane < hi) entries[place[i]] = (int)v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (lo + i * 64 + lane < hi) v[i] = (uint32_t)entries[lo + i * 64 + lane];
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kBatch; ++i) {
    const int64_t n = lo + i * 64 + lane;
    if (n < hi) {
      a.key[0][n] = v[i] >> kAloneTokenBits;
      a.token[0][n] = v[i] & ((1u << kAloneTokenBits) - 1);
    }
  }
}

/* Workgroups 0 .. nb - 1 count the values of a digit in their ranges, the others fill. */
__global__ __launch_bounds__(hap_sort::kThreads) void sort_count_kernel(const SortArgs a, int pass, int nb, const FillArgs f) {
  extern __shared__ int lds[];
  hap_sort::lds_int* const count = (hap_sort::lds_int*)lds;
  if ((int)blockIdx.x >= nb) {
    fill(f, blockIdx.x - nb, gridDim.x - nb);
    return;
  }
  const int values = 1 << a.bits;
  const int64_t begin = (int64_t)blockIdx.x * a.per_block, end = begin + a.per_block < a.tokens ? begin + a.per_block : a.tokens;
  with_entries(a, pass, [&](auto load, auto digit_of, auto) { hap_sort::count_keys(count, values, begin, end, load, digit_of); });
  for (int d = threadIdx.x; d < values; d += hap_sort::kThreads) {
    int s = 0;
    for (int w = 0; w < hap_sort::kWaves; ++w) s += count[w * values + d];
    a.before[(int64_t)blockIdx.x * values + d] = s;
  }
}

__global__ __launch_bounds__(hap_sort::kThreads) void sort_place_kernel(const SortArgs a, int pass, int nb) {
  extern __shared__ int lds[];
  hap_sort::lds_int* const count = (hap_sort::lds_int*)lds;
  __shared__ int sums[hap_sort::kWaves];
  hap_sort::lds_int* const scratch = (hap_sort::lds_int*)sums;
  sort_pass(a, pass, blockIdx.x, nb, count, scratch);
}

/* ---- sums over the sorted tokens */

struct SumArgs {
  int64_t tokens;                      // sorted entries
  const uint32_t *key, *token;
  uint32_t none;                       // the key of tokens without a row
  int chunk, chunks;                   // entries of a chunk (at most 64), chunks
  int first, cols, width, slabs;       // columns [first, cols) from a chunk on, the width of a partial row, waves across the columns
  float* part;                         // [chunks][2][cols]: an id that began before the chunk, one that goes on behind it
  int64_t ldy, ldw;
  float scale;
  int accumulate;
};

template <typename W, int V> __device__ __forceinline__ void store_row(const SumArgs& a, W* dW, uint32_t row, int c, const float (&s)[V]) {
  const auto to = row_at(dW + (int64_t)row * a.ldw, chunk_bytes<W, V>(a.cols));
  Pack<W, V> o;
  if (a.accumulate) o = row_load<W, V>(to, c);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float x = a.scale * s[v];
    o.v[v] = (W)(a.accumulate ? to_f32(o.v[v]) + x : x);
  }
  row_store_part<false, (V > 1)>(to, c, o, a.first, a.cols);
}

template <int V> __device__ __forceinline__ void store_part(const SumArgs& a, int64_t slot, int c, const float (&s)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) a.part[slot * a.width + c + v] = s[v];
}

template <typename T, typename W, int V>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const SumArgs a, const T* dY, W* dW) {
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t chunk = w / a.slabs;
  if (chunk >= a.chunks) return;
  const int c = ((int)(w % a.slabs) * 64 + lane) * V;
  const int64_t first = chunk * a.chunk;
  const int len = (int)(first + a.chunk < a.tokens ? a.chunk : a.tokens - first);
  const uint32_t key = lane < len ? a.key[first + lane] : a.none;
  const uint32_t token = lane < len ? a.token[first + lane] : 0;
  const int n = __popcll(__ballot(key < a.none));                  // sorted: those without a row are last
  if (n == 0) return;
  const uint32_t before = first > 0 ? a.key[first - 1] : a.none;
  const uint32_t behind = first + len < a.tokens ? a.key[first + len] : a.none;
  const bool mine = c < a.cols;
  float s[V];
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = 0.0f;
  constexpr int U = 8;                                             // rows in flight
  for (int i = 0; i < n; i += U) {
    Pack<T, V> p[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      p[u] = row_load<T, V>(row_at(dY + (int64_t)from_lane(token, i + u < n ? i + u : n - 1) * a.ldy, chunk_bytes<T, V>(a.cols)), c);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= n) break;
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] += to_f32(p[u].v[v]);
      const uint32_t k = from_lane(key, i + u);
      const bool last = i + u == len - 1;
      const uint32_t after = last ? behind : from_lane(key, i + u + 1 < 64 ? i + u + 1 : 63);
      if (!last && after == k) continue;
      // the id's tokens end here, or the chunk does
      const bool goes_on = last && behind == k;
      const bool began_before = k == before && from_lane(key, 0) == k;
      if (mine) {
        if (began_before) store_part<V>(a, chunk * 2, c, s);
        else if (goes_on) store_part<V>(a, chunk * 2 + 1, c, s);
        else store_row<W, V>(a, dW, k, c, s);
      }
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = 0.0f;
    }
  }
}

/* The ids that cross chunks: the workgroup of the chunk in which one begins adds up its partial rows, four waves taking every fourth. */
template <typename W, int V>
__global__ __launch_bounds__(256) void embedding_join_kernel(const SumArgs a, W* dW) {
  __shared__ float red[4][64 * V];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t chunk = blockIdx.x / a.slabs;
  const int64_t first = chunk * a.chunk, next = first + a.chunk;
  if (next >= a.tokens) return;
  const uint32_t k = a.key[next - 1];
  if (k >= a.none || a.key[next] != k || (first > 0 && a.key[first - 1] == k)) return;
  const int c = ((int)(blockIdx.x % a.slabs) * 64 + lane) * V;
  const bool mine = c < a.cols;
  // the chunks behind that begin with the id
  int64_t ends = chunk + 1;
  for (;;) {
    const int64_t q = ends + lane;
    const uint64_t same = __ballot(q < a.chunks && a.key[(q < a.chunks ? q : 0) * a.chunk] == k);
    if (same == ~0ull) { ends += 64; continue; }
    ends += __builtin_ctzll(~same);
    break;
  }
  float s[V];
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = wave == 0 && mine ? a.part[(chunk * 2 + 1) * a.width + c + v] : 0.0f;
  if (mine) {
#pragma unroll 8
    for (int64_t q = chunk + 1 + wave; q < ends; q += 4) {
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] += a.part[q * 2 * a.width + c + v];
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) red[wave][lane * V + v] = s[v];
  __syncthreads();
  if (wave == 0 && mine) {
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = (red[0][lane * V + v] + red[1][lane * V + v]) + (red[2][lane * V + v] + red[3][lane * V + v]);
    store_row<W, V>(a, dW, k, c, s);
  }
}

/* ---- host */

inline int check_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? HAP_OK : hap_fail(HAP_EDEVICE, "%s launch: %s", what, hipGetErrorString(e));
}

inline int esize(int dtype) { return dtype == HAP_BF16 ? 2 : 4; }
inline int64_t round_up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

/* What the device computes: tokens [t0, t0 + tokens), rows [v0, v0 + rows) and columns [c0, c0 + cols) of the whole. */
struct Part { int64_t t0, tokens, v0, rows, c0, cols; };

int resolve(const hap_embedding_desc* d, int j, Part* p) {
  if (!d) return hap_fail(HAP_EINVAL, "descriptor is NULL");
  if (d->tokens < 0 || d->vocab < 1 || d->hidden < 1) return hap_fail(HAP_EINVAL, "bad sizes");
  if (d->io_dtype != HAP_F32 && d->io_dtype != HAP_BF16) return hap_fail(HAP_EINVAL, "bad io_dtype %d", d->io_dtype);
  if (d->id_bytes != 4 && d->id_bytes != 8) return hap_fail(HAP_EINVAL, "ids of %d bytes", d->id_bytes);
  if (d->mode < HAP_SHARD_BATCH || d->mode > HAP_REPLICATED) return hap_fail(HAP_EINVAL, "bad mode %d", d->mode);
  *p = Part{0, d->tokens, 0, d->vocab, 0, d->hidden};
  int64_t* const lo[] = {&p->t0, &p->c0, &p->v0};
  int64_t* const n[] = {&p->tokens, &p->cols, &p->rows};
  if (d->mode != HAP_REPLICATED) {
    int64_t l, h;
    const int rc = hap_shard_range(d->m, d->offsets, *n[d->mode], j, &l, &h);
    if (rc) return rc;
    *lo[d->mode] = l;
    *n[d->mode] = h - l;
  }
  const int64_t width = d->mode == HAP_SHARD_FEATURE && !d->operands_are_full ? p->cols : d->hidden;
  if (d->ldw < width || d->ldy < width) return hap_fail(HAP_ESHAPE, "leading dimension below %lld columns", (long long)width);
  if (d->tokens > 0x7fffffff || p->rows >= (int64_t)1 << 30 || d->hidden > 0xfffffff)
    return hap_fail(HAP_EUNSUPPORTED, "2^31 tokens, 2^30 rows or 2^28 columns and more");
  return HAP_OK;
}

/* Element offsets of the device's part in W-like and Y-like tensors, and its first id in `ids`. */
int64_t w_offset(const hap_embedding_desc* d, const Part& p) {
  return d->operands_are_full ? p.v0 * d->ldw + p.c0 : 0;
}
int64_t y_offset(const hap_embedding_desc* d, const Part& p) {
  return d->operands_are_full ? p.t0 * d->ldy + p.c0 : 0;
}
Ids ids_of(const hap_embedding_desc* d, const Part& p, const void* ids) {
  return Ids{static_cast<const char*>(ids) + (d->operands_are_full ? p.t0 * d->id_bytes : 0), d->id_bytes, p.v0, p.rows};
}

/* Elements by which views of both tensors lie behind a chunk of V, -1 where they have no common grid of chunks. */
int phase_of(const void* p, const void* q, int es, int qs, int V, int64_t ldp, int64_t ldq) {
  if (ldp % V || ldq % V || (uintptr_t)p % es || (uintptr_t)q % qs) return -1;
  const int a = (int)((uintptr_t)p / es % V), b = (int)((uintptr_t)q / qs % V);
  return a == b ? a : -1;
}

/* The gradient's plan: passes and bits of the sort, its workgroups, chunks, and where things lie in the workspace. */
struct Plan {
  bool alone;                          // one workgroup sorts in LDS
  int passes, bits, blocks, chunk, chunks;
  int64_t key[2], token[2], before, part, bytes;
};
Plan plan_of(const Part& p) {
  Plan q = {};
  int total = 1;
  while (((int64_t)1 << total) <= p.rows) ++total;            // keys 0 .. rows
  q.passes = (total + 8) / 9;                                // (512 values: 32 KB of counts)
  q.bits = (total + q.passes - 1) / q.passes;
  q.alone = p.tokens == 0 || (p.tokens <= kSortAlone && p.rows < (int64_t)1 << (32 - kAloneTokenBits));      // (no tokens: no workspace)
  if (q.alone && total <= 16) { q.bits = 8; q.passes = (total + 7) / 8; }          // (sort_alone_kernel knows digits of 8 and 9 bits)
  else if (q.alone) q.bits = 9;
  const int64_t blocks = (p.tokens + 4095) / 4096;
  q.blocks = q.alone || blocks < 1 ? 1 : (int)(blocks < kSortBlocks ? blocks : kSortBlocks);
  // Chunks as long as four waves for every SIMD remain (1024 SIMDs), 8 to 64 tokens: short ones leave more partial rows, long ones few waves.
  const int64_t slabs = (p.cols + 511) / 512;
  for (q.chunk = 64; q.chunk > 8 && p.tokens / q.chunk * slabs < 4096;) q.chunk /= 2;
  q.chunks = (int)((p.tokens + q.chunk - 1) / q.chunk);
  int64_t at = 0;
  const auto take = [&](int64_t bytes) { const int64_t was = at; at += round_up(bytes, 256); return was; };
  for (int i = 0; i < 2; ++i) { q.key[i] = take(p.tokens * 4); q.token[i] = take(p.tokens * 4); }
  q.before = take(q.alone ? 0 : ((int64_t)q.blocks << q.bits) * 4);
  q.part = take((int64_t)q.chunks * 2 * (p.cols + 16) * 4);        // (rows of whole chunks)
  q.bytes = at;
  return q;
}

template <typename F> void with_type(int dtype, bool vec, F&& f) {
  if (dtype == HAP_BF16) {
    if (vec) f((__bf16)0.0f, std::integral_constant<int, 8>()); else f((__bf16)0.0f, std::integral_constant<int, 1>());
  } else {
    if (vec) f(0.0f, std::integral_constant<int, 4>()); else f(0.0f, std::integral_constant<int, 1>());
  }
}

inline bool fill_streamed(const Plan& q, int64_t tokens, int64_t bytes) { return q.alone && bytes <= 50'000'000 + 11'000 * tokens; }

/* Fills the device's part of the table with zeros and sorts; *sorted: which of the two buffers holds the result. */
int sort_tokens(const SortArgs& a, const Plan& q, const FillArgs& f, int* sorted, hipStream_t s) {
  const size_t lds = (size_t)hap_sort::kWaves * sizeof(int) << q.bits, row = sizeof(int) << q.bits;
  const int64_t want = f.rows > 0 ? (f.rows + hap_sort::kWaves - 1) / hap_sort::kWaves : 0;
  const int fillers = (int)(want < 1024 ? want : 1024);
  *sorted = q.alone ? 0 : (q.passes - 1) & 1;
  if (q.alone) {
    const size_t entries = (size_t)(a.tokens > 512 ? a.tokens : 512) * sizeof(int);       // (and the digit's first places)
    static bool configured[2][64];
    const auto kernel = q.bits == 8 ? sort_alone_kernel<8> : sort_alone_kernel<9>;
    if (const int e = hap_sort::reserve_lds(reinterpret_cast<const void*>(kernel), configured[q.bits == 8], lds + entries, hap_sort::kWaves * 512 * sizeof(int) + kSortAlone * sizeof(int))) return e;
    hipLaunchKernelGGL(kernel, dim3(1 + fillers), dim3(hap_sort::kThreads), lds + entries, s, a, f);
    return check_launch("embedding_bwd sort");
  }
  for (int pass = 0; pass < q.passes; ++pass) {
    hipLaunchKernelGGL(sort_count_kernel, dim3(q.blocks + (pass == 0 ? fillers : 0)), dim3(hap_sort::kThreads), lds, s, a, pass, q.blocks, f);
    int rc = check_launch("embedding_bwd count");
    if (rc) return rc;
    hipLaunchKernelGGL(sort_place_kernel, dim3(q.blocks), dim3(hap_sort::kThreads), lds + 2 * row, s, a, pass, q.blocks);
    if ((rc = check_launch("embedding_bwd place"))) return rc;
  }
  return HAP_OK;
}

}  // namespace

extern "C" {

int hap_embedding_fwd(const hap_embedding_desc* d, int shard_index, const void* ids, const void* W, void* Y, void* stream) {
  hap_clear_error();
  Part p;
  const int rc = resolve(d, shard_index, &p);
  if (rc) return rc;
  if (p.tokens == 0 || p.cols == 0) return HAP_OK;
  if (!grid_fits(p.tokens / 4 + 1)) return hap_fail(HAP_EUNSUPPORTED, "2^26 tokens and more");
  if (!ids || !Y || (p.rows > 0 && !W)) return hap_fail(HAP_EINVAL, "ids, W or Y is NULL");
  const int es = esize(d->io_dtype), V = 16 / es;
  const char* w = static_cast<const char*>(W) + w_offset(d, p) * es;
  char* y = static_cast<char*>(Y) + y_offset(d, p) * es;
  const int first = phase_of(w, y, es, es, V, d->ldw, d->ldy);
  const bool vec = first >= 0;
  if (first > 0) { w -= first * es; y -= first * es; }
  const Ids i = ids_of(d, p, ids);
  with_type(d->io_dtype, vec, [&](auto t, auto v) {
    using T = decltype(t);
    constexpr int N = decltype(v)::value;
    // Non-temporal stores from 80 MB on.  Write-through / non-temporal with a pass behind that reads the result and writes as much, bf16 rows of 2048 and of 5120, us:
    // 56 MB 36.1 / 37.9 and 37.5 / 40.6, 72 MB 45.6 / 46.5 and 49.0 / 51.4, 88 MB 59.3 / 56.0 and 63.2 / 61.4, 104 MB 73.0 / 67.2 and 76.7 / 73.6, 152 MB 106 / 106 and
    // 111 / 115, 256 MB 170 / 168 and 181 / 186, 400 MB 257 / 250 and 277 / 277, 800 MB 495 / 480 and 540 / 520: -8 to +3.4 % from 88 MB on, -1.4 % in the mean (wide rows
    // of 128 to 320 MB are those that lose).  Without a reader at once it takes less at every size (88 MB 27.9 / 26.5 and 33.2 / 29.6, 256 MB 76.2 / 73.9 and 92.0 / 76.7).
    const auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)((p.tokens + 3) / 4)), dim3(256), 0, (hipStream_t)stream, p.tokens, vec ? first : 0, (int)p.cols + (vec ? first : 0), i, reinterpret_cast<const T*>(w), d->ldw, d->scale,
                         reinterpret_cast<T*>(y), d->ldy);
    };
    if (N > 1 && (first > 0 || p.cols % N)) launch(embedding_fwd_kernel<T, N, false, (N > 1)>);
    else if (N > 1 && p.tokens * p.cols * es >= (int64_t)80 << 20) launch(embedding_fwd_kernel<T, N, (N > 1), false>);
    else launch(embedding_fwd_kernel<T, N, false, false>);
  });
  return check_launch("embedding_fwd");
}

size_t hap_embedding_bwd_workspace(const hap_embedding_desc* d, int shard_index) {
  Part p;
  if (resolve(d, shard_index, &p) != HAP_OK || p.tokens == 0 || p.rows == 0 || p.cols == 0) return 0;
  return (size_t)plan_of(p).bytes;
}

int hap_embedding_bwd(const hap_embedding_desc* d, int shard_index, const void* ids, const void* dY, void* dW, int dW_dtype, int accumulate,
                      void* ws, size_t ws_bytes, void* stream) {
  hap_clear_error();
  Part p;
  int rc = resolve(d, shard_index, &p);
  if (rc) return rc;
  if (dW_dtype != HAP_F32 && dW_dtype != HAP_BF16) return hap_fail(HAP_EINVAL, "bad dW_dtype %d", dW_dtype);
  if (d->io_dtype == HAP_F32 && dW_dtype != HAP_F32) return hap_fail(HAP_EINVAL, "fp32 table needs fp32 dW");
  if (p.rows == 0 || p.cols == 0 || (p.tokens == 0 && accumulate)) return HAP_OK;
  if (!dW || (p.tokens > 0 && (!ids || !dY))) return hap_fail(HAP_EINVAL, "ids, dY or dW is NULL");
  const Plan q = plan_of(p);
  if (p.tokens > 0 && (!ws || ws_bytes < (size_t)q.bytes)) return hap_fail(HAP_EWORKSPACE, "embedding_bwd needs %lld workspace bytes", (long long)q.bytes);
  if (p.tokens > 0 && (uintptr_t)ws % sizeof(uint32_t)) return hap_fail(HAP_EINVAL, "ws is not on a multiple of %zu bytes", sizeof(uint32_t));
  hipStream_t s = (hipStream_t)stream;
  const int es = esize(d->io_dtype), wes = esize(dW_dtype), V = 16 / wes;
  const char* y = static_cast<const char*>(dY) + y_offset(d, p) * es;
  char* w = static_cast<char*>(dW) + w_offset(d, p) * wes;
  const int first = phase_of(w, y, wes, es, V, d->ldw, d->ldy), from = first > 0 ? first : 0, cols = (int)p.cols + from, slab = 64 * (first >= 0 ? V : 1);
  const int64_t waves = (int64_t)q.chunks * ((cols + slab - 1) / slab);
  if (!grid_fits(waves)) return hap_fail(HAP_EUNSUPPORTED, "%lld chunks of 64 tokens and %d columns, 2^24 and more", (long long)waves, slab);
  const int64_t pitch = d->ldw * wes, width = p.cols * wes;
  const uintptr_t phase = (uintptr_t)w | (uintptr_t)pitch | (uintptr_t)width;
  const FillArgs f = {w, accumulate ? 0 : p.rows, pitch, (int)width, phase % 4 == 0 ? 4 : 2, fill_streamed(q, p.tokens, p.rows * width)};
  char* const b = static_cast<char*>(ws);
  SortArgs a = {p.tokens, (p.tokens + q.blocks - 1) / q.blocks, ids_of(d, p, ids), q.passes, q.bits, {}, {}, NULL};
  for (int i = 0; i < 2; ++i) {
    a.key[i] = reinterpret_cast<uint32_t*>(b + q.key[i]);
    a.token[i] = reinterpret_cast<uint32_t*>(b + q.token[i]);
  }
  a.before = reinterpret_cast<int*>(b + q.before);
  int sorted;
  if ((rc = sort_tokens(a, q, f, &sorted, s))) return rc;
  if (p.tokens == 0) return HAP_OK;
  if (first > 0) { w -= first * wes; y -= first * es; }
  SumArgs sum = {p.tokens, a.key[sorted], a.token[sorted], (uint32_t)p.rows, q.chunk, q.chunks, from, cols, first >= 0 ? (cols + V - 1) / V * V : cols, (cols + slab - 1) / slab,
                 reinterpret_cast<float*>(b + q.part), d->ldy, d->ldw, d->scale, accumulate != 0};
  const auto launch = [&](auto t, auto wt) {
    using T = decltype(t);
    using W = decltype(wt);
    const auto with = [&](auto v) {
      constexpr int N = decltype(v)::value;
      hipLaunchKernelGGL((embedding_sum_kernel<T, W, N>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, sum, reinterpret_cast<const T*>(y), reinterpret_cast<W*>(w));
      if (q.chunks > 1) hipLaunchKernelGGL((embedding_join_kernel<W, N>), dim3((unsigned)waves), dim3(256), 0, s, sum, reinterpret_cast<W*>(w));
    };
    if (first >= 0) with(std::integral_constant<int, 16 / (int)sizeof(W)>()); else with(std::integral_constant<int, 1>());
  };
  if (d->io_dtype == HAP_F32) launch(0.0f, 0.0f);
  else if (dW_dtype == HAP_F32) launch((__bf16)0.0f, 0.0f);
  else launch((__bf16)0.0f, (__bf16)0.0f);
  return check_launch("embedding_bwd");
}

}  // extern "C"
