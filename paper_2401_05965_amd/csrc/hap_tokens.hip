/*
 * The tokens' way to the experts and back on one device (Sec. 7.6; the exchange between devices is not part of this library):
 *
 *   plan       position[t][i]: the row that choice i of token t takes in its expert's buffer, in the order of (t, i); -1 where the buffer is full
 *   dispatch   X_e[position] = x[t];                        gradient  dx[t] = sum_i dX_e[position]
 *   combine    out[t] = sum_i w_i Y_e[position];            gradient  dY_e[position] = w_i dout[t],  dw_i = <dout[t], Y_e[position]>
 *
 * Bound: HBM.  One wave moves a token: it reads the token's row once whatever the number of choices, and the choices' rows, whose places are
 * known to the whole wave, in 16-byte chunks.  Walking tokens rather than buffer rows needs no table of what lies in a row, leaves rows behind
 * an expert's last alone by itself, and gives every sum a fixed order.
 */
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "hap_internal.h"
#include "hap_lanes.h"
#include "hap_sort.h"

namespace {

using namespace hap_lanes;

constexpr int kMaxExperts = 1024, kMaxTopK = 64;

struct PlanArgs {
  int64_t slots, per_block;            // choices in all, and of a workgroup
  int experts, capacity, bits;
  const int* indices;
  int *position, *rows, *counts, *before;      // before: [workgroups][experts] counts, NULL for a single workgroup
};

__device__ __forceinline__ int expert_of(const PlanArgs& a, int index) { return (unsigned)index < (unsigned)a.experts ? index : -1; }

__global__ __launch_bounds__(hap_sort::kThreads) void plan_count_kernel(const PlanArgs a) {
  extern __shared__ int lds[];
  hap_sort::lds_int* const count = (hap_sort::lds_int*)lds;
  const int64_t begin = (int64_t)blockIdx.x * a.per_block, end = begin + a.per_block < a.slots ? begin + a.per_block : a.slots;
  hap_sort::count_keys(count, a.experts, begin, end, [&](int64_t n) { return a.indices[n]; }, [&](int v) { return expert_of(a, v); });
  for (int e = threadIdx.x; e < a.experts; e += hap_sort::kThreads) {
    int s = 0;
    for (int w = 0; w < hap_sort::kWaves; ++w) s += count[w * a.experts + e];
    a.before[(int64_t)blockIdx.x * a.experts + e] = s;
  }
}

/* Choices of every expert in the workgroups before this one into total[expert] (zeros before), from the counts that plan_count_kernel left: the waves take every
 * sixteenth workgroup, several loads in flight. */
__device__ __forceinline__ void sum_before(const PlanArgs& a, hap_sort::lds_int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int e = lane; e < a.experts; e += 64) {
    int s = 0;
#pragma unroll 4
    for (int b = wave; b < (int)blockIdx.x; b += hap_sort::kWaves) s += a.before[(int64_t)b * a.experts + e];
    if (s) __hip_atomic_fetch_add(&total[e], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
}

/* A workgroup takes kPlanRounds rounds per wave, whose experts and ranks stay in registers between counting and placing.  Without counts of the workgroups before
 * (up to kPlanDirect choices: one launch) it counts their choices itself, in four copies (lanes that meet in one word go one by one). */
constexpr int kPlanRounds = 4;
__global__ __launch_bounds__(hap_sort::kThreads) void plan_direct_kernel(const PlanArgs a) {
  using namespace hap_sort;
  extern __shared__ int lds[];
  lds_int *const count = (lds_int*)lds, *const total = count + kWaves * a.experts;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t begin = (int64_t)blockIdx.x * a.per_block, end = begin + a.per_block < a.slots ? begin + a.per_block : a.slots;
  int64_t lo, hi;
  part_of(begin, end, &lo, &hi);
  int key[kPlanRounds], rank[kPlanRounds];
  if (lo < hi) {
#pragma unroll
    for (int i = 0; i < kPlanRounds; ++i) {
      const int64_t n = lo + i * 64 + lane;
      key[i] = a.indices[n < hi ? n : hi - 1];
    }
  }
  for (int i = threadIdx.x; i < (kWaves + 4) * a.experts; i += kThreads) count[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPlanRounds; ++i)
    if (lo + i * 64 < hi) rank[i] = take_place(count + wave * a.experts, lo + i * 64 + lane < hi ? expert_of(a, key[i]) : -1, a.bits);
  if (a.before) {
    sum_before(a, total);
  } else if (begin > 0) {
    int64_t from, to;
    part_of(0, begin, &from, &to);
    rounds(from, to, [&](int64_t n) { return a.indices[n]; }, [&](int64_t, int v, bool entry) {
      const int e = entry ? expert_of(a, v) : -1;
      if (e >= 0) __hip_atomic_fetch_add(&total[(lane & 3) * a.experts + e], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    });
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    const int next = first_places(count, a.experts, e, (total[e] + total[a.experts + e]) + (total[2 * a.experts + e] + total[3 * a.experts + e]));
    if (blockIdx.x == gridDim.x - 1) {
      if (a.counts) a.counts[e] = next;
      a.rows[e] = next < a.capacity ? next : a.capacity;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPlanRounds; ++i) {
    const int64_t n = lo + i * 64 + lane;
    if (n < hi) {
      const int p = rank[i] < 0 ? -1 : count[wave * a.experts + key[i]] + rank[i];
      a.position[n] = p < a.capacity ? p : -1;
    }
  }
}

/* Batches of more than kPlanMost such workgroups: each takes a longer range and walks it twice. */
__global__ __launch_bounds__(hap_sort::kThreads) void plan_kernel(const PlanArgs a) {
  using namespace hap_sort;
  extern __shared__ int lds[];
  lds_int *const count = (lds_int*)lds, *const total = count + kWaves * a.experts;
  const int64_t begin = (int64_t)blockIdx.x * a.per_block, end = begin + a.per_block < a.slots ? begin + a.per_block : a.slots;
  const auto load = [&](int64_t n) { return a.indices[n]; };
  const auto key_of = [&](int v) { return expert_of(a, v); };
  for (int e = threadIdx.x; e < a.experts; e += kThreads) total[e] = 0;
  count_keys(count, a.experts, begin, end, load, key_of);
  sum_before(a, total);
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    const int next = first_places(count, a.experts, e, total[e]);
    if (blockIdx.x == gridDim.x - 1) {
      if (a.counts) a.counts[e] = next;
      a.rows[e] = next < a.capacity ? next : a.capacity;
    }
  }
  __syncthreads();
  place_keys(count, a.experts, a.bits, begin, end, load, key_of, [&](int64_t n, int, int p) { a.position[n] = p < a.capacity ? p : -1; });
}

struct TokenArgs {
  int64_t tokens, ldt, lde, capacity;
  int features, top_k, lo, n;          // experts lo .. lo + n
  const int *indices, *position;
};

/* Element offset of the buffer row of lane i's choice, from the first expert of the device; -1 where the choice has no row here. */
__device__ __forceinline__ int64_t row_of_choice(const TokenArgs& a, int64_t t, int lane) {
  if (lane >= a.top_k) return -1;
  const unsigned e = (unsigned)a.indices[t * a.top_k + lane] - (unsigned)a.lo;
  const int p = a.position[t * a.top_k + lane];
  return e < (unsigned)a.n && p >= 0 && p < a.capacity ? ((int64_t)e * a.capacity + p) * a.lde : -1;
}

/* The token of this wave. */
__device__ __forceinline__ int64_t token_of_wave() { return (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

/* The token's values are on their way before its choices are known. */
template <typename T, int V, bool STREAM, bool CUT>
__global__ __launch_bounds__(256) void dispatch_fwd_kernel(const TokenArgs a, const T* x, T* X) {
  constexpr int U = 4, STEP = 64 * V;
  const int lane = threadIdx.x & 63, bytes = chunk_bytes<T, V>(a.features);
  const int64_t t = token_of_wave();
  if (t >= a.tokens) return;
  const auto from = row_at(x + t * a.ldt, bytes);
  Pack<T, V> p[U];
#pragma unroll
  for (int u = 0; u < U; ++u) p[u] = row_load<T, V>(from, lane * V + u * STEP);
  const int64_t row = row_of_choice(a, t, lane);
  const uint64_t live = __ballot(row >= 0);
  if (!live) return;
  for (int c = lane * V;;) {
    for (uint64_t m = live; m; m &= m - 1) {
      const auto to = row_at(X + from_lane(row, __builtin_ctzll(m)), bytes);
#pragma unroll
      for (int u = 0; u < U; ++u) row_store_part<STREAM, CUT>(to, c + u * STEP, p[u], 0, a.features);
    }
    c += U * STEP;
    if (c - lane * V >= a.features) break;
#pragma unroll
    for (int u = 0; u < U; ++u) p[u] = row_load<T, V>(from, c + u * STEP);
  }
}

/* out[t] = sum over the choices of w_i Y[row_i] (dispatch's gradient: without weights).  fp32 sums in the order of i, rounded once.  K choices' rows,
 * U chunks each, are in flight together; a choice that is not there reads as a row without bytes. */
template <typename T, int V, int K, bool WEIGHTED, bool CUT>
__global__ __launch_bounds__(256) void combine_fwd_kernel(const TokenArgs a, const T* Y, const float* weights, T* out) {
  constexpr int U = 2, STEP = 64 * V;
  const int lane = threadIdx.x & 63, bytes = chunk_bytes<T, V>(a.features);
  const int64_t t = token_of_wave();
  if (t >= a.tokens) return;
  const float given = WEIGHTED && lane < a.top_k ? weights[t * a.top_k + lane] : 0.0f;
  const int64_t row = row_of_choice(a, t, lane);
  const float w = row >= 0 ? given : 0.0f;
  const uint64_t live = __ballot(row >= 0);
  const auto to = row_at(out + t * a.ldt, bytes);
  for (int c0 = 0; c0 < a.features; c0 += U * STEP) {
    const int c = c0 + lane * V;
    float s[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int v = 0; v < V; ++v) s[u][v] = 0.0f;
    for (uint64_t m = live; m;) {
      Pack<T, V> p[K][U];
      float wi[K];
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int i = m ? __builtin_ctzll(m) : 0;
        const auto from = row_at(Y + (m ? from_lane(row, i) : 0), m ? bytes : 0);
        wi[k] = m ? from_lane(w, i) : 0.0f;
        m &= m - 1;                    // (0 stays 0)
#pragma unroll
        for (int u = 0; u < U; ++u) p[k][u] = row_load<T, V>(from, c + u * STEP);
      }
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int v = 0; v < V; ++v) s[u][v] = WEIGHTED ? fmaf(wi[k], to_f32(p[k][u].v[v]), s[u][v]) : s[u][v] + to_f32(p[k][u].v[v]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Pack<T, V> o;
#pragma unroll
      for (int v = 0; v < V; ++v) o.v[v] = (T)s[u][v];
      row_store_part<false, CUT>(to, c + u * STEP, o, 0, a.features);
    }
  }
}

/* Two choices at a time, whose sums run through the whole row: dout is read again for the next two (from the caches). */
template <typename T, int V, bool CUT>
__global__ __launch_bounds__(256) void combine_bwd_kernel(const TokenArgs a, const T* Y, const float* weights, const T* dout, T* dY, float* dweights) {
  constexpr int U = 2, STEP = 64 * V;
  const int lane = threadIdx.x & 63, bytes = chunk_bytes<T, V>(a.features);
  const int64_t t = token_of_wave();
  if (t >= a.tokens) return;
  const auto from = row_at(dout + t * a.ldt, bytes);
  const float given = lane < a.top_k ? weights[t * a.top_k + lane] : 0.0f;
  const int64_t row = row_of_choice(a, t, lane);
  const float w = row >= 0 ? given : 0.0f;
  float dw = 0.0f;                     // lane i: its choice's sum
  for (uint64_t m = __ballot(row >= 0); m;) {
    const int i = __builtin_ctzll(m);
    m &= m - 1;
    const bool two = m != 0;
    const int j = two ? __builtin_ctzll(m) : i;
    m &= m - 1;
    const int64_t ri = from_lane(row, i), rj = from_lane(row, j);
    const float wi = from_lane(w, i), wj = from_lane(w, j);
    const auto yi = row_at(Y + ri, bytes), yj = row_at(Y + rj, two ? bytes : 0);
    const auto di = row_at(dY + ri, dY ? bytes : 0), dj = row_at(dY + rj, dY && two ? bytes : 0);
    float si = 0.0f, sj = 0.0f;
    for (int c0 = 0; c0 < a.features; c0 += U * STEP) {
      const int c = c0 + lane * V;
      Pack<T, V> g[U], p[U], q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        g[u] = row_load<T, V>(from, c + u * STEP);
        p[u] = row_load<T, V>(yi, c + u * STEP);
        q[u] = row_load<T, V>(yj, c + u * STEP);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (CUT && c + u * STEP + V > a.features) {                // what lies behind the rows' ends takes no part in the sums
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (c + u * STEP + v >= a.features) g[u].v[v] = p[u].v[v] = q[u].v[v] = (T)0.0f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float x = to_f32(g[u].v[v]);
          si = fmaf(x, to_f32(p[u].v[v]), si);
          sj = fmaf(x, to_f32(q[u].v[v]), sj);
          p[u].v[v] = (T)(wi * x);
          q[u].v[v] = (T)(wj * x);
        }
        row_store_part<false, CUT>(di, c + u * STEP, p[u], 0, a.features);      // (without dY, without a second choice: rows without bytes)
        row_store_part<false, CUT>(dj, c + u * STEP, q[u], 0, a.features);
      }
    }
    si = sum<64>(si);
    sj = sum<64>(sj);
    if (lane == i) dw = si;
    if (two && lane == j) dw = sj;
  }
  if (dweights && lane < a.top_k) dweights[t * a.top_k + lane] = dw;
}

inline int check_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? HAP_OK : hap_fail(HAP_EDEVICE, "%s launch: %s", what, hipGetErrorString(e));
}

inline int esize(int dtype) { return dtype == HAP_BF16 ? 2 : 4; }

/* Up to kPlanDirect choices go in one launch, beyond in two; up to kPlanMost workgroups of kPlanRounds rounds, longer ones beyond.  us, in one launch / in two: 32768 choices
 * of 30 experts 8.8 / 11.6. */
constexpr int64_t kPlanDirect = 32768, kPlanMost = 256, kPlanRange = kPlanRounds * hap_sort::kThreads;
inline int64_t plan_blocks(int64_t slots) {
  const int64_t n = (slots + kPlanRange - 1) / kPlanRange;
  return n < 1 ? 1 : n < kPlanMost ? n : kPlanMost;
}

int plan_check(int64_t tokens, int top_k, int64_t experts) {
  if (tokens < 0 || top_k < 1 || experts < 1) return hap_fail(HAP_EINVAL, "bad sizes");
  if (experts > kMaxExperts || top_k > kMaxTopK) return hap_fail(HAP_EUNSUPPORTED, "more than %d experts or %d choices", kMaxExperts, kMaxTopK);
  if (tokens > 0x7fffffff / top_k) return hap_fail(HAP_EUNSUPPORTED, "more than 2^31 choices");
  return HAP_OK;
}

/* What every movement checks, and the kernels' arguments.  *first: elements from the buffers' start to the device's first expert. */
int resolve(const hap_moe_tokens_desc* d, int j, TokenArgs* a, int64_t* first) {
  if (!d) return hap_fail(HAP_EINVAL, "descriptor is NULL");
  int rc = plan_check(d->tokens, d->top_k, d->experts);
  if (rc) return rc;
  if (!grid_fits(d->tokens / 4 + 1)) return hap_fail(HAP_EUNSUPPORTED, "2^26 tokens and more");
  if (d->capacity < 0 || d->features < 1) return hap_fail(HAP_EINVAL, "bad sizes");
  if (d->io_dtype != HAP_F32 && d->io_dtype != HAP_BF16) return hap_fail(HAP_EINVAL, "bad io_dtype %d", d->io_dtype);
  int64_t lo, hi;
  if ((rc = hap_shard_range(d->m, d->offsets, d->experts, j, &lo, &hi))) return rc;
  if (d->ldt < d->features || d->lde < d->features) return hap_fail(HAP_ESHAPE, "leading dimension below %lld features", (long long)d->features);
  if (d->capacity > 0x7fffffff || d->features > 0xfffffff) return hap_fail(HAP_EUNSUPPORTED, "capacity beyond 2^31 or features beyond 2^28");
  *a = TokenArgs{d->tokens, d->ldt, d->lde, d->capacity, (int)d->features, d->top_k, (int)lo, (int)(hi - lo), NULL, NULL};
  *first = d->operands_are_full ? lo * d->capacity * d->lde : 0;
  return HAP_OK;
}

/* Whether all rows take 16-byte chunks; the last one of a row may be cut (what lies behind it is within the row's pitch). */
inline bool vectors(const TokenArgs& a, int dtype, const void* p, const void* q, const void* r, const void* s) {
  const int V = 16 / esize(dtype);
  return a.ldt % V == 0 && a.lde % V == 0 && (((uintptr_t)p | (uintptr_t)q | (uintptr_t)r | (uintptr_t)s) & 15) == 0;
}

/* Whether rows end inside a chunk of V. */
inline bool cut(const TokenArgs& a, int V) { return a.features % V != 0; }

template <typename F> void with_type(int dtype, bool vec, F&& f) {
  if (dtype == HAP_BF16) {
    if (vec) f((__bf16)0.0f, std::integral_constant<int, 8>()); else f((__bf16)0.0f, std::integral_constant<int, 1>());
  } else {
    if (vec) f(0.0f, std::integral_constant<int, 4>()); else f(0.0f, std::integral_constant<int, 1>());
  }
}

inline dim3 token_grid(const TokenArgs& a) { return dim3((unsigned)((a.tokens + 3) / 4)); }

/* Whether dispatch stores non-temporally: where the choices can fill more than 300 MB of the device's buffers (the last-level cache holds 256).  Write-through /
 * non-temporal, alone and with the experts' product that reads the buffers (bf16, eight choices): 268 MB 60.5 / 53.0 and 354 / 358 us, 403 MB 89.0 / 76.7 and 502 / 496,
 * 537 MB 117 / 102 and 631 / 628, 805 MB 181 / 154 and 984 / 983, 1074 MB 236 / 210 and 1249 / 1258; two choices, 537 MB 153 / 153 and 2150 / 2151: a gain of up to 15 % where
 * the product does not follow at once (an exchange between devices comes first), and within its runs' spread where it does.  Combine's gradient gains nothing either way
 * (403 MB 174 / 172 and 575 / 575, 1074 MB 459 / 455 and 1460 / 1461). */
inline bool buffers_streamed(const TokenArgs& a, size_t es) {
  const int64_t rows = a.tokens * a.top_k < a.n * a.capacity ? a.tokens * a.top_k : a.n * a.capacity;
  return rows * a.features * (int64_t)es > (int64_t)300 << 20;
}

template <typename T> T* shift(T* p, int64_t elems, int dtype) {
  using byte = typename std::conditional<std::is_const<T>::value, const char, char>::type;
  return p ? static_cast<T*>(static_cast<byte*>(p) + elems * esize(dtype)) : p;
}

}  // namespace

extern "C" {

size_t hap_moe_plan_workspace(int64_t tokens, int top_k, int64_t experts) {
  if (plan_check(tokens, top_k, experts) != HAP_OK) return 0;
  return tokens * top_k > kPlanDirect ? (size_t)(plan_blocks(tokens * top_k) * experts) * sizeof(int) : 0;
}

int hap_moe_plan(int64_t tokens, int top_k, int64_t experts, int64_t capacity, const int32_t* indices, int32_t* position, int32_t* rows,
                 int32_t* counts, void* ws, size_t ws_bytes, void* stream) {
  hap_clear_error();
  const int rc = plan_check(tokens, top_k, experts);
  if (rc) return rc;
  if (capacity < 0) return hap_fail(HAP_EINVAL, "negative capacity");
  if (capacity > 0x7fffffff) return hap_fail(HAP_EUNSUPPORTED, "capacity beyond 2^31");
  if (!rows || (tokens > 0 && (!indices || !position))) return hap_fail(HAP_EINVAL, "indices, position or rows is NULL");
  const size_t need = hap_moe_plan_workspace(tokens, top_k, experts);
  if (need && (!ws || ws_bytes < need)) return hap_fail(HAP_EWORKSPACE, "moe_plan needs %zu workspace bytes", need);
  if (need && (uintptr_t)ws % sizeof(int)) return hap_fail(HAP_EINVAL, "ws is not on a multiple of %zu bytes", sizeof(int));
  const int64_t slots = tokens * top_k, blocks = plan_blocks(slots);
  const bool direct = slots <= kPlanDirect, ranges = slots > kPlanMost * kPlanRange;
  PlanArgs a = {slots, ranges ? (slots + blocks - 1) / blocks : kPlanRange, (int)experts, (int)capacity, 0, indices, position, rows, counts, direct ? NULL : static_cast<int*>(ws)};
  while ((1 << a.bits) < experts) ++a.bits;
  const size_t row = (size_t)experts * sizeof(int), most = (hap_sort::kWaves + 4) * kMaxExperts * sizeof(int);
  hipStream_t s = (hipStream_t)stream;
  static bool configured[2][64];
  if (!direct) {
    hipLaunchKernelGGL(plan_count_kernel, dim3((unsigned)blocks), dim3(hap_sort::kThreads), hap_sort::kWaves * row, s, a);
    if (const int e = check_launch("moe_plan count")) return e;
  }
  const size_t lds = (hap_sort::kWaves + (ranges ? 1 : 4)) * row;
  const auto kernel = ranges ? plan_kernel : plan_direct_kernel;
  if (const int e = hap_sort::reserve_lds(reinterpret_cast<const void*>(kernel), configured[ranges], lds, most)) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(hap_sort::kThreads), lds, s, a);
  return check_launch("moe_plan");
}

int hap_moe_dispatch_fwd(const hap_moe_tokens_desc* d, int shard_index, const void* x, const int32_t* indices, const int32_t* position, void* X, void* stream) {
  hap_clear_error();
  TokenArgs a;
  int64_t first;
  const int rc = resolve(d, shard_index, &a, &first);
  if (rc) return rc;
  if (a.n == 0 || a.tokens == 0 || a.capacity == 0) return HAP_OK;
  if (!x || !indices || !position || !X) return hap_fail(HAP_EINVAL, "x, indices, position or X is NULL");
  a.indices = indices; a.position = position;
  X = shift(X, first, d->io_dtype);
  with_type(d->io_dtype, vectors(a, d->io_dtype, x, X, NULL, NULL), [&](auto t, auto v) {
    using T = decltype(t);
    constexpr int V = decltype(v)::value;
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, token_grid(a), dim3(256), 0, (hipStream_t)stream, a, (const T*)x, (T*)X); };
    if (cut(a, V)) launch(dispatch_fwd_kernel<T, V, false, (V > 1)>);
    else if (V > 1 && buffers_streamed(a, sizeof(T))) launch(dispatch_fwd_kernel<T, V, (V > 1), false>);
    else launch(dispatch_fwd_kernel<T, V, false, false>);
  });
  return check_launch("moe_dispatch_fwd");
}

/* combine's forward, or (without weights) dispatch's gradient: a device without rows still owes its partial sum, zeros. */
static int gather_sum(const hap_moe_tokens_desc* d, int shard_index, const void* Y, const int32_t* indices, const int32_t* position, bool weighted,
                      const float* weights, void* out, void* stream, const char* what) {
  TokenArgs a;
  int64_t first;
  const int rc = resolve(d, shard_index, &a, &first);
  if (rc) return rc;
  if (a.tokens == 0) return HAP_OK;
  const bool rows = a.n > 0 && a.capacity > 0;
  if (!out || !indices || !position || (rows && !Y) || (weighted && !weights)) return hap_fail(HAP_EINVAL, "NULL pointer");
  if (!rows) a.n = 0;
  a.indices = indices; a.position = position;
  Y = shift(Y, first, d->io_dtype);
  with_type(d->io_dtype, vectors(a, d->io_dtype, Y, out, NULL, NULL), [&](auto t, auto v) {
    using T = decltype(t);
    constexpr int V = decltype(v)::value;
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, token_grid(a), dim3(256), 0, (hipStream_t)stream, a, (const T*)Y, weights, (T*)out); };
    const auto choose = [&](auto k, auto w) {
      constexpr int K = decltype(k)::value;
      constexpr bool WEIGHTED = decltype(w)::value;
      if (cut(a, V)) launch(combine_fwd_kernel<T, V, K, WEIGHTED, (V > 1)>); else launch(combine_fwd_kernel<T, V, K, WEIGHTED, false>);
    };
    const auto with_k = [&](auto w) { if (a.top_k <= 2) choose(std::integral_constant<int, 2>(), w); else choose(std::integral_constant<int, 4>(), w); };
    if (weighted) with_k(std::true_type()); else with_k(std::false_type());
  });
  return check_launch(what);
}

int hap_moe_dispatch_bwd(const hap_moe_tokens_desc* d, int shard_index, const void* dX, const int32_t* indices, const int32_t* position, void* dx, void* stream) {
  hap_clear_error();
  return gather_sum(d, shard_index, dX, indices, position, false, NULL, dx, stream, "moe_dispatch_bwd");
}

int hap_moe_combine_fwd(const hap_moe_tokens_desc* d, int shard_index, const void* Y, const int32_t* indices, const int32_t* position,
                        const float* weights, void* out, void* stream) {
  hap_clear_error();
  return gather_sum(d, shard_index, Y, indices, position, true, weights, out, stream, "moe_combine_fwd");
}

int hap_moe_combine_bwd(const hap_moe_tokens_desc* d, int shard_index, const void* Y, const int32_t* indices, const int32_t* position,
                        const float* weights, const void* dout, void* dY, float* dweights, void* stream) {
  hap_clear_error();
  TokenArgs a;
  int64_t first;
  const int rc = resolve(d, shard_index, &a, &first);
  if (rc) return rc;
  if (a.tokens == 0 || (!dY && !dweights)) return HAP_OK;
  const bool rows = a.n > 0 && a.capacity > 0;
  if (!indices || !position || !weights || !dout || (rows && !Y)) return hap_fail(HAP_EINVAL, "NULL pointer");
  if (!rows) a.n = 0;
  a.indices = indices; a.position = position;
  Y = shift(Y, first, d->io_dtype); dY = shift(dY, first, d->io_dtype);
  with_type(d->io_dtype, vectors(a, d->io_dtype, Y, dout, dY, NULL), [&](auto t, auto v) {
    using T = decltype(t);
    constexpr int V = decltype(v)::value;
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, token_grid(a), dim3(256), 0, (hipStream_t)stream, a, (const T*)Y, weights, (const T*)dout, (T*)dY, dweights); };
    if (cut(a, V)) launch(combine_bwd_kernel<T, V, (V > 1)>); else launch(combine_bwd_kernel<T, V, false>);
  });
  return check_launch("moe_combine_bwd");
}

}  // extern "C"
