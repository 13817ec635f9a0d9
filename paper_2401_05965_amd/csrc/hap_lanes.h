/* Exchanges between the lanes of a wavefront and vector accesses, for the row kernels around the experts and the embedding table. */
#ifndef HAP_LANES_H
#define HAP_LANES_H

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace hap_lanes {

/* T in LDS, said to be there: behind a plain pointer that a function was handed the compiler may take it for any memory, and lanes of one wave that
 * exchange through LDS rely on its operations keeping their order. */
template <typename T> using in_lds = __attribute__((address_space(3))) T;

/* V elements of T moved as one access. */
template <typename T, int V> struct Pack { T v[V]; } __attribute__((aligned(sizeof(T) * V)));

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }

/* The value of the partner lane in step S of a butterfly (S = 1, 2, 4, ... 32) over lanes that already agree within groups of S: any lane of
 * the neighbouring group will do, so that the steps up to 8 are DPP moves inside a row of 16 lanes (mirrors) and the two above swap halves;
 * none goes through LDS as a general shuffle does. */
template <int S> __device__ __forceinline__ uint32_t partner(uint32_t v) {
  static_assert(S == 1 || S == 2 || S == 4 || S == 8 || S == 16 || S == 32, "a butterfly step");
  if constexpr (S == 1) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true);          // quad_perm 1,0,3,2
  else if constexpr (S == 2) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true);     // quad_perm 2,3,0,1
  else if constexpr (S == 4) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true);    // row_half_mirror
  else if constexpr (S == 8) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true);    // row_mirror
  else if constexpr (S == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return (threadIdx.x & 16) ? r[0] : r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (threadIdx.x & 32) ? r[0] : r[1];
  }
}
template <int S> __device__ __forceinline__ uint64_t partner(uint64_t v) {
  return (uint64_t)partner<S>((uint32_t)(v >> 32)) << 32 | partner<S>((uint32_t)v);
}

template <int S> __device__ __forceinline__ double partner(double v) { return __longlong_as_double((long long)partner<S>((uint64_t)__double_as_longlong(v))); }

/* This lane's value and its partner's, in either order, where swapping halves leaves both: a commutative fold needs to know no more. */
template <int S> __device__ __forceinline__ void pair(uint32_t v, uint32_t* a, uint32_t* b) {
  if constexpr (S == 16) { const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false); *a = r[0]; *b = r[1]; }
  else if constexpr (S == 32) { const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false); *a = r[0]; *b = r[1]; }
  else { *a = v; *b = partner<S>(v); }
}
template <int S> __device__ __forceinline__ void pair(float v, float* a, float* b) {
  uint32_t x, y;
  pair<S>(__float_as_uint(v), &x, &y);
  *a = __uint_as_float(x); *b = __uint_as_float(y);
}
template <int S> __device__ __forceinline__ void pair(uint64_t v, uint64_t* a, uint64_t* b) {
  uint32_t xl, yl, xh, yh;
  pair<S>((uint32_t)v, &xl, &yl); pair<S>((uint32_t)(v >> 32), &xh, &yh);
  *a = (uint64_t)xh << 32 | xl; *b = (uint64_t)yh << 32 | yl;
}
template <int S> __device__ __forceinline__ void pair(double v, double* a, double* b) {
  uint64_t x, y;
  pair<S>((uint64_t)__double_as_longlong(v), &x, &y);
  *a = __longlong_as_double((long long)x); *b = __longlong_as_double((long long)y);
}

/* Folds v by a commutative f over groups of L consecutive lanes (L a power of two up to 64); every lane of a group gets the result. */
template <int L, int S = 1, typename T, typename F> __device__ __forceinline__ T fold(T v, F&& f) {
  if constexpr (S < L) {
    T a, b;
    pair<S>(v, &a, &b);
    v = f(a, b);
    return fold<L, S * 2>(v, f);
  } else {
    return v;
  }
}
template <int L, typename T> __device__ __forceinline__ T sum(T v) { return fold<L>(v, [](T a, T b) { return a + b; }); }

/* Sum of the values of this lane and the lower ones: DPP shifts within rows of 16 lanes, then the rows' last lanes to the rows behind (missing ones read as 0). */
__device__ __forceinline__ int sum_up_to_lane(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast 15 to rows 1 and 3, row_bcast 31 to rows 2 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

/* The lowest of the L lanes around this one (counted from their first) whose bit is set in a ballot; one of them is. */
template <int L> __device__ __forceinline__ int lowest_lane(uint64_t ballot) {
  if constexpr (L == 64) return __builtin_ctzll(ballot);
  else return __builtin_ctz(((threadIdx.x & 32) ? (uint32_t)(ballot >> 32) : (uint32_t)ballot) >> (threadIdx.x & 31 & ~(unsigned)(L - 1)));
}

/* Lane i's value, i the same in all lanes. */
__device__ __forceinline__ uint32_t from_lane(uint32_t v, int i) { return (uint32_t)__builtin_amdgcn_readlane((int)v, i); }
__device__ __forceinline__ int from_lane(int v, int i) { return __builtin_amdgcn_readlane(v, i); }
__device__ __forceinline__ float from_lane(float v, int i) { return __uint_as_float(from_lane(__float_as_uint(v), i)); }
__device__ __forceinline__ int64_t from_lane(int64_t v, int i) {
  return (int64_t)((uint64_t)from_lane((uint32_t)((uint64_t)v >> 32), i) << 32 | from_lane((uint32_t)v, i));
}

/* The lanes whose key equals this lane's, among those of `active`; bits <= MOST: how many low bits of the keys differ at all. */
template <int MOST> __device__ __forceinline__ uint64_t same_key(uint32_t key, int bits, uint64_t active) {
  uint32_t lo = (uint32_t)active, hi = (uint32_t)(active >> 32);
#pragma unroll
  for (int b = 0; b < MOST; ++b) {
    if (b < bits) {
      const uint32_t bit = (key >> b) & 1;
      const uint64_t ones = __ballot(bit);
      const uint32_t flip = bit - 1u;               // all ones where the bit is 0: the lanes wanted are those without it
      lo &= (uint32_t)ones ^ flip;
      hi &= (uint32_t)(ones >> 32) ^ flip;
    }
  }
  return (uint64_t)hi << 32 | lo;
}

/* ---- rows that a whole wave reads or writes, through buffer descriptors
 *
 * Reads behind the row's end give zeros and writes there do nothing, so that a wave can have several chunks of a row of any length in flight without
 * a branch between the loads: behind a condition, the compiler waits for each before it issues the next (dispatch of 16384 tokens of 768 values
 * to two experts each: 25 -> 10 us).  A row's address has to be the same in all lanes; a row has less than 2^31 bytes. */
template <typename T> __device__ __forceinline__ T* uniform(T* p) {
  const uint64_t v = (uint64_t)p;
  return (T*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_at(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(uniform(p)), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);      // raw, 32-bit data format
}

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

template <typename T, int V> __device__ __forceinline__ Pack<T, V> row_load(__amdgpu_buffer_rsrc_t row, int element) {
  const int at = element * (int)sizeof(T);
  if constexpr (sizeof(Pack<T, V>) == 16) return __builtin_bit_cast(Pack<T, V>, __builtin_amdgcn_raw_buffer_load_b128(row, at, 0, 0));
  else if constexpr (sizeof(Pack<T, V>) == 8) return __builtin_bit_cast(Pack<T, V>, __builtin_amdgcn_raw_buffer_load_b64(row, at, 0, 0));
  else if constexpr (sizeof(Pack<T, V>) == 4) return __builtin_bit_cast(Pack<T, V>, __builtin_amdgcn_raw_buffer_load_b32(row, at, 0, 0));
  else return __builtin_bit_cast(Pack<T, V>, __builtin_amdgcn_raw_buffer_load_b16(row, at, 0, 0));
}

/* Whole chunks are written through to the level that all XCDs share (sc1) while the line stays where the next kernel can find it: at a kernel's end its
 * XCD's L2 then has nothing left to write back.  Plain, non-temporal and write-through stores, dispatch alone and with the experts' product behind it: 16384 x 768 to two of
 * thirty 10.9, 10.6, 10.1 us and 134.6, 137.6, 129.7; 4096 x 1024 to two of eight 5.7, 4.5, 4.3 and 97.1, 98.6, 94.0; 8192 x 2048 to two of sixteen
 * 15.9, 14.1, 15.0 and 114.0, 134.7, 106.5.  STREAM: non-temporal, for outputs that the last-level cache would not hold until they are read. */
template <bool STREAM, typename T, int V> __device__ __forceinline__ void row_store(__amdgpu_buffer_rsrc_t row, int element, const Pack<T, V>& p) {
  const int at = element * (int)sizeof(T);
  if constexpr (sizeof(Pack<T, V>) == 16) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, p), row, at, 0, STREAM ? 2 : 16);
  else if constexpr (sizeof(Pack<T, V>) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned int, p), row, at, 0, 0);
  else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(short, p), row, at, 0, 0);
}

/* A chunk of which only the elements in [first, last) belong to the row: CUT, a row whose chunks are aligned may begin and end inside one (without: 16384 tokens'
 * combine gradient 18.3 -> 15.8 us). */
template <bool STREAM, bool CUT, typename T, int V> __device__ __forceinline__ void row_store_part(__amdgpu_buffer_rsrc_t row, int element, const Pack<T, V>& p, int first, int last) {
  if (!CUT || (element >= first && element + V <= last)) {
    row_store<STREAM>(row, element, p);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (element + v >= first && element + v < last) row_store<STREAM>(row, element + v, Pack<T, 1>{{p.v[v]}});
  }
}

/* A grid has fewer than 2^32 threads: what workgroups of 256 can be launched. */
inline bool grid_fits(int64_t workgroups) { return workgroups < (int64_t)1 << 24; }

/* Bytes of `count` elements in whole chunks of V. */
template <typename T, int V> __device__ __forceinline__ int chunk_bytes(int count) { return (count + V - 1) / V * V * (int)sizeof(T); }

}  // namespace hap_lanes

#endif
