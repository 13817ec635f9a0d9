/*
 * The norm over all gradients that a device holds, and their scaling where it is too large:
 *
 *   sumsq = sum over the tensors of g^2      (fp64; the devices' values are added up by an All-Reduce of one number)
 *   norm = sqrt(sumsq),  out = g * min(1, max_norm / norm)
 *
 * Squares and sums are fp64: a square of an fp32 value is exact there and cannot overflow, and half a billion terms lose nothing.
 *
 * Bound: HBM, one read for the norm, one read and one write for the scaling.  All tensors of a launch are cut into items of about 8192 values
 * (whole rows of a matrix with a pitch, stretches of a contiguous one) that the workgroups stride over, so that large and small tensors share
 * the chip; the table of tensors travels in the kernel's arguments, kBatch of them a launch.  A thread has four 16-byte chunks of an item in flight, fetched
 * through a buffer descriptor without a condition between them (an index behind the item reads as zeros).  Partial sums have fixed places: the same bits in
 * every run.
 */
#include <hip/hip_runtime.h>

#include <stdint.h>
#include <stdlib.h>

#include <type_traits>

#include "hap_internal.h"
#include "hap_lanes.h"

namespace {

using namespace hap_lanes;

constexpr int kBatch = 100;            // tensors of a launch: as many as 4 KB of arguments hold
constexpr int kSpan = 8192;            // values of an item
constexpr int kBlocks = 2048;          // workgroups of a launch, at most
constexpr int kUnroll = 4;

struct Tensor {
  const char* g;                       // moved down by `skew` elements to a 16-byte boundary
  char* out;
  union {
    int64_t values;                    // a contiguous tensor: cut into rows of kSpan values
    struct { int rows, cols, ld, ldo; } m;
  };
};
struct Table {
  int n, items;
  int first[kBatch];                   // first item of each tensor
  uint16_t per_item[kBatch];           // rows of an item; 0: a contiguous tensor, a row each
  int8_t skew[kBatch];                 // < 0: values one by one
  uint8_t bf16[kBatch];
  Tensor t[kBatch];
};
static_assert(sizeof(Table) + 3 * 8 <= 4096, "the arguments of a kernel");

/* The tensor of an item: lane i looks at tensors i and i + 64 (a binary search waits for its table seven times). */
__device__ __forceinline__ int tensor_of(const Table& a, int item) {
  const int i = threadIdx.x & 63;
  return __popcll(__ballot(i < a.n && a.first[i] <= item)) + __popcll(__ballot(i + 64 < a.n && a.first[i + 64 < kBatch ? i + 64 : 0] <= item)) - 1;
}

/* A tensor as its items see it. */
struct View {
  const char* g;
  char* out;
  int ld, ldo, rows, cols, last, per_item, skew;      // rows of `cols` values, the last of `last`
};
__device__ __forceinline__ View view_of(const Table& a, int which) {
  const Tensor& t = a.t[which];
  const int per = a.per_item[which], skew = a.skew[which];
  if (per) return {t.g, t.out, t.m.ld, t.m.ldo, t.m.rows, t.m.cols, t.m.cols, per, skew};
  const int rows = (int)((t.values + kSpan - 1) / kSpan);
  return {t.g, t.out, kSpan, kSpan, rows, kSpan, (int)(t.values - (int64_t)(rows - 1) * kSpan), 1, skew};
}

/* f(chunk, row within the item, first column of the chunk, first and one past the last column of the values) for the chunks of an item; columns count from
 * the aligned base. */
template <typename T, int V, typename F> __device__ __forceinline__ void item_chunks(const View& t, int item, F&& f) {
  const int64_t r0 = (int64_t)item * t.per_item;
  const int rows = (int)(r0 + t.per_item < t.rows ? t.per_item : t.rows - r0);
  const int skew = V > 1 ? t.skew : 0, end = (t.per_item == 1 && r0 == t.rows - 1 ? t.last : t.cols) + skew, per = (end + V - 1) / V, total = rows * per;
  const int pitch = t.ld * (int)sizeof(T);                         // (an item's rows span less than 2^30 bytes, or are one)
  const auto from = row_at(t.g + r0 * t.ld * (int64_t)sizeof(T), (rows - 1) * pitch + per * V * (int)sizeof(T));
  for (int i0 = threadIdx.x; i0 - (int)threadIdx.x < total; i0 += 256 * kUnroll) {
    Pack<T, V> p[kUnroll];
    int r[kUnroll], c[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int i = i0 + u * 256;
      r[u] = rows > 1 ? i / per : 0;
      c[u] = (i - r[u] * per) * V;
      p[u] = row_load<T, V>(from, i < total ? r[u] * (pitch / (int)sizeof(T)) + c[u] : 0x7fffffff / (int)sizeof(T));
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i0 + u * 256 < total) f(p[u], r[u], c[u], skew, end);
  }
}

/* f(type tag, vector width tag) of a tensor. */
template <typename F> __device__ __forceinline__ void with_type_of(const View& t, bool bf16, F&& f) {
  if (bf16) {
    if (t.skew >= 0) f((__bf16)0.0f, std::integral_constant<int, 8>()); else f((__bf16)0.0f, std::integral_constant<int, 1>());
  } else {
    if (t.skew >= 0) f(0.0f, std::integral_constant<int, 4>()); else f(0.0f, std::integral_constant<int, 1>());
  }
}

__global__ __launch_bounds__(256) void sumsq_kernel(const Table a, double* part) {
  __shared__ double red[4];
  double s = 0.0;
  for (int item = blockIdx.x; item < a.items; item += gridDim.x) {
    const int which = __builtin_amdgcn_readfirstlane(tensor_of(a, item));
    const View t = view_of(a, which);
    with_type_of(t, a.bf16[which], [&](auto type, auto width) {
      using T = decltype(type);
      constexpr int V = decltype(width)::value;
      item_chunks<T, V>(t, item - a.first[which], [&](Pack<T, V> p, int, int c, int lo, int hi) {
        if (c < lo || c + V > hi) {
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (c + v < lo || c + v >= hi) p.v[v] = (T)0.0f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const double x = (double)to_f32(p.v[v]);
          s = fma(x, x, s);
        }
      });
    });
  }
  s = sum<64>(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(1024) void sumsq_final_kernel(int n, const double* part, double* sumsq) {
  __shared__ double red[16];
  double s = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = sum<64>(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
#pragma unroll
    for (int w = 0; w < 16; ++w) t += red[w];
    *sumsq = t;
  }
}

/* From the last tensor to the first (the table's order) and from a tensor's last item to its first: what the norm's pass read last is still in the last-level cache. */
template <bool STREAM> __global__ __launch_bounds__(256) void clip_kernel(const Table a, const double* sumsq, double max_norm, float* norm) {
  const double total = *sumsq;
  // The factor is mantissa * 2^power: as one fp32 number it would have few bits below 2^-126 (a norm of 1e36, clipped to 1e-3).  Not known yet: root and quotient
  // are taken while the first chunks are on their way.
  float mantissa = -1.0f;
  int power = 0;
  const auto known = [&] {
    if (mantissa < 0.0f) {
      const double n = sqrt(total);
      mantissa = n <= max_norm ? 1.0f : (float)frexp(max_norm / n, &power);       // (NaN for a NaN norm)
      if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    }
  };
  for (int item = blockIdx.x; item < a.items; item += gridDim.x) {
    const int which = __builtin_amdgcn_readfirstlane(tensor_of(a, item));
    const View t = view_of(a, which);
    if (t.g == t.out) {
      known();
      if (mantissa == 1.0f && power == 0) continue;    // in place and nothing to change
    }
    with_type_of(t, a.bf16[which], [&](auto type, auto width) {
      using T = decltype(type);
      constexpr int V = decltype(width)::value;
      const int i = (which + 1 < a.n ? a.first[which + 1] : a.items) - 1 - item;      // the tensor's items backwards
      const int64_t r0 = (int64_t)i * t.per_item;
      T* const out = reinterpret_cast<T*>(t.out) + r0 * t.ldo;
      const auto to = row_at(out, 0x7fffffff);      // (every store below lies within the tensor)
      item_chunks<T, V>(t, i, [&](Pack<T, V> p, int r, int c, int lo, int hi) {
        known();
        const int at = r * t.ldo + c;
#pragma unroll
        for (int v = 0; v < V; ++v) p.v[v] = (T)ldexpf(to_f32(p.v[v]) * mantissa, power);
        if (c >= lo && c + V <= hi) {
          if constexpr (STREAM && V > 1) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, p), reinterpret_cast<u32x4*>(out + at));
          else row_store<false>(to, at, p);
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (c + v >= lo && c + v < hi) out[at + v] = p.v[v];
        }
      });
    });
  }
  if (norm) known();                   // (a table without values)
}

inline int check_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? HAP_OK : hap_fail(HAP_EDEVICE, "%s launch: %s", what, hipGetErrorString(e));
}

int check(const hap_grad_desc* d) {
  if (!d) return hap_fail(HAP_EINVAL, "descriptor is NULL");
  if (d->n < 0) return hap_fail(HAP_EINVAL, "negative number of tensors");
  if (d->n > 0 && (!d->rows || !d->cols || !d->ld || !d->dtype)) return hap_fail(HAP_EINVAL, "rows, cols, ld or dtype is NULL");
  int64_t left = (int64_t)1 << 40;       // (items are counted in 32 bits)
  for (int i = 0; i < d->n; ++i) {
    if (d->rows[i] < 0 || d->cols[i] < 0) return hap_fail(HAP_EINVAL, "tensor %d: negative size", i);
    if (d->dtype[i] != HAP_F32 && d->dtype[i] != HAP_BF16) return hap_fail(HAP_EINVAL, "tensor %d: bad dtype %d", i, d->dtype[i]);
    if (d->rows[i] > 1 && d->ld[i] < d->cols[i]) return hap_fail(HAP_ESHAPE, "tensor %d: leading dimension %lld below %lld columns", i, (long long)d->ld[i], (long long)d->cols[i]);
    if (d->rows[i] && d->cols[i] > left / d->rows[i]) return hap_fail(HAP_EUNSUPPORTED, "more than 2^40 values up to tensor %d", i);
    left -= d->rows[i] * d->cols[i];
    if (d->rows[i] > 1 && d->ld[i] != d->cols[i] && (d->ld[i] > 0xfffffff || d->rows[i] > 0x7fffffff))
      return hap_fail(HAP_EUNSUPPORTED, "tensor %d: 2^31 rows or a pitch of 2^28 elements and more", i);
  }
  return HAP_OK;
}

/* Fills the table with tensors from `*next` on (`step` 1, or -1 to go backwards, with those of a table backwards, too) that have values; false when
 * there are none left. */
bool next_batch(const hap_grad_desc* d, const void* const* grads, void* const* out, const int64_t* ldo, int step, int* next, Table* a) {
  a->n = a->items = 0;
  for (; *next >= 0 && *next < d->n && a->n < kBatch; *next += step) {
    const int i = *next;
    int64_t rows = d->rows[i], cols = d->cols[i];
    if (rows == 0 || cols == 0) continue;
    const int es = d->dtype[i] == HAP_BF16 ? 2 : 4, V = 16 / es;
    int64_t ld = d->ld[i], lo = ldo ? ldo[i] : ld, items;
    const bool whole = rows == 1 || (ld == cols && (!out || lo == cols));
    const uintptr_t g = (uintptr_t)grads[i], o = out ? (uintptr_t)out[i] : g;
    const bool vec = g % es == 0 && g % 16 == o % 16 && (whole || (ld % V == 0 && lo % V == 0));
    const int skew = vec ? (int)(g % 16 / es) : -1, k = a->n++;
    Tensor& t = a->t[k];
    t.g = (const char*)grads[i] - (skew > 0 ? skew * es : 0);
    t.out = out ? (char*)out[i] - (skew > 0 ? skew * es : 0) : NULL;
    if (whole) {
      t.values = rows * cols;
      a->per_item[k] = 0;
      items = (t.values + kSpan - 1) / kSpan;
    } else {
      const int64_t fit = ((int64_t)1 << 27) / (ld > lo ? ld : lo);                // rows within reach of an item's 32-bit offsets
      int64_t per = kSpan / cols < fit ? kSpan / cols : fit;
      if (per < 1) per = 1;
      t.m = {(int)rows, (int)cols, (int)ld, (int)lo};
      a->per_item[k] = (uint16_t)per;
      items = (rows + per - 1) / per;
    }
    a->first[k] = a->items;
    a->skew[k] = (int8_t)skew;
    a->bf16[k] = d->dtype[i] == HAP_BF16;
    a->items += (int)items;
  }
  return a->n > 0;
}

/* Refuses an output that is listed twice: two workgroups would scale it.  (A hash table of the addresses; views that interleave differ in theirs.) */
int each_once(const hap_grad_desc* d, void* const* out) {
  size_t size = 16;
  while (size < (size_t)d->n * 2) size *= 2;
  const void** const seen = (const void**)calloc(size, sizeof(void*));
  if (!seen) return hap_fail(HAP_EINVAL, "no host memory for %d addresses", d->n);
  int rc = HAP_OK;
  for (int i = 0; i < d->n && rc == HAP_OK; ++i) {
    if (d->rows[i] == 0 || d->cols[i] == 0) continue;
    size_t at = (size_t)(((uint64_t)(uintptr_t)out[i] * 0x9E3779B97F4A7C15ull) >> 32) & (size - 1);
    while (seen[at] && seen[at] != out[i]) at = (at + 1) & (size - 1);
    if (seen[at]) rc = hap_fail(HAP_EINVAL, "tensor %d: its output is that of another tensor", i);
    seen[at] = out[i];
  }
  free(seen);
  return rc;
}

inline int grid_of(const Table& a) { return a.items < kBlocks ? a.items : kBlocks; }

}  // namespace

extern "C" {

size_t hap_grad_sumsq_workspace(const hap_grad_desc* d) {
  if (check(d) != HAP_OK) return 0;
  return (size_t)((d->n + kBatch - 1) / kBatch + 1) * kBlocks * sizeof(double);
}

int hap_grad_sumsq(const hap_grad_desc* d, const void* const* grads, double* sumsq, void* ws, size_t ws_bytes, void* stream) {
  hap_clear_error();
  int rc = check(d);
  if (rc) return rc;
  if (!sumsq || (d->n > 0 && !grads)) return hap_fail(HAP_EINVAL, "grads or sumsq is NULL");
  for (int i = 0; i < d->n; ++i)
    if (!grads[i] && d->rows[i] > 0 && d->cols[i] > 0) return hap_fail(HAP_EINVAL, "tensor %d is NULL", i);
  const size_t need = hap_grad_sumsq_workspace(d);
  if (!ws || ws_bytes < need) return hap_fail(HAP_EWORKSPACE, "grad_sumsq needs %zu workspace bytes", need);
  if ((uintptr_t)ws % sizeof(double)) return hap_fail(HAP_EINVAL, "ws is not on a multiple of %zu bytes", sizeof(double));
  hipStream_t s = (hipStream_t)stream;
  double* part = static_cast<double*>(ws);
  int64_t parts = 0;                   // (at most kBlocks for each of the tables: the workspace's size)
  Table a;
  for (int next = 0; next_batch(d, grads, NULL, NULL, 1, &next, &a);) {
    hipLaunchKernelGGL(sumsq_kernel, dim3(grid_of(a)), dim3(256), 0, s, a, part + parts);
    if ((rc = check_launch("grad_sumsq"))) return rc;
    parts += grid_of(a);
  }
  hipLaunchKernelGGL(sumsq_final_kernel, dim3(1), dim3(1024), 0, s, (int)parts, part, sumsq);
  return check_launch("grad_sumsq final");
}

int hap_grad_clip(const hap_grad_desc* d, const void* const* grads, void* const* out, const int64_t* ldo, const double* sumsq, float* norm, void* stream) {
  hap_clear_error();
  int rc = check(d);
  if (rc) return rc;
  if (!(d->max_norm > 0.0)) return hap_fail(HAP_EINVAL, "max_norm %g is not positive", d->max_norm);
  if (!sumsq || (d->n > 0 && (!grads || !out))) return hap_fail(HAP_EINVAL, "grads, out or sumsq is NULL");
  for (int i = 0; i < d->n; ++i) {
    if (d->rows[i] == 0 || d->cols[i] == 0) continue;
    if (!grads[i] || !out[i]) return hap_fail(HAP_EINVAL, "tensor %d is NULL", i);
    if (grads[i] == out[i] && ldo && d->rows[i] > 1 && ldo[i] != d->ld[i]) return hap_fail(HAP_EINVAL, "tensor %d: in place with another leading dimension", i);
    if (ldo && d->rows[i] > 1 && ldo[i] != d->cols[i] && (ldo[i] > 0xfffffff || d->rows[i] > 0x7fffffff)) return hap_fail(HAP_EUNSUPPORTED, "tensor %d: 2^31 rows or a pitch of 2^28 elements and more", i);
    if (ldo && d->rows[i] > 1 && ldo[i] < d->cols[i]) return hap_fail(HAP_ESHAPE, "tensor %d: leading dimension of the output below %lld columns", i, (long long)d->cols[i]);
  }
  if ((rc = each_once(d, out))) return rc;
  hipStream_t s = (hipStream_t)stream;
  int64_t bytes = 0;
  for (int i = 0; i < d->n; ++i) bytes += d->rows[i] * d->cols[i] * (d->dtype[i] == HAP_BF16 ? 2 : 4);
  // More than the last-level cache holds.  Norm and clipping, fp32, written through / non-temporally, alone and with a pass that reads the result: 260 MB 160 / 132 and
  // 304 / 289 us, 400 MB 241 / 213 and 457 / 446, 1100 MB 651 / 618 and 1229 / 1208.
  const bool stream_out = bytes > (int64_t)256 << 20;
  Table a;
  bool any = false;
  for (int next = d->n - 1; next_batch(d, grads, out, ldo, -1, &next, &a); any = true) {
    if (stream_out) hipLaunchKernelGGL(clip_kernel<true>, dim3(grid_of(a)), dim3(256), 0, s, a, sumsq, d->max_norm, any ? NULL : norm);
    else hipLaunchKernelGGL(clip_kernel<false>, dim3(grid_of(a)), dim3(256), 0, s, a, sumsq, d->max_norm, any ? NULL : norm);
    if ((rc = check_launch("grad_clip"))) return rc;
  }
  if (!any && norm) {
    hipLaunchKernelGGL(clip_kernel<false>, dim3(1), dim3(256), 0, s, a, sumsq, d->max_norm, norm);      // (an empty table)
    return check_launch("grad_clip");
  }
  return HAP_OK;
}

}  // extern "C"
