/*
 * Routing of tokens to experts, the step before the expert layers of Sec. 7.6: scores, choice and weights from the router's logits, and the
 * logits' gradient.
 *
 *   s = softmax(x) or sigmoid(x);  c = s + bias;  groups of experts by the sum of their best one or two c;  the top_k best c of the groups
 *   that stay;  w_i = scale * s[e_i], divided by the sum over the chosen where asked
 *
 * The choice follows the scores before any rounding.  Without a bias both scores rise with the logit, so the logits themselves are compared,
 * exactly; where sums decide (scores with a bias; among groups also the best two of each) they are formed and compared in fp64.
 */
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "hap_internal.h"
#include "hap_lanes.h"

namespace {

using namespace hap_lanes;

constexpr int kMaxExperts = 1024, kMaxTopK = 64, kMaxGroups = 64;

struct RouteArgs {
  int64_t tokens, ld;
  int experts, top_k, groups, top_groups, per_group;
  int best;                // members of a group whose scores it is ranked by
  int sigmoid, renormalise;
  float scale;
  int vec, vec_bias;       // rows, the bias start on 16-byte boundaries
  int group_lanes;         // lanes of a group where groups are whole lanes, a power of two; 0: they are not
};

/* R values of a row, `none` for those behind its end, in pieces of up to 16 bytes: piece c of lane l starts at element (c * stride + l) * V, so that stride 1 and
 * pieces of R elements are R consecutive elements a lane, and stride L interleaves the lanes.  No condition around a load: the compiler would wait for each. */
template <typename T, int R> struct Pieces { static constexpr int V = R * sizeof(T) >= 16 ? 16 / sizeof(T) : R, N = R / V; };
template <typename T, int R> __device__ __forceinline__ int element_of(int l, int r, int lanes, bool interleaved) {
  constexpr int V = Pieces<T, R>::V;
  return interleaved ? ((r / V) * lanes + l) * V + r % V : l * R + r;
}
template <typename T, int R, bool INTERLEAVED> __device__ __forceinline__ void load_values(const T* row, int l, int lanes, int count, int vec, float none, float (&x)[R]) {
  constexpr int V = Pieces<T, R>::V, N = Pieces<T, R>::N;
  if (vec && element_of<T, R>(l, R - 1, lanes, INTERLEAVED) < count) {
    Pack<T, V> p[N];
#pragma unroll
    for (int c = 0; c < N; ++c) p[c] = *reinterpret_cast<const Pack<T, V>*>(row + element_of<T, R>(l, c * V, lanes, INTERLEAVED));
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = to_f32(p[r / V].v[r % V]);
  } else {
    T v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int e = element_of<T, R>(l, r, lanes, INTERLEAVED);
      v[r] = row[e < count ? e : count - 1];
    }
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = element_of<T, R>(l, r, lanes, INTERLEAVED) < count ? to_f32(v[r]) : none;
  }
}

/* ---- ranks: numbers as they are compared, NaN above everything and the infinities as finite ones in their order (v_max_f64 passes a NaN over); kNone (and anything
 * as low, which no fp32 number or sum of them is) stands for what cannot be chosen. */
constexpr double kNone = -1.7e308, kInfinite = 0x1.ffffffffff800p+1023, kNan = 0x1.fffffffffff00p+1023;
__device__ __forceinline__ double rank_of(double v) {
  const double low = fmax(fmin(v, kInfinite), kNone);                 // (of a NaN: either bound)
  return v != v ? kNan : low;
}
__device__ __forceinline__ bool is_rank(double k) { return k > -1e300; }
template <int L> __device__ __forceinline__ double greatest(double k) { return fold<L>(k, [](double a, double b) { return fmax(a, b); }); }

/* ---- keys: the rank of an fp32 number with the index of what it belongs to in its last ten bits (29 of a double's are free).  The greater key wins, equal numbers go by
 * the lower index: one v_max_f64 decides both and carries the index along. */
__device__ __forceinline__ double key_of(double rank, int index) {
  if (rank == kNone) return kNone;
  const uint64_t b = (uint64_t)__double_as_longlong(rank + 0.0);      // (-0 is 0)
  return __longlong_as_double((long long)((b & ~(uint64_t)1023) | (uint64_t)((b >> 63) ? index : 1023 - index)));
}
__device__ __forceinline__ int index_of(double k) {
  const uint64_t b = (uint64_t)__double_as_longlong(k);
  const int low = (int)(b & 1023);
  return (b >> 63) ? low : 1023 - low;
}

/* The two greatest of a set. */
struct Two { double first, second; };
__device__ __forceinline__ Two merge(Two a, Two b) { return {fmax(a.first, b.first), fmax(fmin(a.first, b.first), fmax(a.second, b.second))}; }

/* Closes (kNone) the ranks of all groups but the top_groups best.  `scratch`: LDS for the token's ranks, where groups are no whole lanes. */
template <int L, int R> __device__ __forceinline__ void keep_groups(const RouteArgs& a, double (&rank)[R], int l, volatile in_lds<double>* scratch) {
  const int e0 = l * R, span = a.group_lanes;
  Two two = {kNone, kNone};
  if (span) {
    // a group is `span` whole lanes: its best two by a butterfly over them, in every lane of it
#pragma unroll
    for (int r = 0; r < R; ++r) two = merge(two, Two{rank[r], kNone});
    if (span > 1) two = merge(two, Two{partner<1>(two.first), partner<1>(two.second)});
    if constexpr (L > 2) if (span > 2) two = merge(two, Two{partner<2>(two.first), partner<2>(two.second)});
    if constexpr (L > 4) if (span > 4) two = merge(two, Two{partner<4>(two.first), partner<4>(two.second)});
    if constexpr (L > 8) if (span > 8) two = merge(two, Two{partner<8>(two.first), partner<8>(two.second)});
    if constexpr (L > 16) if (span > 16) two = merge(two, Two{partner<16>(two.first), partner<16>(two.second)});
  } else {
    // (one wave: its LDS operations keep their order)
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (e0 + r < a.experts) scratch[e0 + r] = rank[r];
    __builtin_amdgcn_wave_barrier();
    if (l < a.groups)                  // (as many lanes as groups: the host chose L)
      for (int e = 0; e < a.per_group; ++e) two = merge(two, Two{scratch[l * a.per_group + e], kNone});
    __builtin_amdgcn_wave_barrier();
  }
  // the best group is that of the lowest lane that has the greatest sum
  double score = a.best > 1 && is_rank(two.second) ? (two.first == kNan ? kNan : fmin(two.first + two.second, kInfinite)) : two.first;
  const int unit = span ? span : 1;
  uint64_t stays = 0;                  // lanes of the groups that stay, each group's lowest
  bool mine = false;
  for (int i = 0; i < a.top_groups; ++i) {
    const double best = greatest<L>(score);
    if (!is_rank(best)) break;
    const int won = lowest_lane<L>(__ballot(score == best));
    stays |= 1ull << won;
    if (((won ^ l) & -unit) == 0) { mine = true; score = kNone; }
  }
  if (span) {
#pragma unroll
    for (int r = 0; r < R; ++r) rank[r] = mine ? rank[r] : kNone;
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (e0 + r < a.experts && !((stays >> ((e0 + r) / a.per_group)) & 1)) rank[r] = kNone;
  }
}

enum Order { kLogits, kSumsOfGroups, kSums };      // what is compared

/* One token per L lanes, R consecutive experts per lane; choice i of the token ends up in lane i.  kSums: scores with a bias decide, formed and compared in fp64;
 * otherwise the logits themselves, as keys, in groups that rank by their best logit or (kSumsOfGroups) by sums of scores.
 *
 * Bound: instructions (the logits are a few MB).  A choice is a maximum over the lane's own ranks and a butterfly, both of v_max_f64; few lanes with many
 * experts each do more tokens per instruction than one lane per expert.  8192 tokens, 8 of 256 in groups, bias and sums: 30 us with one token per wave, integer keys
 * and indices exchanged beside them, 21 with sums in fp32 that fall back to fp64 where they do not decide (the few waves that do set the time), 11.8 now.  Keys
 * decide the logits' order (7.5 us for the same without sums); for sums they would leave 42 bits to compare (11.4 us, and sigmoid scores of logits above 30 equal). */
template <typename T, int L, int R, Order ORDER>
__global__ __launch_bounds__(256) void route_fwd_kernel(const RouteArgs a, const T* logits, const float* bias, int* indices, float* weights) {
  constexpr bool SUMS = ORDER != kLogits, KEYS = ORDER != kSums;
  extern __shared__ double group_ranks[];           // [tokens of the block][experts], where groups are no whole lanes
  const int l = threadIdx.x % L, e0 = l * R;
  int64_t t = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const bool live = t < a.tokens;
  if (!live) t = a.tokens - 1;
  const T* row = logits + t * a.ld;
  float x[R], given[R];
  load_values<T, R, false>(row, l, L, a.experts, a.vec, -__builtin_inff(), x);
  if constexpr (ORDER == kSums) {
    load_values<float, R, false>(bias, l, L, a.experts, a.vec_bias, 0.0f, given);
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r) given[r] = 0.0f;
  }

  // statistics of the whole row, where the scores are a softmax over all of it
  float top = 0.0f, inv_total = 0.0f;
  if (!a.sigmoid && (SUMS || !a.renormalise)) {
    top = x[0];
#pragma unroll
    for (int r = 1; r < R; ++r) top = fmaxf(top, x[r]);
    top = fold<L>(top, [](float p, float q) { return fmaxf(p, q); });
    if (top == -__builtin_inff()) top = 0.0f;       // nothing can be chosen: no score is needed
  }
  double rank[R];
  if constexpr (!SUMS) {
    if (!a.sigmoid && !a.renormalise) {
      float s = 0.0f;
#pragma unroll
      for (int r = 0; r < R; ++r) s += expf(x[r] - top);
      inv_total = 1.0f / sum<L>(s);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) rank[r] = rank_of((double)x[r]);
  } else {
    double scale = 1.0;
    if (a.sigmoid) {
#pragma unroll
      for (int r = 0; r < R; ++r) rank[r] = 1.0 / (1.0 + exp(-(double)x[r]));
    } else {
      double n = 0.0;
#pragma unroll
      for (int r = 0; r < R; ++r) { rank[r] = exp((double)x[r] - (double)top); n += rank[r]; }
      n = sum<L>(n);
      scale = n == n ? 1.0 / n : 0.0;      // a NaN or +inf among the logits: their scores stay NaN, the others' are 0
      inv_total = (float)(1.0 / n);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {          // (closed by either, whatever the score is: a NaN plus -inf is a NaN)
      const bool shut = (x[r] == -__builtin_inff()) | (given[r] == -__builtin_inff());
      const double c = rank_of(rank[r] * scale + (double)given[r]);
      rank[r] = shut ? kNone : c;
    }
  }
  if (a.groups > 1) keep_groups<L, R>(a, rank, l, (in_lds<double>*)group_ranks + (threadIdx.x / L) * a.experts);

  if constexpr (KEYS) {
#pragma unroll
    for (int r = 0; r < R; ++r) {          // (the sums were the groups': inside them the logits decide, whose scores may be equal)
      const double logit = rank_of((double)x[r]);
      rank[r] = key_of(!SUMS ? rank[r] : is_rank(rank[r]) ? logit : kNone, e0 + r);
    }
  }
  int chosen = -1;
  for (int i = 0; i < a.top_k; ++i) {
    double k[R];
#pragma unroll
    for (int r = 0; r < R; ++r) k[r] = rank[r];
#pragma unroll
    for (int n = R / 2; n > 0; n /= 2)
#pragma unroll
      for (int r = 0; r < n; ++r) k[r] = fmax(k[r], k[r + n]);
    const double best = greatest<L>(k[0]);
    if (!is_rank(best)) break;
    const auto close = [&](int r, bool taken) {      // (one word: below every number)
      rank[r] = __hiloint2double(taken ? (int)0xffe00000 : __double2hiint(rank[r]), __double2loint(rank[r]));
    };
    if constexpr (KEYS) {
      if (l == i) chosen = index_of(best);
#pragma unroll
      for (int r = 0; r < R; ++r) close(r, rank[r] == best);
    } else {
      // all 64 bits are compared: of equals the lowest lane's first
      const int won = lowest_lane<L>(__ballot(k[0] == best));
      bool open = l == won;
      int e = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const bool taken = open & (rank[r] == best);
        e = taken ? e0 + r : e;
        close(r, taken);
        open = open & !taken;
      }
      e = __shfl(e, won, L);
      if (l == i) chosen = e;
    }
  }

  const float xi = chosen >= 0 ? to_f32(row[chosen]) : -__builtin_inff();
  float w;
  if (!a.renormalise) {
    w = a.sigmoid ? 1.0f / (1.0f + expf(-xi)) : expf(xi - top) * inv_total;
  } else {
    // ratios of the chosen scores with the largest of them as the unit: no sum can vanish
    float m = fold<L>(xi, [](float p, float q) { return fmaxf(p, q); });
    if (a.sigmoid) m = fminf(m, 0.0f);
    float s = chosen >= 0 ? (a.sigmoid ? (xi >= 0.0f ? 1.0f : expf(xi - m)) / (1.0f + expf(-fabsf(xi))) : expf(xi - m)) : 0.0f;
    w = s / sum<L>(s);
    if (SUMS && inv_total != inv_total) w = inv_total;                // a softmax without a value, whoever was chosen (a bias can bar the culprit)
  }
  if (live && l < a.top_k) {
    indices[t * a.top_k + l] = chosen;
    weights[t * a.top_k + l] = chosen >= 0 ? w * a.scale : 0.0f;
  }
}

/* With the choice held fixed and g_i the weights' gradients:
 *   softmax          dx_e = s_e (d_e - sum_f s_f d_f),   d_e = scale * sum of the g_i whose e_i is e
 *   sigmoid          dx_e = s_e (1 - s_e) d_e
 *   renormalised     a_i = scale * u_i (g_i - sum_j u_j g_j), u_i the ratios of the scores;  dx_e = sum of the a_i (times 1 - s_e for the sigmoid)
 * The choices' terms meet in an LDS row, which the lanes then read in the interleaved order that stores whole lines. */
template <typename T, int L, int R>
__global__ __launch_bounds__(256) void route_bwd_kernel(const RouteArgs a, const T* logits, const int* indices, const float* dweights, T* dlogits) {
  constexpr int V = Pieces<T, R>::V, N = Pieces<T, R>::N;
  __shared__ float sums[256 * R];                   // [tokens of the block][L * R]
  const int l = threadIdx.x % L;
  int64_t t = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const bool live = t < a.tokens;
  if (!live) t = a.tokens - 1;
  const T* row = logits + t * a.ld;
  volatile in_lds<float>* const mine = (in_lds<float>*)sums + (threadIdx.x / L) * (L * R);
#pragma unroll
  for (int r = 0; r < R; ++r) mine[r * L + l] = 0.0f;
  int chosen = -1;
  float g = 0.0f, xi = -__builtin_inff();
  const bool whole = !a.sigmoid && !a.renormalise;
  float x[R];
  if (whole) load_values<T, R, true>(row, l, L, a.experts, a.vec, -__builtin_inff(), x);
  if (l < a.top_k) {
    chosen = indices[t * a.top_k + l];
    g = dweights[t * a.top_k + l];
    const bool expert = chosen >= 0 && chosen < a.experts;
    xi = to_f32(row[expert ? chosen : 0]);
    if (!expert || xi == -__builtin_inff()) { chosen = -1; xi = -__builtin_inff(); }      // (a masked one's score is 0 whatever the others do)
    g = chosen >= 0 ? g * a.scale : 0.0f;
  }
  float dx[R], ai = 0.0f;
#pragma unroll
  for (int r = 0; r < R; ++r) dx[r] = 0.0f;
  if (a.renormalise) {
    float m = fold<L>(xi, [](float p, float q) { return fmaxf(p, q); });
    if (a.sigmoid) m = fminf(m, 0.0f);
    const float z = expf(-fabsf(xi));
    float u = chosen >= 0 ? (a.sigmoid ? (xi >= 0.0f ? 1.0f : expf(xi - m)) / (1.0f + z) : expf(xi - m)) : 0.0f;
    u /= sum<L>(u);
    if (chosen < 0) u = 0.0f;
    ai = u * (g - sum<L>(u * g));
    if (a.sigmoid) ai *= (xi >= 0.0f ? z : 1.0f) / (1.0f + z);       // 1 - s
  } else if (a.sigmoid) {
    const float z = expf(-fabsf(xi)), q = 1.0f / (1.0f + z);
    ai = chosen >= 0 ? g * z * q * q : 0.0f;
  } else {
    float top = x[0];
#pragma unroll
    for (int r = 1; r < R; ++r) top = fmaxf(top, x[r]);
    top = fold<L>(top, [](float p, float q) { return fmaxf(p, q); });
    if (top == -__builtin_inff()) top = 0.0f;
    float n = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) { dx[r] = expf(x[r] - top); n += dx[r]; }
    n = sum<L>(n);
    const float inv = n > 0.0f ? 1.0f / n : (n == 0.0f ? 0.0f : n);
    ai = chosen >= 0 ? g * (expf(xi - top) * inv) : 0.0f;
    const float dot = sum<L>(ai) * inv;
#pragma unroll
    for (int r = 0; r < R; ++r) dx[r] *= -dot;
  }
  // one wave: its LDS operations keep their order, and adds to one word within an instruction go lane by lane
  __builtin_amdgcn_wave_barrier();
  if (chosen >= 0) __hip_atomic_fetch_add(&mine[chosen], ai, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int r = 0; r < R; ++r) dx[r] += mine[element_of<T, R>(l, r, L, true)];
  if (!live) return;
  T* out = dlogits + t * a.ld;
  if (a.vec && element_of<T, R>(l, R - 1, L, true) < a.experts) {
#pragma unroll
    for (int c = 0; c < N; ++c) {
      Pack<T, V> p;
#pragma unroll
      for (int v = 0; v < V; ++v) p.v[v] = (T)dx[c * V + v];
      *reinterpret_cast<Pack<T, V>*>(out + element_of<T, R>(l, c * V, L, true)) = p;
    }
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (element_of<T, R>(l, r, L, true) < a.experts) out[element_of<T, R>(l, r, L, true)] = (T)dx[r];
  }
}

inline int check_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? HAP_OK : hap_fail(HAP_EDEVICE, "%s launch: %s", what, hipGetErrorString(e));
}

/* Checks a descriptor and turns it into the kernels' arguments. */
int resolve(const hap_route_desc* d, RouteArgs* a) {
  if (!d) return hap_fail(HAP_EINVAL, "descriptor is NULL");
  if (d->tokens < 0 || d->experts < 1 || d->top_k < 1) return hap_fail(HAP_EINVAL, "bad sizes");
  if (d->score != HAP_SCORE_SOFTMAX && d->score != HAP_SCORE_SIGMOID) return hap_fail(HAP_EINVAL, "bad score %d", d->score);
  if (d->io_dtype != HAP_F32 && d->io_dtype != HAP_BF16) return hap_fail(HAP_EINVAL, "bad io_dtype %d", d->io_dtype);
  if (d->experts > kMaxExperts || d->top_k > kMaxTopK || d->groups > kMaxGroups)
    return hap_fail(HAP_EUNSUPPORTED, "more than %d experts, %d choices or %d groups", kMaxExperts, kMaxTopK, kMaxGroups);
  if (d->groups < 1 || d->experts % d->groups) return hap_fail(HAP_ESHAPE, "%d groups do not divide %lld experts", d->groups, (long long)d->experts);
  const int per = (int)(d->experts / d->groups);
  if (d->top_groups < 1 || d->top_groups > d->groups) return hap_fail(HAP_EINVAL, "top_groups %d outside 1 .. %d", d->top_groups, d->groups);
  if (d->group_best < 1 || d->group_best > 2) return hap_fail(HAP_EINVAL, "group_best %d is neither 1 nor 2", d->group_best);
  if (d->top_k > (int64_t)d->top_groups * per) return hap_fail(HAP_ESHAPE, "top_k %d beyond the %d experts of %d groups", d->top_k, d->top_groups * per, d->top_groups);
  if (!grid_fits(d->tokens / 4 + 1)) return hap_fail(HAP_EUNSUPPORTED, "2^26 tokens and more");          // (four a workgroup in the widest layout)
  if (d->ld < d->experts) return hap_fail(HAP_ESHAPE, "leading dimension %lld below %lld experts", (long long)d->ld, (long long)d->experts);
  *a = RouteArgs{d->tokens, d->ld, (int)d->experts, d->top_k, d->groups, d->top_groups, per, d->group_best, d->score == HAP_SCORE_SIGMOID, d->renormalise != 0, d->scale, 0, 0, 0};
  return HAP_OK;
}

/* f(lanes per token, experts per lane): lanes for the choices and the groups, many experts each.  With a bias, 8192 / 65536 tokens: 8 of 256 in groups 11.8 / 57.6 us with 16 x 16
 * and 12.2 / 69.4 with 32 x 8; 8 of 512 16.2 / 98.4 with 32 x 16 and 17.8 / 117.7 with 64 x 8; 8 of 64 19.3 with 16 x 4 and 50.1 with 64 x 1 (65536). */
template <typename F> void with_layout(const RouteArgs& a, F&& f) {
  const int lanes = a.top_k > a.groups ? a.top_k : a.groups;
#define HAP_LAYOUT(L, R) f(std::integral_constant<int, L>(), std::integral_constant<int, R>())
  if (lanes <= 8 && a.experts <= 8) HAP_LAYOUT(8, 1);
  else if (lanes <= 8 && a.experts <= 32) HAP_LAYOUT(8, 4);
  else if (lanes <= 16 && a.experts <= 64) HAP_LAYOUT(16, 4);
  else if (lanes <= 16 && a.experts <= 128) HAP_LAYOUT(16, 8);
  else if (lanes <= 16 && a.experts <= 256) HAP_LAYOUT(16, 16);
  else if (lanes <= 32 && a.experts > 256 && a.experts <= 512) HAP_LAYOUT(32, 16);
  else if (a.experts <= 64) HAP_LAYOUT(64, 1);
  else if (a.experts <= 256) HAP_LAYOUT(64, 4);
  else if (a.experts <= 512) HAP_LAYOUT(64, 8);
  else HAP_LAYOUT(64, 16);
#undef HAP_LAYOUT
}

template <typename T> int route_fwd_t(RouteArgs a, const void* logits, const float* bias, int* indices, float* weights, hipStream_t s) {
  with_layout(a, [&](auto l, auto r) {
    constexpr int L = decltype(l)::value, R = decltype(r)::value;
    const dim3 grid((unsigned)((a.tokens + 256 / L - 1) / (256 / L)));
    const int gl = a.per_group % R ? 0 : a.per_group / R;
    a.group_lanes = gl && (gl & (gl - 1)) == 0 && gl < L ? gl : 0;
    const size_t lds = a.groups > 1 && !a.group_lanes ? (size_t)(256 / L) * a.experts * 8 : 0;
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), lds, s, a, (const T*)logits, bias, indices, weights); };
    if (bias) launch(route_fwd_kernel<T, L, R, kSums>);
    else if (a.groups > 1 && a.best > 1) launch(route_fwd_kernel<T, L, R, kSumsOfGroups>);
    else launch(route_fwd_kernel<T, L, R, kLogits>);
  });
  return check_launch("moe_route_fwd");
}

template <typename T> int route_bwd_t(const RouteArgs& a, const void* logits, const int* indices, const float* dweights, void* dlogits, hipStream_t s) {
  with_layout(a, [&](auto l, auto r) {
    constexpr int L = decltype(l)::value, R = decltype(r)::value;
    const dim3 grid((unsigned)((a.tokens + 256 / L - 1) / (256 / L)));
    hipLaunchKernelGGL((route_bwd_kernel<T, L, R>), grid, dim3(256), 0, s, a, (const T*)logits, indices, dweights, (T*)dlogits);
  });
  return check_launch("moe_route_bwd");
}

inline bool rows_aligned(const void* p, int64_t ld, int dtype) { return (uintptr_t)p % 16 == 0 && ld % (dtype == HAP_BF16 ? 8 : 4) == 0; }

}  // namespace

extern "C" {

int hap_moe_route_fwd(const hap_route_desc* d, const void* logits, const float* bias, int32_t* indices, float* weights, void* stream) {
  hap_clear_error();
  RouteArgs a;
  const int rc = resolve(d, &a);
  if (rc) return rc;
  if (a.tokens == 0) return HAP_OK;
  if (!logits || !indices || !weights) return hap_fail(HAP_EINVAL, "logits, indices or weights is NULL");
  a.vec = rows_aligned(logits, a.ld, d->io_dtype);
  a.vec_bias = (uintptr_t)bias % 16 == 0;
  return d->io_dtype == HAP_BF16 ? route_fwd_t<__bf16>(a, logits, bias, indices, weights, (hipStream_t)stream)
                                 : route_fwd_t<float>(a, logits, bias, indices, weights, (hipStream_t)stream);
}

int hap_moe_route_bwd(const hap_route_desc* d, const void* logits, const int32_t* indices, const float* dweights, void* dlogits, void* stream) {
  hap_clear_error();
  RouteArgs a;
  const int rc = resolve(d, &a);
  if (rc) return rc;
  if (a.tokens == 0) return HAP_OK;
  if (!logits || !indices || !dweights || !dlogits) return hap_fail(HAP_EINVAL, "logits, indices, dweights or dlogits is NULL");
  a.vec = rows_aligned(logits, a.ld, d->io_dtype) && rows_aligned(dlogits, a.ld, d->io_dtype);
  return d->io_dtype == HAP_BF16 ? route_bwd_t<__bf16>(a, logits, indices, dweights, dlogits, (hipStream_t)stream)
                                 : route_bwd_t<float>(a, logits, indices, dweights, dlogits, (hipStream_t)stream);
}

}  // extern "C"
