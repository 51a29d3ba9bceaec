// Routing of tokens to experts, its gradient, and the order of the assignments
// by expert.
//
// Routing.  For a token's logits l: scores s = softmax(l) or 1 / (1 + exp(-l)),
// selection values v = s + bias, or l itself without a bias (scores grow with
// their logit, so the order is the same and no rounding of s takes part in it).
// With groups, the values of the consecutive groups (their largest v, or the sum of their
// two largest s + bias, of the scores themselves without a bias: sums of logits would be in another
// order) pick the groups that stay.  The k largest v are taken, equal ones by the lowest index; w = s of each, over their sum if asked, times
// the scale.  An expert whose logit is -inf is never taken; a place with none left
// holds index -1 and weight 0.
// A group of G lanes holds a token's values in registers, NPL consecutive ones
// a lane, so that the first lane with the largest value also has its lowest index.
// Bound by the k rounds of reductions over the group, not by memory: the logits
// are read once, in 16-byte loads where they are aligned.  16384 tokens, 8 of 256 in 4 of 8 groups by two, float32:
// 22 us (0.8 TB/s of logits); 32771 tokens, 4 of 60, bfloat16: 8 us.
//
// Gradient.  With ds the gradient of the chosen scores: softmax dl = s (ds - sum ds s),
// sigmoid dl = ds s (1 - s); dividing by the sum S turns dw into (dw - sum dw w) / S, so ds s into (dw - sum dw w) w.
// The softmax is computed again from the logits, each with an exponential and a division, and k values are handed
// round the group.  32771 tokens of 60, bfloat16: 8 us, of which the launch is half; its bytes pass at 1 TB/s.
//
// Order.  A stable counting sort: a workgroup counts its piece of the assignments for
// each wave and expert, adds what earlier pieces counted, and places its own.  131072 assignments of 64 experts:
// 5 us for the counts and 9 us for the places, bound by the launches and by a workgroup's 2048 assignments in turn.
#include <algorithm>

#include "block_common.h"

namespace cfp {
namespace {

constexpr int kRouteThreads = 256;

// Order-preserving key of a selection value: 0 for "gone", 1 for NaN.
__device__ __forceinline__ uint32_t key_of(float v, bool gone) {
  if (gone) return 0u;
  if (v != v) return 1u;
  const uint32_t u = __float_as_uint(v + 0.f);  // -0 as +0
  const uint32_t k = u & 0x80000000u ? ~u : u | 0x80000000u;
  return k < 2u ? 2u : k;
}

template <typename T, int NPL, bool ALIGNED>
__device__ __forceinline__ void load_logits(const T *row, int e0, int n, float (&l)[NPL]) {
  constexpr int V = NPL * (int)sizeof(T) >= 16 ? 16 / (int)sizeof(T) : NPL;
  if (ALIGNED && e0 + NPL <= n) {
#pragma unroll
    for (int i = 0; i < NPL; i += V) {
      float x[V];
      load_vec<T, V>(row + e0 + i, x);
#pragma unroll
      for (int j = 0; j < V; ++j) l[i + j] = x[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < NPL; ++i) l[i] = e0 + i < n ? (float)row[e0 + i] : -INFINITY;
  }
}

// Largest logit and sum of exp(l - largest); a row of -inf alone gives 0 and 0.
template <int NPL, int G>
__device__ __forceinline__ void softmax_sum(const float (&l)[NPL], float &top, float &sum) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < NPL; ++i) m = fmaxf(m, l[i]);
  m = group_max<G>(m);
  top = m == -INFINITY ? 0.f : m;
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < NPL; ++i) z += expf(l[i] - top);
  sum = group_sum<G>(z);
}

__device__ __forceinline__ float score_of(float l, bool softmax, float top, float sum) {
  if (!softmax) return 1.f / (1.f + expf(-l));
  const float e = expf(l - top);
  return sum == 0.f ? 0.f : e / sum;
}

struct RouteArgs {
  const void *logits;
  int64_t stride, n_tokens;
  const float *bias;
  float *weight;
  int32_t *index;
  const float *dweight;
  void *dlogits;
  int32_t n, k, groups, top_groups;
  int32_t softmax, top2, renorm;
  float scale;
};

// Two largest of two descending pairs, into the first.
__device__ __forceinline__ void merge_two(float &a, float &b, float c, float d) {
  b = fmaxf(fminf(a, c), fmaxf(b, d));
  a = fmaxf(a, c);
}

enum Grouping { kNoGroups, kLaneGroups, kAnyGroups };

template <typename T, int NPL, int G, bool ALIGNED, int GROUPS>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(RouteArgs A) {
  constexpr int kTok = kRouteThreads / G;
  __shared__ int32_t chosen[kTok][CFP_ROUTE_MAX_K];
  __shared__ float logit[kTok][CFP_ROUTE_MAX_K];
  extern __shared__ float values[];  // kAnyGroups: [kTok][n + groups]
  const int lane = threadIdx.x % G, sub = threadIdx.x / G;
  const int base = (threadIdx.x % 64) / G * G;  // first lane of the group in its wave
  const int64_t t = (int64_t)block_id() * kTok + sub;
  const bool live = t < A.n_tokens;
  const int n = A.n, e0 = lane * NPL;
  float l[NPL], v[NPL];
  load_logits<T, NPL, ALIGNED>(reinterpret_cast<const T *>(A.logits) + (live ? t : 0) * A.stride, e0, n, l);
  float top = 0.f, sum = 1.f;
  if (A.softmax) softmax_sum<NPL, G>(l, top, sum);
  uint32_t key[NPL];
#pragma unroll
  for (int i = 0; i < NPL; ++i) {
    v[i] = l[i];
    if (A.bias != nullptr && e0 + i < n) v[i] = score_of(l[i], A.softmax, top, sum) + A.bias[e0 + i];
    key[i] = key_of(v[i], e0 + i >= n || l[i] == -INFINITY);
  }
  if constexpr (GROUPS != kNoGroups) {
    const int per = n / A.groups;
    float gval[NPL];  // what counts for a group: masked experts count for nothing
#pragma unroll
    for (int i = 0; i < NPL; ++i)
      gval[i] = key[i] == 0u                ? -INFINITY
                : A.top2 && A.bias == nullptr ? score_of(l[i], A.softmax, top, sum)
                                              : v[i];
    if constexpr (GROUPS == kLaneGroups) {  // a group is a power of two of whole lanes
      const int wide = per / NPL;
      float a = -INFINITY, b = -INFINITY;
      uint32_t bad = 0u;
#pragma unroll
      for (int i = 0; i < NPL; ++i) {
        bad |= gval[i] != gval[i];
        merge_two(a, b, gval[i], -INFINITY);
      }
      for (int off = 1; off < wide; off <<= 1) {
        merge_two(a, b, __shfl_xor(a, off, 64), __shfl_xor(b, off, 64));
        bad |= (uint32_t)__shfl_xor((int)bad, off, 64);
      }
      const float gv = bad ? __builtin_nanf("") : A.top2 ? a + b : a;
      const uint32_t mine = key_of(gv, gv == -INFINITY);
      int before = 0;
      for (int o = 0; o < A.groups; ++o) {
        const uint32_t other = (uint32_t)__shfl((int)mine, base + o * wide, 64);
        before += other > mine || (other == mine && o < lane / wide);
      }
#pragma unroll
      for (int i = 0; i < NPL; ++i)
        if (before >= A.top_groups) key[i] = 0u;
    } else {
      float *val = values + sub * (n + A.groups);
      float *gv = val + n;
#pragma unroll
      for (int i = 0; i < NPL; ++i)
        if (e0 + i < n) val[e0 + i] = gval[i];
      __syncthreads();
      for (int g = lane; g < A.groups; g += G) {
        float a = -INFINITY, b = -INFINITY;
        for (int i = 0; i < per; ++i) {
          const float x = val[g * per + i];
          if (x != x) {
            a = b = x;
            break;
          }
          merge_two(a, b, x, -INFINITY);
        }
        gv[g] = A.top2 ? a + b : a;
      }
      __syncthreads();
      // a group stays if fewer than top_groups come before it
      int held = -1;
      bool stays = true;
#pragma unroll
      for (int i = 0; i < NPL; ++i) {
        if (e0 + i >= n) continue;
        const int g = (e0 + i) / per;
        if (g != held) {
          held = g;
          const uint32_t mine = key_of(gv[g], gv[g] == -INFINITY);
          int before = 0;
          for (int o = 0; o < A.groups; ++o) {
            const uint32_t other = key_of(gv[o], gv[o] == -INFINITY);
            before += other > mine || (other == mine && o < g);
          }
          stays = before < A.top_groups;
        }
        if (!stays) key[i] = 0u;
      }
    }
  }
  // k rounds: the first lane with the largest key gives it up
  const uint64_t mask = (~0ull >> (64 - G)) << base;
  for (int j = 0; j < A.k; ++j) {
    uint32_t best = 0u;
#pragma unroll
    for (int i = 0; i < NPL; ++i) best = best > key[i] ? best : key[i];
    const uint32_t all = group_umax<G>(best);
    const uint64_t who = __ballot(best == all) & mask;
    if ((int)(threadIdx.x % 64) == __ffsll((unsigned long long)who) - 1) {
      int e = -1;
      float lv = 0.f;
      if (all != 0u) {
#pragma unroll
        for (int i = NPL - 1; i >= 0; --i) {  // the lowest index with this key is the last that is met
          e = key[i] == all ? i : e;
          lv = key[i] == all ? l[i] : lv;
        }
#pragma unroll
        for (int i = 0; i < NPL; ++i) key[i] = i == e ? 0u : key[i];
        e += e0;
      }
      chosen[sub][j] = e;
      logit[sub][j] = lv;
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // a group's results are written and read by its own wave
  __builtin_amdgcn_wave_barrier();
  float w[2] = {0.f, 0.f};
  int32_t at[2] = {-1, -1};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = lane + h * G;
    if (j >= A.k) continue;
    at[h] = chosen[sub][j];
    w[h] = at[h] < 0 ? 0.f : score_of(logit[sub][j], A.softmax, top, sum);
  }
  const float total = group_sum<G>(w[0] + w[1]);
  if (!live) return;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = lane + h * G;
    if (j >= A.k) continue;
    if (A.renorm) w[h] = total == 0.f ? 0.f : w[h] / total;
    A.weight[t * A.k + j] = w[h] * A.scale;
    A.index[t * A.k + j] = at[h];
  }
}

template <typename T, int NPL, int G, bool ALIGNED>
__global__ __launch_bounds__(kRouteThreads) void route_bwd_kernel(RouteArgs A) {
  constexpr int kTok = kRouteThreads / G;
  const int lane = threadIdx.x % G;
  const int base = (threadIdx.x % 64) / G * G;
  const int64_t t = (int64_t)block_id() * kTok + threadIdx.x / G;
  if (t >= A.n_tokens) return;  // whole groups: the others' shuffles stay inside their group
  const int n = A.n, e0 = lane * NPL;
  const T *row = reinterpret_cast<const T *>(A.logits) + t * A.stride;
  float l[NPL], ds[NPL];
  load_logits<T, NPL, ALIGNED>(row, e0, n, l);
  float top = 0.f, sum = 1.f;
  if (A.softmax) softmax_sum<NPL, G>(l, top, sum);
  float s[2], d[2];
  int at[2];
  float total = 0.f, dot = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = lane + h * G;
    at[h] = j < A.k ? A.index[t * A.k + j] : -1;
    if (at[h] >= n) at[h] = -1;
    s[h] = at[h] < 0 ? 0.f : score_of((float)row[at[h]], A.softmax, top, sum);
    d[h] = at[h] < 0 ? 0.f : A.dweight[t * A.k + j] * A.scale;
    total += s[h];
    dot += d[h] * s[h];
  }
  if (!A.renorm) {
    dot = group_sum<G>(dot);
  } else {  // from here on d holds ds s: 1 / S may be no float where (dw - sum dw w) w is one
    total = group_sum<G>(total);
    float w[2], mean = 0.f, again = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      w[h] = total == 0.f ? 0.f : s[h] / total;
      mean += d[h] * w[h];
    }
    mean = group_sum<G>(mean);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      d[h] = at[h] < 0 ? 0.f : (d[h] - mean) * w[h];
      again += d[h];
    }
    dot = group_sum<G>(again);
  }
#pragma unroll
  for (int i = 0; i < NPL; ++i) ds[i] = 0.f;
  for (int j = 0; j < A.k; ++j) {
    const int src = base + j % G;
    const int e = __shfl(j < G ? at[0] : at[1], src, 64) - e0;
    const float x = __shfl(j < G ? d[0] : d[1], src, 64);
#pragma unroll
    for (int i = 0; i < NPL; ++i) ds[i] += e == i ? x : 0.f;
  }
  T *out = reinterpret_cast<T *>(A.dlogits) + t * (int64_t)n;
#pragma unroll
  for (int i = 0; i < NPL; ++i) {
    const float p = score_of(l[i], A.softmax, top, sum);
    if (A.renorm)
      ds[i] = A.softmax ? ds[i] - p * dot : ds[i] * (1.f - p);
    else
      ds[i] = A.softmax ? p * (ds[i] - dot) : ds[i] * p * (1.f - p);
  }
  if (ALIGNED && e0 + NPL <= n) {
    store_vec<T, NPL>(out + e0, ds);
  } else {
#pragma unroll
    for (int i = 0; i < NPL; ++i)
      if (e0 + i < n) out[e0 + i] = (T)ds[i];
  }
}

// f(NPL, G): the least lanes and values a lane that hold a row, 16 lanes at least so
// that k <= 32 results fit two registers of a group.
template <typename F>
hipError_t with_shape(int n, F f) {
  using std::integral_constant;
  if (n <= 64) return f(integral_constant<int, 4>{}, integral_constant<int, 16>{});
  if (n <= 128) return f(integral_constant<int, 8>{}, integral_constant<int, 16>{});
  if (n <= 256) return f(integral_constant<int, 8>{}, integral_constant<int, 32>{});
  if (n <= 512) return f(integral_constant<int, 8>{}, integral_constant<int, 64>{});
  return f(integral_constant<int, 16>{}, integral_constant<int, 64>{});
}

template <typename F>
hipError_t with_type(int dtype, F f) {
  switch (dtype) {
    case CFP_DT_F32: return f(float{});
    case CFP_DT_F16: return f(f16_t{});
    default: return f(bf16_t{});
  }
}

RouteArgs args_of(const cfp_route_desc &d) {
  RouteArgs A{};
  A.logits = d.logits, A.stride = d.stride, A.n_tokens = d.n_tokens, A.bias = d.bias;
  A.n = d.n_experts, A.k = d.k, A.groups = d.groups, A.top_groups = d.top_groups;
  A.softmax = d.score == CFP_SCORE_SOFTMAX, A.top2 = d.group_score == CFP_GROUP_TOP_TWO;
  A.renorm = d.renormalise, A.scale = d.scale;
  return A;
}

bool rows_aligned(const cfp_route_desc &d, int npl, const void *out) {
  const size_t bytes = std::min(16, npl * elem_bytes(d.dtype));
  const size_t el = elem_bytes(d.dtype);
  return reinterpret_cast<uintptr_t>(d.logits) % bytes == 0 && (d.stride * el % bytes == 0 || d.n_tokens == 1) &&
         (out == nullptr || (reinterpret_cast<uintptr_t>(out) % bytes == 0 && d.n_experts * el % bytes == 0));
}

// ------------------------------------------------------------------ order --

constexpr int kPlanWaves = 8;
constexpr int kPlanThreads = kPlanWaves * 64;
constexpr int kPlanParts = 8;      // threads that share a bin's counts of the pieces
// Assignments of a workgroup: one takes up to 4096, which saves the counting launch.  Every workgroup reads all
// pieces' counts, so above kPlanPieces of 2048 the pieces grow and not their number.
constexpr int kPlanPieces = 512;
inline int plan_piece(int64_t n) {
  return n <= 4096 ? 4096 : (int)std::max<int64_t>(2048, (n + kPlanPieces - 1) / kPlanPieces);
}

struct PlanArgs {
  const int32_t *index;
  int32_t *offsets, *rows, *slot, *count;
  int64_t n;
  int32_t experts, first, piece;
};

__device__ __forceinline__ int bin_of(const PlanArgs &A, int64_t i) {
  const int64_t e = (int64_t)A.index[i] - A.first;
  return e >= 0 && e < A.experts ? (int)e : A.experts;  // the last bin: dropped
}

// Assignments of each bin in a piece.
__global__ __launch_bounds__(kPlanThreads) void plan_count_kernel(PlanArgs A) {
  extern __shared__ int32_t hist[];
  const int bins = A.experts + 1;
  for (int b = threadIdx.x; b < bins; b += kPlanThreads) hist[b] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * A.piece, hi = min(lo + A.piece, A.n);
  for (int64_t i = lo + threadIdx.x; i < hi; i += kPlanThreads) atomicAdd(&hist[bin_of(A, i)], 1);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kPlanThreads) A.count[(int64_t)blockIdx.x * bins + b] = hist[b];
}

// Wave w of a workgroup places the w-th part of its piece, 64 assignments at a time:
// a lane's rank among the lanes of its bin is a ballot's population count.
__global__ __launch_bounds__(kPlanThreads) void plan_place_kernel(PlanArgs A) {
  extern __shared__ int32_t next[];  // [waves][bins], then start [bins] and base [bins]
  const int bins = A.experts + 1;
  if (blockIdx.x == 0 && threadIdx.x < CFP_PLAN_PAD) A.rows[A.n + threadIdx.x] = -1;
  int32_t *start = next + kPlanWaves * bins;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int64_t lo = (int64_t)blockIdx.x * A.piece, hi = min(lo + A.piece, A.n);
  const int each = (int)(((hi - lo) + kPlanWaves * 64 - 1) / (kPlanWaves * 64)) * 64;
  const int64_t from = min(lo + (int64_t)wave * each, hi), to = min(from + each, hi);
  for (int b = threadIdx.x; b < kPlanWaves * bins; b += kPlanThreads) next[b] = 0;
  __syncthreads();
  for (int64_t i = from + lane; i < to; i += 64) atomicAdd(&next[wave * bins + bin_of(A, i)], 1);
  __syncthreads();
  // bins' totals and what earlier pieces hold of them
  int32_t *base = start + bins;
  if (gridDim.x > 1) {
    for (int b = threadIdx.x; b < bins; b += kPlanThreads) start[b] = base[b] = 0;
    __syncthreads();
    const int pieces = gridDim.x, each = (pieces + kPlanParts - 1) / kPlanParts;
    for (int x = threadIdx.x; x < bins * kPlanParts; x += kPlanThreads) {
      const int part = x / bins, b = x - part * bins, to = min((part + 1) * each, pieces);
      int32_t before = 0, all = 0;
#pragma unroll 8
      for (int p = part * each; p < to; ++p) {
        const int32_t c = A.count[(int64_t)p * bins + b];
        before += p < (int)blockIdx.x ? c : 0;
        all += c;
      }
      atomicAdd(&start[b], all);
      atomicAdd(&base[b], before);
    }
    __syncthreads();
  }
  for (int b = threadIdx.x; b < bins; b += kPlanThreads) {
    int32_t before = gridDim.x > 1 ? base[b] : 0, own = 0;
    for (int w = 0; w < kPlanWaves; ++w) {
      const int32_t c = next[w * bins + b];
      next[w * bins + b] = before + own;
      own += c;
    }
    if (gridDim.x == 1) start[b] = own;
  }
  __syncthreads();
  if (wave == 0) {  // exclusive prefix sums of the totals
    int32_t run = 0;
    for (int b0 = 0; b0 < bins; b0 += 64) {
      const int b = b0 + lane;
      const int32_t own = b < bins ? start[b] : 0;
      int32_t x = own;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int32_t y = __shfl_up(x, off, 64);
        if (lane >= off) x += y;
      }
      if (b < bins) {
        start[b] = run + x - own;
        if (blockIdx.x == 0) A.offsets[b] = run + x - own;
      }
      run += __shfl(x, 63, 64);
    }
  }
  __syncthreads();
  for (int64_t i0 = from; i0 < to; i0 += 64) {
    const int64_t i = i0 + lane;
    const int bin = i < to ? bin_of(A, i) : -1;
    uint64_t same = __ballot(bin >= 0);
    for (int bit = 0; (bins - 1) >> bit; ++bit) {
      const bool on = bin >= 0 && (bin >> bit & 1);
      const uint64_t set = __ballot(on);
      same &= on ? set : ~set;
    }
    if (bin >= 0) {
      const int rank = __popcll(same & ((1ull << lane) - 1));
      const int32_t at = start[bin] + next[wave * bins + bin] + rank;
      A.rows[at] = bin == A.experts ? -1 : (int32_t)i;
      A.slot[i] = bin == A.experts ? -1 : at;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // every lane has read before the first of a bin writes
    __builtin_amdgcn_wave_barrier();
    if (bin >= 0 && (same & ((1ull << lane) - 1)) == 0) next[wave * bins + bin] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace

hipError_t launch_route(const cfp_route_desc &d, float *weight, int32_t *index, hipStream_t st) {
  RouteArgs A = args_of(d);
  A.weight = weight, A.index = index;
  return with_type(d.dtype, [&](auto t) {
    using T = decltype(t);
    return with_shape(d.n_experts, [&](auto npl, auto g) {
      constexpr int kTok = kRouteThreads / g.value;
      const dim3 grid = grid_of((d.n_tokens + kTok - 1) / kTok);
      const int per = d.n_experts / d.groups, wide = per / npl.value;
      const bool lanes = per % npl.value == 0 && (wide & (wide - 1)) == 0;
      auto go = [&](auto a) {
        if (d.top_groups == d.groups)
          route_kernel<T, npl.value, g.value, a.value, kNoGroups><<<grid, kRouteThreads, 0, st>>>(A);
        else if (lanes)
          route_kernel<T, npl.value, g.value, a.value, kLaneGroups><<<grid, kRouteThreads, 0, st>>>(A);
        else
          route_kernel<T, npl.value, g.value, a.value, kAnyGroups>
              <<<grid, kRouteThreads, (size_t)kTok * (d.n_experts + d.groups) * 4, st>>>(A);
      };
      rows_aligned(d, npl.value, nullptr) ? go(std::true_type{}) : go(std::false_type{});
      return hipGetLastError();
    });
  });
}

hipError_t launch_route_bwd(const cfp_route_desc &d, const int32_t *index, const float *dweight, void *dlogits,
                            hipStream_t st) {
  RouteArgs A = args_of(d);
  A.index = const_cast<int32_t *>(index), A.dweight = dweight, A.dlogits = dlogits;
  return with_type(d.dtype, [&](auto t) {
    using T = decltype(t);
    return with_shape(d.n_experts, [&](auto npl, auto g) {
      constexpr int kTok = kRouteThreads / g.value;
      const dim3 grid = grid_of((d.n_tokens + kTok - 1) / kTok);
      if (rows_aligned(d, npl.value, dlogits))
        route_bwd_kernel<T, npl.value, g.value, true><<<grid, kRouteThreads, 0, st>>>(A);
      else
        route_bwd_kernel<T, npl.value, g.value, false><<<grid, kRouteThreads, 0, st>>>(A);
      return hipGetLastError();
    });
  });
}

size_t plan_bytes(int64_t n_assign, int n_experts) {
  const int64_t pieces = (n_assign + plan_piece(n_assign) - 1) / plan_piece(n_assign);
  return pieces <= 1 ? 0 : (size_t)pieces * (n_experts + 1) * 4;
}

hipError_t launch_expert_plan(const cfp_plan_desc &d, int32_t *offsets, int32_t *rows, int32_t *slot, int32_t *scratch,
                              hipStream_t st) {
  PlanArgs A{d.index, offsets, rows, slot, scratch, d.n_tokens * d.k, d.n_experts, d.first, 0};
  A.piece = plan_piece(A.n);
  const int bins = d.n_experts + 1;
  const unsigned pieces = (unsigned)std::max<int64_t>(1, (A.n + A.piece - 1) / A.piece);
  if (pieces > 1) plan_count_kernel<<<pieces, kPlanThreads, (size_t)bins * 4, st>>>(A);
  plan_place_kernel<<<pieces, kPlanThreads, (size_t)(kPlanWaves + 2) * bins * 4, st>>>(A);
  return hipGetLastError();
}

}  // namespace cfp
