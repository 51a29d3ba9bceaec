// Keys and values into a paged cache and back.
//
// A key's entries lie behind each other, a value's tokens do: [dim][page].  In 8 bits a token's row x of one head is
// held as e4m3(x 2^-e), e the least integer >= -126 with max |x| <= 448 2^e, found from the bits of the maximum:
// with max |x| = m 2^t, m in [1, 2), e = t - 8 where m <= 1.75 (448 = 1.75 2^8), else t - 7.  A power of two costs
// a float no precision, so x 2^-e is exact and the entry is rounded once.
//
// Bound by memory.  A workgroup takes 16 tokens of one page and one head, 16 bytes a lane of keys, values and
// results: values pass through LDS, where rows of tokens become rows of entries.  The 16 are aligned in the page, not in the
// call, so that whole pieces of 16 bytes of values' tokens are written (by single entries only at a sequence's ends).
// Measured, 8 heads of 128: 32768 tokens in bfloat16 written as 8 bits 55 us (3.7 TB/s), 119992 tokens read back 157 us
// (4.7 TB/s; a copy reaches 5.1); a few tokens 4 us each way, the launch.
#include <algorithm>
#include <type_traits>

#include "cache_common.h"

namespace cfp {
namespace {

constexpr int kThreads = 256;
constexpr int kUnit = 16;  // tokens of a workgroup

struct CacheArgs {
  SeqArgs s;
  void *k, *v;               // the cache
  uint8_t *ks, *vs;
  int64_t kp, vp, ksp, vsp;  // strides of its pages, in elements
  void *x[2];                // the rows: keys, values
  HeadStrides sx[2];
  int32_t heads, dim, wide;  // wide: rows start on 16 bytes
};

// Units of sequence b: its tokens by aligned runs of kUnit, the first of which holds token max(pos, 0)
// (rows before the first token count as that many units more when they are read).
__device__ __forceinline__ uint32_t units_of(const Seq &q) {
  const int lo = q.pos & ~(kUnit - 1);
  return q.n ? (uint32_t)(q.pos + q.n - lo + kUnit - 1) / kUnit : 0u;
}
int64_t most_units(int64_t n_tokens, int64_t n_seqs) { return std::min(n_tokens, n_tokens / kUnit + 2 * n_seqs); }

struct UnitAt {
  Seq q;
  int32_t b, first;   // token of the first place
  int32_t lo, hi;     // places that are tokens of the call: lo <= place < hi
  uint32_t page;
  bool ok;
};
__device__ __forceinline__ bool unit_at(const SeqArgs &S, uint32_t id, UnitAt &u) {
  uint32_t k;
  int b;
  if (!find_unit(S, id, [](const Seq &q) { return units_of(q); }, b, k, u.q)) return false;
  u.b = b;
  u.first = (u.q.pos & ~(kUnit - 1)) + (int)k * kUnit;
  u.lo = max(u.q.pos - u.first, 0);
  u.hi = min(u.q.pos + u.q.n - u.first, kUnit);
  u.page = 0, u.ok = false;
  if (u.first >= 0) u.page = page_of(S, b, u.first, u.ok);
  return true;
}

// 8 entries of a row
template <typename T>
__device__ __forceinline__ void load_row(const T *p, bool wide, float (&x)[8]) {
  if (wide) {
    load_vec<T, 8>(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)p[i];
  }
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// x [8] of a row of which a group of G lanes holds the whole: 8 bytes, and the row's scale.
template <typename T, int G>
__device__ __forceinline__ vec<uint32_t, 2> quantise(const float (&x)[8], uint32_t &scale) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, finite(x[i]) ? fabsf(x[i]) : 0.f);
  top = group_max<G>(top);
  const uint32_t bits = __float_as_uint(top);
  const int e = max((int)(bits >> 23) - 127 - ((bits & 0x7fffffu) <= 0x600000u ? 8 : 7), -126);
  scale = (uint32_t)(e + 127);
  const float by = __uint_as_float((uint32_t)(127 - e) << 23);
  // at the end of T's range 240 2^e is the largest value of both types, and rounding up would leave T's
  const float most = e == (std::is_same<T, f16_t>::value ? 8 : 120) ? 240.f : 448.f;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = finite(x[i]) ? fminf(fmaxf(x[i] * by, -most), most) : __builtin_nanf("");
  vec<uint32_t, 2> r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
    r[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true);
  }
  return r;
}

__device__ __forceinline__ void unpack8(vec<uint32_t, 2> w, float s, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
    x[4 * i] = a[0] * s, x[4 * i + 1] = a[1] * s, x[4 * i + 2] = b[0] * s, x[4 * i + 3] = b[1] * s;
  }
}

// T: type of the rows; H: of what is held, T or uint8_t.  G lanes hold a row of up to 8 G entries.
template <typename T, typename H, int G>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CacheArgs A) {
  constexpr bool kByte = sizeof(H) == 1;
  constexpr int kRows = kThreads / G, kPass = kRows < kUnit ? kUnit / kRows : 1;
  constexpr int kLd = 8 * G + 16 / (int)sizeof(H);  // of a row in LDS
  __shared__ __align__(16) H tile[kUnit * kLd];
  const uint32_t id = block_id();
  const int head = (int)(id % A.heads);
  UnitAt u;
  if (!unit_at(A.s, id / A.heads, u) || !u.ok) return;  // the same for all threads
  const int D = A.dim, page = 1 << A.s.page_shift, place = u.first & (page - 1);
  const int c = 8 * (threadIdx.x % G);
  H *kd = reinterpret_cast<H *>(A.k) + u.page * A.kp + (int64_t)(head * page + place) * D;
  H *vd = reinterpret_cast<H *>(A.v) + u.page * A.vp + (int64_t)head * D * page + place;
  float x[2][kPass][8];
#pragma unroll
  for (int p = 0; p < kPass; ++p) {
    const int r = threadIdx.x / G + p * kRows;
    const bool in = r >= u.lo && r < u.hi && c < D;
    const int64_t row = u.q.row + (u.first + r - u.q.pos);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const T *from = reinterpret_cast<const T *>(A.x[w]) + row * A.sx[w].tok + head * A.sx[w].head + c;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[w][p][i] = 0.f;
      if (in) load_row<T>(from, A.wide != 0, x[w][p]);
    }
  }
#pragma unroll
  for (int p = 0; p < kPass; ++p) {
    const int r = threadIdx.x / G + p * kRows;
    const bool in = r >= u.lo && r < u.hi;
    if constexpr (kByte) {
      uint32_t sk, sv;
      const vec<uint32_t, 2> k = quantise<T, G>(x[0][p], sk), v = quantise<T, G>(x[1][p], sv);
      if (in && c < D) *reinterpret_cast<vec<uint32_t, 2> *>(kd + r * D + c) = k;
      if (r < kUnit) *reinterpret_cast<vec<uint32_t, 2> *>(tile + r * kLd + c) = v;
      if (in && c == 0) {
        A.ks[u.page * A.ksp + head * page + place + r] = (uint8_t)sk;
        A.vs[u.page * A.vsp + head * page + place + r] = (uint8_t)sv;
      }
    } else {
      if (in && c < D) store_vec<T, 8>(kd + r * D + c, x[0][p]);
      if (r < kUnit) store_vec<T, 8>(tile + r * kLd + c, x[1][p]);
    }
  }
  __syncthreads();
  // pieces of 16 bytes: kPer tokens of an entry
  constexpr int kPer = 16 / (int)sizeof(H), kParts = kUnit / kPer;
  for (int e = threadIdx.x; e < D * kParts; e += kThreads) {
    const int d = e / kParts, t = e % kParts * kPer;
    H *to = vd + (int64_t)d * page + t;
    if (u.lo <= t && u.hi >= t + kPer) {
      vec<H, kPer> w;
#pragma unroll
      for (int i = 0; i < kPer; ++i) w[i] = tile[(t + i) * kLd + d];
      *reinterpret_cast<vec<H, kPer> *>(to) = w;
    } else {
      for (int i = max(t, u.lo); i < min(t + kPer, u.hi); ++i) to[i - t] = tile[i * kLd + d];
    }
  }
}

template <typename T, typename H, int G>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheArgs A) {
  constexpr bool kByte = sizeof(H) == 1;
  constexpr int kRows = kThreads / G, kPass = kRows < kUnit ? kUnit / kRows : 1;
  constexpr int kLd = 8 * G + 16 / (int)sizeof(H);
  __shared__ __align__(16) H tile[kUnit * kLd];
  const uint32_t id = block_id();
  const int head = (int)(id % A.heads);
  UnitAt u;
  if (!unit_at(A.s, id / A.heads, u)) return;
  const int D = A.dim, page = 1 << A.s.page_shift, place = u.first & (page - 1);
  const H *kd = reinterpret_cast<const H *>(A.k) + u.page * A.kp + (int64_t)(head * page + place) * D;
  const H *vd = reinterpret_cast<const H *>(A.v) + u.page * A.vp + (int64_t)head * D * page + place;
  constexpr int kPer = 16 / (int)sizeof(H), kParts = kUnit / kPer;
  if (u.ok)
    for (int e = threadIdx.x; e < D * kParts; e += kThreads) {
      const int d = e / kParts, t = e % kParts * kPer;
      if (t >= u.hi || t + kPer <= u.lo) continue;
      const vec<H, kPer> w = *reinterpret_cast<const vec<H, kPer> *>(vd + (int64_t)d * page + t);
#pragma unroll
      for (int i = 0; i < kPer; ++i) tile[(t + i) * kLd + d] = w[i];
    }
  __syncthreads();
  const int c = 8 * (threadIdx.x % G);
#pragma unroll
  for (int p = 0; p < kPass; ++p) {
    const int r = threadIdx.x / G + p * kRows;
    if (r < u.lo || r >= u.hi || c >= D) continue;
    const int64_t at = ((int64_t)(u.q.row + (u.first + r - u.q.pos)) * A.heads + head) * D + c;
    float k[8], v[8];
    if (!u.ok) {  // before the first token, or in no page
#pragma unroll
      for (int i = 0; i < 8; ++i) k[i] = v[i] = u.first < 0 ? 0.f : __builtin_nanf("");
    } else if constexpr (kByte) {
      const int64_t sa = head * page + place + r;
      unpack8(*reinterpret_cast<const vec<uint32_t, 2> *>(kd + r * D + c), scale_of(A.ks[u.page * A.ksp + sa]), k);
      unpack8(*reinterpret_cast<const vec<uint32_t, 2> *>(tile + r * kLd + c), scale_of(A.vs[u.page * A.vsp + sa]), v);
    } else {
      load_vec<H, 8>(kd + r * D + c, k);
      load_vec<H, 8>(tile + r * kLd + c, v);
    }
    store_vec<T, 8>(reinterpret_cast<T *>(A.x[0]) + at, k);
    store_vec<T, 8>(reinterpret_cast<T *>(A.x[1]) + at, v);
  }
}

CacheArgs cache_args(const cfp_cache_desc &c, const cfp_sequences_desc &s, int64_t n_tokens) {
  CacheArgs A{};
  A.s = seq_args(c, s, n_tokens);
  A.k = c.k, A.v = c.v, A.ks = c.k_scale, A.vs = c.v_scale;
  A.kp = c.k_page_stride, A.vp = c.v_page_stride, A.ksp = c.k_scale_page_stride, A.vsp = c.v_scale_page_stride;
  A.heads = c.heads, A.dim = c.dim;
  return A;
}

// f(type of the rows, type held, lanes of a row)
template <typename F>
void with_kinds(int dtype, int held, int dim, F f) {
  auto lanes = [&](auto t, auto h) {
    if (dim <= 32) return f(t, h, std::integral_constant<int, 4>{});
    if (dim <= 64) return f(t, h, std::integral_constant<int, 8>{});
    if (dim <= 128) return f(t, h, std::integral_constant<int, 16>{});
    return f(t, h, std::integral_constant<int, 32>{});
  };
  if (dtype == CFP_DT_F16) return held == CFP_DT_E4M3 ? lanes(f16_t{}, uint8_t{}) : lanes(f16_t{}, f16_t{});
  return held == CFP_DT_E4M3 ? lanes(bf16_t{}, uint8_t{}) : lanes(bf16_t{}, bf16_t{});
}

bool on16(const void *p, HeadStrides s) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s.tok % 8 == 0 && s.head % 8 == 0;
}

}  // namespace

hipError_t launch_cache_write(const cfp_cache_desc &c, const cfp_sequences_desc &s, int64_t n_tokens, int dtype, const void *k,
                              HeadStrides sk, const void *v, HeadStrides sv, hipStream_t st) {
  CacheArgs A = cache_args(c, s, n_tokens);
  A.x[0] = const_cast<void *>(k), A.x[1] = const_cast<void *>(v), A.sx[0] = sk, A.sx[1] = sv;
  A.wide = on16(k, sk) && on16(v, sv);
  const dim3 grid = grid_of(most_units(n_tokens, s.n_seqs) * c.heads);
  with_kinds(dtype, c.dtype, c.dim, [&](auto t, auto h, auto g) {
    cache_write_kernel<decltype(t), decltype(h), g.value><<<grid, kThreads, 0, st>>>(A);
  });
  return hipGetLastError();
}

hipError_t launch_cache_read(const cfp_cache_desc &c, const cfp_sequences_desc &s, int64_t n_tokens, int dtype, void *k,
                             void *v, hipStream_t st) {
  CacheArgs A = cache_args(c, s, n_tokens);
  A.x[0] = k, A.x[1] = v;
  const dim3 grid = grid_of(most_units(n_tokens, s.n_seqs) * c.heads);
  with_kinds(dtype, c.dtype, c.dim, [&](auto t, auto h, auto g) {
    cache_read_kernel<decltype(t), decltype(h), g.value><<<grid, kThreads, 0, st>>>(A);
  });
  return hipGetLastError();
}

}  // namespace cfp
