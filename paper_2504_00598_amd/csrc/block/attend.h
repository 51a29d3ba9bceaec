// Attention of new tokens over a paged cache.
//
// A row is one head of one new token: query q, token p of its sequence.  Over the tokens j that it sees, with
// s_j = scale q . k_j:  m = max s_j,  l = sum exp(s_j - m),  o = sum exp(s_j - m) v_j / l,  lse = m + ln l.
// One pass over the tokens: m and l run along, and what is summed so far is multiplied by exp(m_old - m_new)
// where m grows.  It follows the maximum only when that is far over it, which leaves every ratio as it is.
//
// The heads that share a key head, and the tokens of a chunk, are rows of one product.  Scores are made transposed,
// S^T = K Q^T by 32x32x16 products of 32 tokens and 32 rows: a lane holds one row's scores of 16 tokens, so that
// maxima and sums stay in a lane but for one exchange with the lane's partner, and the weights are the next
// product's operand as they lie: O^T += V^T P^T, whose other operand has its tokens behind each other, as the cache
// holds values.  The product's row i is token 16 (i / 4 % 2) + 4 (i / 8) + i % 4 of the 32: then lane l holds the scores of
// tokens 16 (l / 32) .. + 15 in order, which is what the second product takes from it (8 at a time), and both
// halves of a wave read whole 16-token runs of one page each.
//
// What is masked is left out by a choice, not by arithmetic: scores become -inf, and where a tile that some row sees in part
// holds values that are not finite in the type and under the scale that the product takes them with, these are taken out of the
// product and added to the rows that see them.
//
// Single tokens do 2 (query heads a key head) operations a byte and are bound by memory; chunks by the matrix units, beside
// which the exponentials take as long: 32 x 32 scores at dim 128 are 512 cycles of products and about 450 of vector work a SIMD.
// Measured, 32 or 40 query heads over 8, dim 128 (a copy of 1 GiB reaches 5.1 TB/s, a product of 8192 1.4 PFLOP/s):
//     64 sequences of 16 to 16384 tokens, one new each, bfloat16: 396 us, 5.4 TB/s; 32 of 4000 to 12000 in 8 bits: 102 us,
//     5.2 TB/s; one of 777 in 13 us: starts, then the table, then keys and values, two steps of 256 tokens in its first part;
//     8192 new of 32768 tokens, bfloat16: 3530 us, 1.09 PFLOP/s; 2048 of 8192 in 8 bits: 316 to 343 us, 0.72 to 0.77 PFLOP/s.
// The chunk's kernel keeps the matrix unit busy half of its cycles at about 2.1 GHz.  What it was before, for the first of these
// chunks: 128 rows a workgroup, two of them a compute unit, tiles through registers 6800 us; 64 rows a wave so that
// an operand read from LDS serves two products, one wave a SIMD, with copies straight to LDS one tile ahead 8500, two ahead 4950, the
// pages of a tile chosen by masks and not by an index 4060, the first operands of a stage read in the one before it 3860;
// eight waves of 32 rows, two a SIMD, which hide each other's waits, 3640 (on another card 3530).
#pragma once

#include <algorithm>
#include <type_traits>

#include "cache_common.h"

namespace cfp {

constexpr int kTokenRows = 16, kFewRows = 32;  // rows of a sequence and key head that the kernels for few take
constexpr int kManyRows = 128;  // rows of a workgroup of the kernel for many, and of the one for heads up to 128
constexpr int kWideRows = 256, kWideDim = 128;
constexpr int kFewParts = 768;
constexpr int kFewStep = 64, kManyStep = 64;     // parts start and end on these
constexpr int kFewLeast = 256, kTokenLeast = 512, kManyLeast = 256;  // tokens of a part, at least
constexpr int kGroups = 256, kSpare = 16, kManyRounds = 2;  // workgroups at a time; more that are no round; rounds up to which tiles are cut
constexpr int kUncut = 1 << 30;
constexpr int kJoinThreads = 256;

struct AttendArgs {
  SeqArgs s;
  const void *q, *k, *v;
  const uint8_t *ks, *vs;
  int64_t kp, vp, ksp, vsp;  // strides of pages
  int64_t qt, qh;            // strides of tokens and heads
  void *out;
  float *lse;
  float *few_o, *few_ml, *many_o, *many_ml;  // parts: sums over exp(s - m), and m (in powers of two) and l
  int32_t heads, group, dim, max_new;
  int32_t causal, window, wide;  // wide: queries lie on 16 bytes
  int32_t few_units, few_target;  // parts of all sequences with few rows: at most, and for their tokens alone
  int32_t few_least;              // tokens of a part, at least
  int32_t few_rows, joined;       // few_rows: of a sequence and key head, at most; joined: there may be parts
  int32_t *plan;                  // how the other sequences are cut: tokens of a part, parts of all tiles
  int32_t many_rows;              // of a workgroup
  uint32_t tiles, many_units;     // of many_rows rows, and their parts, at most
  uint32_t many_most;             // parts where tiles are cut, at most; 0: they never are
  int32_t many_joined;            // workgroups that join those parts
  float scale;     // times log2(e)
};

hipError_t attend_bf16(const AttendArgs &A, bool bytes, hipStream_t st);
hipError_t attend_f16(const AttendArgs &A, bool bytes, hipStream_t st);

#ifdef __HIPCC__

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// How far below the running maximum (in powers of two) m is set, and how far the maximum may grow above that before m
// follows.  The range of the weights' type is used: bfloat16 has that of 32 bits, so weights up to 2^20 lose nothing, and
// multiplying what is summed so far, which a wave does when one of its rows asks for it, stays rare.  float16 has no bits below
// 2^-24 and ends at 2^16: m stays 8 below the maximum, and weights go up to 2^14.
template <typename T>
constexpr float kBelow = std::is_same<T, f16_t>::value ? 8.f : 0.f;
template <typename T>
constexpr float kGrowth = std::is_same<T, f16_t>::value ? 14.f : 20.f;
constexpr float kLn2F = 0.693147180559945309f;

template <typename T>
__device__ __forceinline__ f32x16 mfma32(vec<T, 8> a, vec<T, 8> b, f32x16 c) {
  if constexpr (std::is_same<T, bf16_t>::value)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// The other half's value.
__device__ __forceinline__ float partner(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// 8 entries of 8 bits times a power of two.
template <typename T>
__device__ __forceinline__ vec<T, 8> widen(u32x2 w, float s) {
  vec<T, 8> r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (std::is_same<T, bf16_t>::value) {
      const auto a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], s, false);
      const auto b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], s, true);
      r[4 * i] = a[0], r[4 * i + 1] = a[1], r[4 * i + 2] = b[0], r[4 * i + 3] = b[1];
    } else {
      const auto a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], s, false);
      const auto b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], s, true);
      r[4 * i] = a[0], r[4 * i + 1] = a[1], r[4 * i + 2] = b[0], r[4 * i + 3] = b[1];
    }
  }
  return r;
}

// 8 entries of 8 bits, each times a power of two of its own (scale bytes).
template <typename T>
__device__ __forceinline__ vec<T, 8> widen(u32x2 w, u32x2 s) {
  vec<T, 8> r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
    const float x[4] = {a[0], a[1], b[0], b[1]};
#pragma unroll
    for (int j = 0; j < 4; ++j) r[4 * i + j] = (T)(x[j] * scale_of(s[i] >> (8 * j) & 0xff));
  }
  return r;
}

// What rows with first and last token p0 <= p1 of a sequence of `len` see, cut into parts of `per`.
struct Span {
  int32_t begin, end, parts;
};
__device__ __forceinline__ Span span_of(const AttendArgs &A, int p0, int p1, int len, int per) {
  Span r;
  r.end = A.causal ? p1 + 1 : len;
  r.begin = (A.window > 0 ? max(p0 - A.window + 1, 0) : 0) & ~(kManyStep - 1);
  const int n = r.end - r.begin;
  r.parts = n > 0 ? (n + per - 1) / per : 0;
  return r;
}

// Sequences with many rows: their tiles of rows, the most tokens that one of these sees, into how many parts each is cut.
__device__ __forceinline__ uint32_t many_tiles(const AttendArgs &A, const Seq &q) {
  const int64_t r = (int64_t)q.n * A.group;
  const bool many = r > A.few_rows && q.n <= A.max_new && q.pos + q.n <= (A.s.width << A.s.page_shift);
  return many ? (uint32_t)((r + A.many_rows - 1) / A.many_rows) : 0u;
}
__device__ __forceinline__ int many_span(const AttendArgs &A, const Seq &q) {
  const int len = q.pos + q.n;
  return A.causal && A.window > 0 ? min(len, A.window + A.many_rows / A.group + kManyStep + 1) : len;
}
__device__ __forceinline__ uint32_t many_parts(const AttendArgs &A, const Seq &q, int per) {
  return (uint32_t)max((many_span(A, q) + per - 1) / per, 1);
}
__device__ __forceinline__ uint32_t many_units(const AttendArgs &A, const Seq &q, int per) {
  const uint32_t tiles = many_tiles(A, q);
  return tiles ? tiles * many_parts(A, q, per) : 0u;
}
// One wave of the first kernel cuts them for the ones that follow: into parts of the same length, so that workgroups have equal work, no
// more of them than fill the rounds that the tiles take anyhow.  A workgroup fills a compute unit; its time is its 64-token
// steps and about five that it takes before the first and behind the last; a launch more joins the parts (three).  Whole tiles in more
// than one round take their mean time, and half of the longest's as the last ones end.  The tiles stay whole
// where parts save less than an eighth, and where they take more than two rounds.  (A chunk of 108 rows in two tiles of 8 heads over
// 12009 tokens of dim 192, beside six single tokens: cut by bounds that the host knows, as if these might be chunks too, 210 us.)
__device__ __forceinline__ void plan_many(const AttendArgs &A) {
  const int lane = threadIdx.x & 63;
  float work = 0.f;
  uint32_t tiles = 0;
  int longest = 0;
  Seq q = {0, 0, 0};  // up to 64 sequences are read once
  for (int first = 0; first < A.s.n_seqs; first += 64) {
    q = {0, 0, 0};
    if (first + lane < A.s.n_seqs) q = seq_of(A.s, first + lane);
    const uint32_t t = many_tiles(A, q);
    const int span = t ? many_span(A, q) : 0;
    // of a chunk that sees itself as a triangle half of it
    work += (float)t * (float)(A.causal ? max(span - q.n / 2, span / 2) : span), tiles += t, longest = max(longest, span);
  }
  work = group_sum<64>(work);
  tiles = (uint32_t)__builtin_amdgcn_readlane((int)lanes_before(tiles), 63);
  for (int m = 32; m > 0; m /= 2) longest = max(longest, __shfl_xor(longest, m));
  int per = kUncut;
  uint32_t units = tiles;
  const int64_t rounds = (max((int64_t)tiles * A.heads - kSpare, (int64_t)1) + kGroups - 1) / kGroups;
  const uint32_t most = min((uint32_t)(rounds * kGroups / A.heads), A.many_most);
  if (tiles && most && rounds <= kManyRounds) {
    auto step = [](int n) { return (n + kManyStep - 1) & ~(kManyStep - 1); };
    const float steps = (float)longest / kManyStep + 5.f;
    const float whole = rounds == 1 ? steps : (work / kManyStep + 5.f * (float)tiles) * (float)A.heads / kGroups + steps / 2;
    int p = max(max(step((int)fminf(work / (float)most, 0x1p29f) + 1), step(longest / 64)), kManyLeast);
    for (;; p += max(p / 32 & ~(kManyStep - 1), kManyStep)) {
      p = __builtin_amdgcn_readfirstlane(p);
      if ((float)rounds * ((float)p / kManyStep + 5.f) + 3.f >= whole * 7 / 8) break;  // and so for all that are longer
      uint32_t u = 0;
      if (A.s.n_seqs <= 64)
        u = many_units(A, q, p);
      else
        for (int first = 0; first < A.s.n_seqs; first += 64)
          if (first + lane < A.s.n_seqs) u += many_units(A, seq_of(A.s, first + lane), p);
      u = (uint32_t)__builtin_amdgcn_readlane((int)lanes_before(u), 63);
      if (u > most) continue;
      per = p, units = u;
      break;
    }
  }
  if (lane == 0) A.plan[0] = per, A.plan[1] = (int32_t)units;
}
// What it wrote, in kernels behind that one.
struct Plan {
  int32_t per, units;
};
__device__ __forceinline__ Plan plan_of(const AttendArgs &A) {
  const const_i32 *p = reinterpret_cast<const const_i32 *>(reinterpret_cast<uintptr_t>(A.plan));
  return {p[0], p[1]};
}

// Sequences with few rows are cut into parts of `per` tokens, the same for all, so that workgroups have equal work.
struct Few {
  bool lost;     // longer than its table, or more rows than the call was laid out for
  bool few;
  int32_t tokens;  // that some row sees, from a multiple of kFewStep on
};
__device__ __forceinline__ Few few_of(const AttendArgs &A, const Seq &q) {
  const int len = q.pos + q.n;
  Few f;
  f.lost = q.n > 0 && (q.n > A.max_new || len > (A.s.width << A.s.page_shift));
  f.few = q.n > 0 && !f.lost && (int64_t)q.n * A.group <= A.few_rows;
  const int begin = (A.window > 0 ? max(q.pos - A.window + 1, 0) : 0) & ~(kFewStep - 1);
  f.tokens = f.few ? max(len - begin, 0) : 0;
  return f;
}
__device__ __forceinline__ uint32_t few_parts(const AttendArgs &A, const Seq &q, int per) {
  const Few f = few_of(A, q);
  return f.lost ? 1u : f.few ? max((uint32_t)((f.tokens + per - 1) / per), 1u) : 0u;
}
__device__ __forceinline__ int few_share(const AttendArgs &A, float tokens) {
  const int per = (int)fminf(ceilf(tokens * 1.002f / (float)A.few_target), 0x1p30f);  // no sequence is longer
  return __builtin_amdgcn_readfirstlane(max((per + kFewStep - 1) & ~(kFewStep - 1), A.few_least));
}
// All 64 lanes of a wave call it.  The sum, of up to 2^20 sequences by 64 lanes, is in 32-bit floats and so at most 0.1% too
// small: the share is taken that much larger, so that there are never more than few_target parts beside each
// sequence's last.
__device__ __forceinline__ int few_per(const AttendArgs &A) {
  float sum = 0.f;
  for (int first = 0; first < A.s.n_seqs; first += 64) {
    const int b = first + (threadIdx.x & 63);
    sum += group_sum<64>(b < A.s.n_seqs ? (float)few_of(A, seq_of(A.s, b)).tokens : 0.f);
  }
  return few_share(A, sum);
}
// Sequence, part and tokens of a part of a workgroup `unit`; false: there is none.  Up to 64 sequences are looked at once.
__device__ __forceinline__ bool find_few(const AttendArgs &A, uint32_t unit, int &b, uint32_t &part, Seq &q, int &per) {
  if (A.s.n_seqs > 64) {
    per = few_per(A);
    return find_unit(A.s, unit, [&](const Seq &s) { return few_parts(A, s, per); }, b, part, q);
  }
  const int lane = threadIdx.x & 63;
  Seq s = {0, 0, 0};
  if (lane < A.s.n_seqs) s = seq_of(A.s, lane);
  per = few_share(A, group_sum<64>((float)few_of(A, s).tokens));
  const uint32_t own = few_parts(A, s, per), sum = lanes_before(own);
  const uint64_t past = __ballot(sum > unit);
  if (past == 0) return false;
  b = __builtin_ctzll(past);
  q = seq_of_lane(s, b);
  part = unit - (uint32_t)__builtin_amdgcn_readlane((int)(sum - own), b);
  return true;
}

// Query of a row as the second operand: entries of its d-th piece of 8.
template <typename T>
__device__ __forceinline__ vec<T, 8> load_q(const T *q, int d, int dim, bool there, bool wide) {
  vec<T, 8> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (T)0.f;
  if (there && d < dim) {
    if (wide) {
      r = *reinterpret_cast<const vec<T, 8> *>(q + d);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = q[d + i];
    }
  }
  return r;
}

// What is infinite or not a number among a word's two entries (the first in the lowest bits): cleared in the word, and
// its bits by sign in `up` and `down` (what is not a number is both).
template <typename T>
__device__ __forceinline__ uint32_t take_odd(uint32_t w, uint32_t &up, uint32_t &down) {
  constexpr uint32_t kInf = std::is_same<T, bf16_t>::value ? 0x7f80 : 0x7c00;
  up = down = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t x = w >> (16 * i) & 0xffff;
    if ((x & kInf) != kInf) continue;
    if ((x & 0x7fff) != kInf || !(x & 0x8000)) up |= 1u << i;
    if ((x & 0x7fff) != kInf || (x & 0x8000)) down |= 1u << i;
    w &= ~(0xffffu << (16 * i));
  }
  return w;
}
// The same of 16 bytes.
template <typename T>
__device__ __forceinline__ void take_odd(u32x4 &w, uint32_t &up, uint32_t &down) {
  up = down = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t u, d;
    w[i] = take_odd<T>(w[i], u, d);
    up |= u << (2 * i), down |= d << (2 * i);
  }
}

// Scale bytes of 255 as 254.  No token that was written has one, but an unwritten place may: its scale would be infinite, and times
// a weight of zero no number.  For tiles that some row sees in part.
__device__ __forceinline__ u32x4 finite_scales(u32x4 w) {
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] -= (((w[i] & 0x7f7f7f7fu) + 0x01010101u) & w[i] & 0x80808080u) >> 7;
  return w;
}

// Of 16 tokens with the scales s (none of them 255) the least magnitude, as a byte of 8 bits without its sign, that is not finite once
// it is widened to T: that of 2^k with k = 16 (float16) or 128 less the scale's exponent, as nothing that is held lies between T's
// largest value and that power; any but zero where k is below the least that is held, and only what is not a number where
// 448 stays in the range, as it does under every scale that was written for rows of T.
template <typename T>
__device__ __forceinline__ u32x4 odd_from(u32x4 s) {
  constexpr bool kHalf = std::is_same<T, f16_t>::value;
  constexpr int kTop = kHalf ? 127 + 16 : 127 + 128;
  constexpr uint32_t kLow = (kTop - 8 - 128) * 0x01010101u;  // scales from kTop - 8 on, without their highest bits
  uint32_t large = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) large |= ((s[i] | 0x80808080u) - kLow) & s[i];
  u32x4 r = {0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
  if (large & 0x80808080u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = kTop - (int)(s[i] >> (8 * j) & 0xff);
        w |= (uint32_t)(k > 8 ? 0x7f : k >= -6 ? 8 * (k + 7) : 8 >> min(-6 - k, 3)) << (8 * j);
      }
      r[i] = w;
    }
  }
  return r;
}
// take_odd of 16 entries of 8 bits: those from the magnitudes `least` on.
__device__ __forceinline__ void take_odd_bytes(u32x4 &w, u32x4 least, uint32_t &up, uint32_t &down) {
  constexpr uint32_t kSigns = 0x80808080u;
  up = down = 0;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) any |= (w[i] | kSigns) - least[i];  // no byte borrows from the next: least is 1 to 0x7f
  if (any & kSigns) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t odd = ((w[i] | kSigns) - least[i]) & kSigns, nan = ((w[i] | kSigns) - 0x7f7f7f7fu) & kSigns;
      auto four = [](uint32_t x) { return (x >> 7) * 0x01020408u >> 24; };  // the bytes' highest bits behind each other
      up |= four(odd & (~w[i] | nan)) << (4 * i), down |= four(odd & (w[i] | nan)) << (4 * i);
      w[i] &= ~((odd >> 7) * 0xffu);
    }
  }
}

// One row's running state and its scores of a tile of 16 N tokens a lane.
template <typename T, int DP>
struct Rows {
  float m, l;            // l: of this lane's tokens
  f32x16 o[DP / 32];
  uint32_t odd[DP / 32];  // infinities to be added to an entry of o: two bits each, of either sign

  __device__ __forceinline__ void clear() {
    m = -__builtin_inff(), l = 0.f;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {
      odd[i] = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    }
  }

  // The tokens (a bit each) that this lane's row sees hold infinities of either sign in its entry j of o[i].
  __device__ __forceinline__ void add_odd(int i, int j, bool up, bool down) {
    odd[i] |= (up ? 1u : 0u) << (2 * j) | (down ? 2u : 0u) << (2 * j);
  }
  __device__ __forceinline__ void finish() {
    l += partner(l);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
      if (__any(odd[i] != 0)) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          o[i][j] += odd[i] >> (2 * j) & 1 ? __builtin_inff() : 0.f;
          o[i][j] -= odd[i] >> (2 * j) & 2 ? __builtin_inff() : 0.f;
        }
      }
  }

  // The weights as the next product's operands.
  template <int N>
  __device__ __forceinline__ void pack(const f32x16 (&s)[N], vec<T, 8> (&p)[2 * N]) {
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) p[2 * u + i / 8][i % 8] = (T)s[u][i];
  }

  // Scores to weights exp2(c s - m).
  template <int N>
  __device__ __forceinline__ void weigh(f32x16 (&s)[N], float c) {
    float top = s[0][0];
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
    top = fmaxf(top, partner(top)) * c;
    if (__any(top > m + kGrowth<T>)) {
      const float to = top > m + kGrowth<T> ? top - kBelow<T> : m;
      const float by = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= by;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] *= by;
    }
    const float from = m == -__builtin_inff() ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[u][i], c, -from));
        s[u][i] = e;
        sum += e;
      }
    l += sum;
  }
};

// Where values of 8 bits are times their tokens' powers of two: bfloat16 has the range of 32 bits, so there the weights
// take them (16 products a lane and 32 tokens); float16's weights could not hold them, and the values do.
template <typename T, bool BYTES>
constexpr bool kWeightsScaled = BYTES && std::is_same<T, bf16_t>::value;

// s times the 16 scales whose bytes are w.
__device__ __forceinline__ void times_scales(f32x16 &s, u32x4 w) {
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] *= scale_of(w[i / 4] >> (8 * (i % 4)) & 0xff);
}

// The largest of three, without a step for each operand that makes signalling NaN quiet.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// Pages of four runs of 16 tokens, as the table has them, and one of them: by masks, as the compiler would make an array in
// memory of what is chosen by an index.
struct Pages4 {
  uint32_t a, b, c, d;
};
__device__ __forceinline__ uint32_t one_of(const Pages4 &p, int i) {
  const uint32_t low = 0u - (uint32_t)(i & 1), high = 0u - (uint32_t)(i >> 1 & 1);
  return (((p.a & ~low) | (p.b & low)) & ~high) | (((p.c & ~low) | (p.d & low)) & high);
}

// The lowest n of 32 bits, all for n >= 32 and none for n <= 0.
__device__ __forceinline__ uint32_t bits_of(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1; }

// Scores that a lane's row does not see; `bad`: the lane's 16 tokens have no page.
__device__ __forceinline__ void mask16(f32x16 &s, int first, int lo, int hi, bool bad) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float x = bad ? __builtin_nanf("") : s[i];
    s[i] = first + i >= lo && first + i <= hi ? x : -__builtin_inff();
  }
}

// What the rows of a sequence become that is too long for its table, or has more rows than the call was laid out for.
template <typename T, int THREADS>
__device__ __forceinline__ void write_lost(const AttendArgs &A, const Seq &sq, int head) {
  const int g = A.group, hq = A.heads * g, D = A.dim;
  for (int64_t e = threadIdx.x; e < (int64_t)sq.n * g * D; e += THREADS) {
    const int64_t r = e / D;
    const int64_t row = (sq.row + r / g) * hq + head * g + r % g;
    reinterpret_cast<T *>(A.out)[row * D + e % D] = (T)__builtin_nanf("");
    if (e % D == 0 && A.lse) A.lse[row] = __builtin_nanf("");
  }
}

// The sums of the waves, laid out in LDS [wave][few_rows][LD] relative to the largest m, to their rows or as a part.
template <typename T, int WAVES, int ROWS, int LD>
__device__ __forceinline__ void write_few(const AttendArgs &A, const float *shared, const float (&ml)[2][WAVES][ROWS], const Seq &sq,
                                          int head, int rows, bool whole, int64_t slot) {
  const int g = A.group, hq = A.heads * g, D = A.dim, quads = D / 4;
  for (int e = threadIdx.x; e < rows * quads; e += 64 * WAVES) {
    const int r = e / quads, d = e % quads * 4;
    float top = ml[0][0][r];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, ml[0][w][r]);
    float l = 0.f;
    vec<float, 4> o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      l += ml[1][w][r] * (ml[0][w][r] == top ? 1.f : __builtin_amdgcn_exp2f(ml[0][w][r] - top));
      o += *reinterpret_cast<const vec<float, 4> *>(shared + (w * A.few_rows + r) * LD + d);
    }
    if (whole) {
      const int64_t row = (int64_t)(sq.row + r / g) * hq + head * g + r % g;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const float y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
      store_vec<T, 4>(reinterpret_cast<T *>(A.out) + row * D + d, y);
      if (d == 0 && A.lse) A.lse[row] = (top + __builtin_amdgcn_logf(l)) * kLn2F;
    } else {
      *reinterpret_cast<vec<float, 4> *>(A.few_o + (slot + r) * D + d) = o;
      if (d == 0) A.few_ml[2 * (slot + r)] = top, A.few_ml[2 * (slot + r) + 1] = l;
    }
  }
}

// ---- up to 16 rows, as a token's heads that share a key head are: like the kernel for up to 32 below, with 16x16x32 products of
// 16 tokens and 16 rows and 64 tokens a wave at a time.  Row i of product u is token 16 (i / 4) + 4 u + i % 4, so lane l has
// scores of tokens 16 (l / 16) .. + 15 of row l % 16, which are its share of the two products with the values.  Half the
// registers of the wider products, so twice the bytes are on their way, and half the exponentials (64 uneven contexts:
// 516 us with the wider ones, 32 in 8 bits 170).
typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename T>
__device__ __forceinline__ f32x4 mfma16(vec<T, 8> a, vec<T, 8> b, f32x4 c) {
  if constexpr (std::is_same<T, bf16_t>::value)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
constexpr int kTokenWaves = 4;  // of a workgroup
// op over the four lanes of a row
__device__ __forceinline__ float row_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <typename T, bool BYTES, int DP>
__global__ __launch_bounds__(64 * kTokenWaves, DP <= 128 ? 2 : 1) void attend_token_kernel(AttendArgs A) {
  typedef std::conditional_t<BYTES, uint8_t, T> H;
  typedef vec<T, 8> Vec8;
  constexpr int kC = DP / 32, kMt = DP / 16, kLd = DP + 4, kWaves = kTokenWaves, kStep = 64 * kWaves;
  constexpr int kK = BYTES ? DP / 64 : DP / 32;  // loads of a key
  static_assert(!BYTES || DP % 64 == 0, "keys of 8 bits are read 64 entries at a time");
  extern __shared__ __align__(16) float shared[];
  __shared__ float ml[2][kWaves][kTokenRows];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, h = lane >> 4;
  const uint32_t id = block_id(), unit = id / A.heads;
  const int head = (int)(id % A.heads);
  int b, per;
  uint32_t part;
  Seq sq;
  if (A.tiles && id == (uint32_t)A.few_units * A.heads - 1 && wave == 0) plan_many(A);
  if (unit >= (uint32_t)A.few_units || !find_few(A, unit, b, part, sq, per)) return;
  const Few few = few_of(A, sq);
  const int g = A.group, D = A.dim;
  if (few.lost) return write_lost<T, kStep>(A, sq, head);
  const int rows = sq.n * g, len = sq.pos + sq.n;
  const bool whole = few.tokens <= per;
  const int begin = len - few.tokens + (int)part * per, end = min(len, begin + per);
  const int i = col / g, p = sq.pos + i;
  const bool mine = col < rows;
  const int hi = mine ? (A.causal ? p : len - 1) : -1, lo = A.window > 0 ? p - A.window + 1 : 0;
  const int all_hi = A.causal ? sq.pos : len - 1, all_lo = A.window > 0 ? len - A.window : 0;  // seen by all rows

  Vec8 q[kC];
  const T *qp = reinterpret_cast<const T *>(A.q) + (int64_t)(sq.row + i) * A.qt + (int64_t)(head * g + col % g) * A.qh;
#pragma unroll
  for (int c = 0; c < kC; ++c)
    q[c] = load_q<T>(qp, BYTES ? 64 * (c / 2) + 16 * h + 8 * (c % 2) : 32 * c + 8 * h, D, mine, A.wide != 0);

  const int page = 1 << A.s.page_shift, inner = page - 1;
  const TableRow table = table_row(A.s, b);
  auto pages = [&](int t) { return Pages4{table.entry(t), table.entry(t + 16), table.entry(t + 32), table.entry(t + 48)}; };
  auto inside = [&](uint32_t e) { return e < A.s.n_pages; };
  auto pick = [&](const Pages4 &pg, int j) -> int64_t {
    const uint32_t e = one_of(pg, j);
    return inside(e) ? e : 0u;
  };
  const int kq = col >> 2;  // the 16 tokens that this lane's keys are of: 16 kq + 4 u + col % 4
  const H *kbase = reinterpret_cast<const H *>(A.k) + (int64_t)(head * page + (col & 3)) * D + (BYTES ? 16 : 8) * h;
  const H *vbase = reinterpret_cast<const H *>(A.v) + (int64_t)(head * D + col) * page;
  u32x4 kr[4][kK], vr[kMt][BYTES ? 1 : 2], ksr, vsr;
  auto load_k = [&](int t, const Pages4 &pg) {
    const int64_t at = pick(pg, kq);
    const int place = (t + 16 * kq) & inner;
    const H *kp = kbase + at * A.kp + place * D;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int c = 0; c < kK; ++c) {
        const int d = BYTES ? 64 * c : 32 * c;
        u32x4 w = {0, 0, 0, 0};
        if (d + (BYTES ? 16 : 8) * h < D) w = *reinterpret_cast<const u32x4 *>(kp + 4 * u * D + d);
        kr[u][c] = w;
      }
    if constexpr (BYTES) ksr = *reinterpret_cast<const u32x4 *>(A.ks + at * A.ksp + head * page + place);
  };
  auto load_v = [&](int t, const Pages4 &pg) {
    const int64_t at = pick(pg, h);
    const int place = (t + 16 * h) & inner;
    const H *vp = vbase + at * A.vp + place;
#pragma unroll
    for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
      for (int j = 0; j < (BYTES ? 1 : 2); ++j) {
        u32x4 w = {0, 0, 0, 0};
        if (16 * mt < D) w = *reinterpret_cast<const u32x4 *>(vp + 16 * mt * page + 8 * j);
        vr[mt][j] = w;
      }
    if constexpr (BYTES) vsr = *reinterpret_cast<const u32x4 *>(A.vs + at * A.vsp + head * page + place);
  };

  float m = -__builtin_inff(), l = 0.f;
  f32x4 o[kMt];
  uint64_t odd[(DP + 127) / 128];  // as in Rows, two bits for each of the 4 kMt entries
#pragma unroll
  for (int x = 0; x < (DP + 127) / 128; ++x) odd[x] = 0;
#pragma unroll
  for (int mt = 0; mt < kMt; ++mt) o[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
  uint32_t *odds = reinterpret_cast<uint32_t *>(shared) + wave * 4 * DP;  // [16 tokens][entry]: bits of either sign
  int t = begin + 64 * wave;
  if (t < end) {
    Pages4 now = pages(t), next = now;
    load_k(t, now);
    load_v(t, now);
    if (t + kStep < end) next = pages(t + kStep);
    for (; t < end; t += kStep) {
      Pages4 later = next;
      if (t + 2 * kStep < end) later = pages(t + 2 * kStep);
      f32x4 s[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (BYTES) {
          const float by = scale_of(ksr[u] >> (8 * (col & 3)) & 0xff);
#pragma unroll
          for (int c = 0; c < kK; ++c) {
            s[u] = mfma16<T>(widen<T>(u32x2{kr[u][c][0], kr[u][c][1]}, by), q[2 * c], s[u]);
            s[u] = mfma16<T>(widen<T>(u32x2{kr[u][c][2], kr[u][c][3]}, by), q[2 * c + 1], s[u]);
          }
        } else {
#pragma unroll
          for (int c = 0; c < kK; ++c) s[u] = mfma16<T>(__builtin_bit_cast(Vec8, kr[u][c]), q[c], s[u]);
        }
      }
      if (t + kStep < end) load_k(t + kStep, next);
      const int first = t + 16 * h;
      const bool edge = t + 63 > all_hi || t < all_lo || !(inside(now.a) && inside(now.b) && inside(now.c) && inside(now.d));
      if (edge) {
        const bool bad = !inside(one_of(now, h));
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float x = bad ? __builtin_nanf("") : s[e / 4][e % 4];
          s[e / 4][e % 4] = first + e >= lo && first + e <= hi ? x : -__builtin_inff();
        }
        if constexpr (BYTES) vsr = finite_scales(vsr);
      }
      float top = s[0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e / 4][e % 4]);
      top = row_max(top) * A.scale;
      if (__any(top > m + kGrowth<T>)) {
        const float to = top > m + kGrowth<T> ? top - kBelow<T> : m;
        const float by = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= by;
#pragma unroll
        for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[mt][r] *= by;
      }
      const float from = m == -__builtin_inff() ? 0.f : m;
      Vec8 w[2];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x = __builtin_amdgcn_exp2f(fmaf(s[e / 4][e % 4], A.scale, -from));
        l += x;
        if constexpr (kWeightsScaled<T, BYTES>) x *= scale_of(vsr[e / 4] >> (8 * (e % 4)) & 0xff);
        w[e / 8][e % 8] = (T)x;
      }
      if (edge) {
        bool any = false;
        u32x4 least = {0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
        if constexpr (BYTES && !kWeightsScaled<T, BYTES>) least = odd_from<T>(vsr);
#pragma unroll
        for (int mt = 0; mt < kMt; ++mt) {
          uint32_t up, down;
          if constexpr (BYTES) {
            take_odd_bytes(vr[mt][0], least, up, down);
          } else {
            uint32_t up1, down1;
            take_odd<T>(vr[mt][0], up, down);
            take_odd<T>(vr[mt][1], up1, down1);
            up |= up1 << 8, down |= down1 << 8;
          }
          odds[h * DP + 16 * mt + col] = up | down << 16;
          any = any || up != 0 || down != 0;
        }
        if (__any(any)) {
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
          __builtin_amdgcn_wave_barrier();
          __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t sees = bits_of(hi + 1 - t - 16 * x) & ~bits_of(lo - t - 16 * x);
#pragma unroll
            for (int e = 0; e < 4 * kMt; ++e) {
              const uint32_t a = odds[x * DP + 16 * (e / 4) + 4 * h + e % 4];
              odd[e / 32] |= (uint64_t)((a & sees & 0xffff ? 1u : 0u) | (a >> 16 & sees ? 2u : 0u)) << (2 * (e % 32));
              __builtin_amdgcn_sched_barrier(0);  // one after the other: seldom run, and not worth registers
            }
          }
        }
      }
#pragma unroll
      for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          Vec8 v;
          if constexpr (kWeightsScaled<T, BYTES>)
            v = widen<T>(u32x2{vr[mt][0][2 * j], vr[mt][0][2 * j + 1]}, 1.f);
          else if constexpr (BYTES)
            v = widen<T>(u32x2{vr[mt][0][2 * j], vr[mt][0][2 * j + 1]}, u32x2{vsr[2 * j], vsr[2 * j + 1]});
          else
            v = __builtin_bit_cast(Vec8, vr[mt][j]);
          o[mt] = mfma16<T>(v, w[j], o[mt]);
        }
      if (t + kStep < end) load_v(t + kStep, next);
      now = next, next = later;
    }
  }

  // the waves' states together
  l = row_sum(l);
#pragma unroll
  for (int x = 0; x < (DP + 127) / 128; ++x)
    if (__any(odd[x] != 0)) {
#pragma unroll
      for (int e = 0; e < 32 && 32 * x + e < 4 * kMt; ++e) {
        const int mt = (32 * x + e) / 4;
        o[mt][e % 4] += odd[x] >> (2 * e) & 1 ? __builtin_inff() : 0.f;
        o[mt][e % 4] -= odd[x] >> (2 * e) & 2 ? __builtin_inff() : 0.f;
      }
    }
  if (h == 0) ml[0][wave][col] = m, ml[1][wave][col] = l;
  __syncthreads();
  float top = ml[0][0][col];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) top = fmaxf(top, ml[0][w][col]);
  const float by = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
  if (mine) {
    float *to = shared + (wave * A.few_rows + col) * kLd + 4 * h;
#pragma unroll
    for (int mt = 0; mt < kMt; ++mt) *reinterpret_cast<f32x4 *>(to + 16 * mt) = o[mt] * by;
  }
  __syncthreads();
  write_few<T, kWaves, kTokenRows, kLd>(A, shared, ml, sq, head, rows, whole, (int64_t)id * A.few_rows);
}

// ---- few rows: a workgroup takes a part of one sequence's tokens for one key head and up to 32 rows.  Each of its
// four waves takes every fourth tile of 32 tokens, operands from memory straight to the matrix instructions'
// registers (16 bytes a lane, the next tile's keys loaded while this one's scores become weights, its values
// while the next scores are made), and a state of its own; the four meet in LDS.
template <typename T, bool BYTES, int DP>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void attend_few_kernel(AttendArgs A) {
  typedef std::conditional_t<BYTES, uint8_t, T> H;
  typedef vec<T, 8> Vec8;
  constexpr int kK = BYTES ? DP / 32 : DP / 16, kLd = DP + 4;
  extern __shared__ __align__(16) float shared[];
  __shared__ float ml[2][4][kFewRows];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5;
  const uint32_t id = block_id(), unit = id / A.heads;
  const int head = (int)(id % A.heads);
  int b, per;
  uint32_t part;
  Seq sq;
  if (A.tiles && id == (uint32_t)A.few_units * A.heads - 1 && wave == 0) plan_many(A);
  if (unit >= (uint32_t)A.few_units || !find_few(A, unit, b, part, sq, per)) return;
  const Few few = few_of(A, sq);
  const int g = A.group, D = A.dim;
  if (few.lost) return write_lost<T, 256>(A, sq, head);
  const int rows = sq.n * g, len = sq.pos + sq.n;
  const bool whole = few.tokens <= per;
  const int begin = len - few.tokens + (int)part * per, end = min(len, begin + per);
  const int i = col / g;
  const int p = sq.pos + i;
  const bool mine = col < rows;
  const int hi = mine ? (A.causal ? p : len - 1) : -1, lo = A.window > 0 ? p - A.window + 1 : 0;
  const int all_hi = A.causal ? sq.pos : len - 1, all_lo = A.window > 0 ? len - A.window : 0;  // seen by all rows

  vec<T, 8> q[DP / 16];
  const T *qp = reinterpret_cast<const T *>(A.q) + (int64_t)(sq.row + i) * A.qt + (int64_t)(head * g + col % g) * A.qh;
#pragma unroll
  for (int c = 0; c < DP / 16; ++c)
    q[c] = load_q<T>(qp, BYTES ? 32 * (c / 2) + 16 * h + 8 * (c % 2) : 16 * c + 8 * h, D, mine, A.wide != 0);

  const int page = 1 << A.s.page_shift, inner = page - 1;
  const int ki = 16 * (col >> 2 & 1) + 4 * (col >> 3) + (col & 3);  // token of this lane's key
  u32x4 kr[kK], vr[DP / 32][BYTES ? 1 : 2], vsr;
  uint32_t ksr = 0;

  struct Pages {
    uint32_t at[2];  // as the table has them
  };
  const TableRow table = table_row(A.s, b);
  auto pages = [&](int t) { return Pages{{table.entry(t), table.entry(t + 16)}}; };
  auto inside = [&](uint32_t page) { return page < A.s.n_pages; };
  auto load_k = [&](int t, const Pages &pg) {
    const uint32_t entry = col & 4 ? pg.at[1] : pg.at[0], at = inside(entry) ? entry : 0u;
    const int place = (t + ki) & inner;
    const H *kp = reinterpret_cast<const H *>(A.k) + at * A.kp + (int64_t)(head * page + place) * D;
#pragma unroll
    for (int c = 0; c < kK; ++c) {
      const int d = BYTES ? 32 * c + 16 * h : 16 * c + 8 * h;
      u32x4 w = {0, 0, 0, 0};
      if (d < D) w = *reinterpret_cast<const u32x4 *>(kp + d);
      kr[c] = w;
    }
    if constexpr (BYTES) ksr = A.ks[at * A.ksp + head * page + place];
  };
  auto load_v = [&](int t, const Pages &pg) {
    const uint32_t entry = h ? pg.at[1] : pg.at[0], at = inside(entry) ? entry : 0u;
    const int place = (t + 16 * h) & inner;
    const H *vp = reinterpret_cast<const H *>(A.v) + at * A.vp + (int64_t)head * D * page + place;
#pragma unroll
    for (int mt = 0; mt < DP / 32; ++mt) {
      const int d = 32 * mt + col;
#pragma unroll
      for (int j = 0; j < (BYTES ? 1 : 2); ++j) {
        u32x4 w = {0, 0, 0, 0};
        if (d < D) w = *reinterpret_cast<const u32x4 *>(vp + (int64_t)d * page + 8 * j);
        vr[mt][j] = w;
      }
    }
    if constexpr (BYTES) vsr = *reinterpret_cast<const u32x4 *>(A.vs + at * A.vsp + head * page + place);
  };

  Rows<T, DP> st;
  st.clear();
  uint32_t *odds = reinterpret_cast<uint32_t *>(shared) + wave * 2 * DP;
  int t = begin + 32 * wave;
  if (t < end) {
    Pages now = pages(t), next = now;
    load_k(t, now);
    load_v(t, now);
    if (t + 128 < end) next = pages(t + 128);
    for (; t < end; t += 128) {
      Pages later = next;
      if (t + 256 < end) later = pages(t + 256);
      f32x16 s[1];
#pragma unroll
      for (int j = 0; j < 16; ++j) s[0][j] = 0.f;
      if constexpr (BYTES) {
        const float by = scale_of(ksr);
#pragma unroll
        for (int c = 0; c < kK; ++c) {
          s[0] = mfma32<T>(widen<T>(u32x2{kr[c][0], kr[c][1]}, by), q[2 * c], s[0]);
          s[0] = mfma32<T>(widen<T>(u32x2{kr[c][2], kr[c][3]}, by), q[2 * c + 1], s[0]);
        }
      } else {
#pragma unroll
        for (int c = 0; c < kK; ++c) s[0] = mfma32<T>(__builtin_bit_cast(Vec8, kr[c]), q[c], s[0]);
      }
      if (t + 128 < end) load_k(t + 128, next);
      const bool edge = t + 31 > all_hi || t < all_lo || !inside(now.at[0]) || !inside(now.at[1]);
      const int first = t + 16 * h;
      if (edge) {
        mask16(s[0], first, lo, hi, !inside(h ? now.at[1] : now.at[0]));
        if constexpr (BYTES) vsr = finite_scales(vsr);
      }
      vec<T, 8> w[2];
      st.weigh(s, A.scale);
      if constexpr (kWeightsScaled<T, BYTES>) times_scales(s[0], vsr);
      st.pack(s, w);
      if (edge) {
        bool any = false;
        u32x4 least = {0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
        if constexpr (BYTES && !kWeightsScaled<T, BYTES>) least = odd_from<T>(vsr);
#pragma unroll
        for (int mt = 0; mt < DP / 32; ++mt) {
          uint32_t up, down;
          if constexpr (BYTES) {
            take_odd_bytes(vr[mt][0], least, up, down);
          } else {
            uint32_t up1, down1;
            take_odd<T>(vr[mt][0], up, down);
            take_odd<T>(vr[mt][1], up1, down1);
            up |= up1 << 8, down |= down1 << 8;
          }
          odds[h * DP + 32 * mt + col] = up | down << 16;
          any = any || up != 0 || down != 0;
        }
        if (__any(any)) {
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
          __builtin_amdgcn_wave_barrier();
          __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
          const uint32_t sees = bits_of(hi + 1 - t) & ~bits_of(lo - t);
#pragma unroll
          for (int mt = 0; mt < DP / 32; ++mt)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int d = 32 * mt + 8 * (j / 4) + 4 * h + j % 4;
              const uint32_t a = odds[d], b = odds[DP + d];
              st.add_odd(mt, j, ((a & 0xffff) | b << 16) & sees, (a >> 16 | (b & 0xffff0000)) & sees);
            }
        }
      }
#pragma unroll
      for (int mt = 0; mt < DP / 32; ++mt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          vec<T, 8> v;
          if constexpr (kWeightsScaled<T, BYTES>)
            v = widen<T>(u32x2{vr[mt][0][2 * j], vr[mt][0][2 * j + 1]}, 1.f);
          else if constexpr (BYTES)
            v = widen<T>(u32x2{vr[mt][0][2 * j], vr[mt][0][2 * j + 1]}, u32x2{vsr[2 * j], vsr[2 * j + 1]});
          else
            v = __builtin_bit_cast(Vec8, vr[mt][j]);
          st.o[mt] = mfma32<T>(v, w[j], st.o[mt]);
        }
      if (t + 128 < end) load_v(t + 128, next);
      now = next, next = later;
    }
  }

  // the waves' states together
  st.finish();
  if (h == 0) ml[0][wave][col] = st.m, ml[1][wave][col] = st.l;
  __syncthreads();
  float top = ml[0][0][col];
#pragma unroll
  for (int w = 1; w < 4; ++w) top = fmaxf(top, ml[0][w][col]);
  const float by = st.m == top ? 1.f : __builtin_amdgcn_exp2f(st.m - top);
  if (mine) {
    float *to = shared + (wave * A.few_rows + col) * kLd + 4 * h;
#pragma unroll
    for (int mt = 0; mt < DP / 32; ++mt)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        vec<float, 4> x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = st.o[mt][4 * a + j] * by;
        *reinterpret_cast<vec<float, 4> *>(to + 32 * mt + 8 * a) = x;
      }
  }
  __syncthreads();
  write_few<T, 4, kFewRows, kLd>(A, shared, ml, sq, head, rows, whole, (int64_t)id * A.few_rows);
}

// ---- many rows of heads over 128: a workgroup takes 128 rows of one sequence and key head, 32 a wave, over tiles of 64
// tokens whose keys and values lie in LDS (two tiles, so that the next one's lands while this one is worked on).  Rings of four
// such tiles, as the kernel below holds them, would be 192 and 256 KiB; rings of 32 tokens have not been tried.  4096 tokens of 32 heads over 8: 0.45 PFLOP/s at dim 192, 0.42 at
// 256, where one wave a SIMD has nothing to do while it waits.
template <typename T, bool BYTES, int DP>
__global__ __launch_bounds__(256, 1) void attend_many_kernel(AttendArgs A) {
  typedef std::conditional_t<BYTES, uint8_t, T> H;
  // rows of LDS are 16 bytes longer than their entries: then 16 lanes that read one piece of 16 rows meet all banks
  constexpr int kKLd = DP + 8, kVLd = kManyStep + 8;
  constexpr int kTile = kManyStep * kKLd + DP * kVLd;
  constexpr int kPer = BYTES ? 16 : 8;                       // entries of a piece of 16 bytes in memory
  constexpr int kAll = kManyStep * DP / kPer, kPieces = (kAll + 255) / 256;  // pieces of a tile's keys, of a thread
  extern __shared__ __align__(16) char shared_bytes[];
  T *lds = reinterpret_cast<T *>(shared_bytes);
  // of a tile that some row sees in part: the tokens whose values are not finite, a bit each, [2][DP][sign][8 bytes], and
  // in odd_at the tile (its first token + 1) that last had any
  uint8_t *odds = reinterpret_cast<uint8_t *>(lds + 2 * kTile);
  typedef volatile __attribute__((address_space(3))) int lds_int;
  lds_int *odd_at = (lds_int *)(odds + 2 * DP * 16);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, h = lane >> 5;
  const uint32_t id = block_id();
  const int head = (int)(id % A.heads);
  const Plan plan = plan_of(A);
  // The last tiles of a chunk see the most and come first, but for workgroups with no unit, which end at once: behind
  // the others they would wait for a compute unit each (2048 rows of 4 in 8 bits over 8192 tokens: 369 us, so 358).
  const uint32_t unit = A.many_units - 1u - id / A.heads;
  int b;
  uint32_t tile;
  Seq sq;
  const int g = A.group, hq = A.heads * g, D = A.dim;
  if (!find_unit(A.s, unit, [&](const Seq &s) { return many_units(A, s, plan.per); }, b, tile, sq)) return;
  const uint32_t parts = many_parts(A, sq, plan.per);
  const int part = (int)(tile % parts);
  tile /= parts;
  const int len = sq.pos + sq.n, rows = sq.n * g;
  const int r0 = (int)tile * kManyRows, r1 = min(r0 + kManyRows, rows);
  const int p0 = sq.pos + r0 / g, p1 = sq.pos + (r1 - 1) / g;
  const Span sp = span_of(A, p0, p1, len, plan.per);
  if (part >= max(sp.parts, 1)) return;
  const int r = r0 + wave * 32 + col;
  const bool mine = r < rows;
  const int i = r / g, p = sq.pos + i;
  const int hi = mine ? (A.causal ? p : len - 1) : -1, lo = A.window > 0 ? p - A.window + 1 : 0;
  const int all_hi = A.causal ? p0 : len - 1, all_lo = A.window > 0 ? p1 - A.window + 1 : 0;

  vec<T, 8> q[DP / 16];
  const T *qp = reinterpret_cast<const T *>(A.q) + (int64_t)(sq.row + i) * A.qt + (int64_t)(head * g + r % g) * A.qh;
#pragma unroll
  for (int c = 0; c < DP / 16; ++c) q[c] = load_q<T>(qp, 16 * c + 8 * h, D, mine, A.wide != 0);

  const int page = 1 << A.s.page_shift, inner = page - 1;
  u32x4 kr[kPieces], vr[kPieces], vsr = {0, 0, 0, 0};
  uint32_t ksr[BYTES ? kPieces : 1];
  typedef Pages4 Pages;
  const TableRow table = table_row(A.s, b);
  auto pages = [&](int t) { return Pages{table.entry(t), table.entry(t + 16), table.entry(t + 32), table.entry(t + 48)}; };
  auto inside = [&](uint32_t page) { return page < A.s.n_pages; };
  auto pick = [&](const Pages &pg, int j) {
    const uint32_t e = one_of(pg, j);
    return inside(e) ? e : 0u;
  };
  constexpr int kKRow = DP / kPer, kVRow = kManyStep / kPer;  // pieces of a row
  auto load = [&](int t, const Pages &pg) {
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
      const int n = e * 256 + tid;
      {
        const int row = n / kKRow, d = n % kKRow * kPer;
        const int64_t at = pick(pg, row >> 4 & 3);
        const int place = (t + row) & inner;
        if (n < kAll && d < D) kr[e] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const H *>(A.k) + at * A.kp + (int64_t)(head * page + place) * D + d);
        if constexpr (BYTES) ksr[e] = A.ks[at * A.ksp + head * page + place];  // n >= kAll: of another row, not used
      }
      {
        const int d = n / kVRow, tok = n % kVRow * kPer;
        const int64_t at = pick(pg, tok >> 4);
        const int place = (t + tok) & inner;
        if (n < kAll && d < D) vr[e] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const H *>(A.v) + at * A.vp + (int64_t)(head * D + d) * page + place);
        if constexpr (BYTES)
          if (e == 0) vsr = *reinterpret_cast<const u32x4 *>(A.vs + at * A.vsp + head * page + place);
      }
    }
  };
  // whether some row does not see all of the tokens from t on
  auto partly = [&](int t) { return t + kManyStep - 1 > all_hi || t < all_lo; };
  auto store = [&](int buf, int t) {
    T *k = lds + buf * kTile, *v = k + kManyStep * kKLd;
    const bool edge = partly(t);
    u32x4 least = {0, 0, 0, 0};
    if constexpr (BYTES)
      if (edge) vsr = finite_scales(vsr), least = odd_from<T>(vsr);
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
      const int n = e * 256 + tid;
      {
        const int row = n / kKRow, d = n % kKRow * kPer;
        T *to = k + row * kKLd + d;
        if (n < kAll && d < D) {
          if constexpr (BYTES) {
            const float by = scale_of(ksr[e]);
            *reinterpret_cast<vec<T, 8> *>(to) = widen<T>(u32x2{kr[e][0], kr[e][1]}, by);
            *reinterpret_cast<vec<T, 8> *>(to + 8) = widen<T>(u32x2{kr[e][2], kr[e][3]}, by);
          } else {
            *reinterpret_cast<u32x4 *>(to) = kr[e];
          }
        }
      }
      {
        const int d = n / kVRow, tok = n % kVRow * kPer;
        T *to = v + d * kVLd + tok;
        if (n < kAll && d < D) {
          if (edge) {
            uint32_t up, down;
            if constexpr (BYTES)
              take_odd_bytes(vr[e], least, up, down);
            else
              take_odd<T>(vr[e], up, down);
            uint8_t *at = odds + (buf * DP + d) * 16 + tok / 8;
            at[0] = (uint8_t)up, at[8] = (uint8_t)down;
            if constexpr (BYTES) at[1] = (uint8_t)(up >> 8), at[9] = (uint8_t)(down >> 8);
            if (up | down) odd_at[buf] = t + 1;
          }
          if constexpr (BYTES) {
            *reinterpret_cast<vec<T, 8> *>(to) = widen<T>(u32x2{vr[e][0], vr[e][1]}, u32x2{vsr[0], vsr[1]});
            *reinterpret_cast<vec<T, 8> *>(to + 8) = widen<T>(u32x2{vr[e][2], vr[e][3]}, u32x2{vsr[2], vsr[3]});
          } else {
            *reinterpret_cast<u32x4 *>(to) = vr[e];
          }
        }
      }
    }
  };

  Rows<T, DP> st;
  st.clear();
  int t = sp.begin + part * plan.per;
  const int end = min(sp.end, t + plan.per);
  if (t < end) {
    if (tid < 2) odd_at[tid] = 0;
    if (D < DP)  // what no entry is written to is zero
      for (int e = tid; e < 2 * kTile / 8; e += 256) reinterpret_cast<u32x4 *>(lds)[e] = u32x4{0, 0, 0, 0};
    __syncthreads();
    Pages now = pages(t), next = now;
    load(t, now);
    if (t + kManyStep < end) next = pages(t + kManyStep);
    store(0, t);
    int buf = 0;
    for (; t < end; t += kManyStep) {
      const bool more = t + kManyStep < end;
      Pages later = next;
      if (t + 2 * kManyStep < end) later = pages(t + 2 * kManyStep);
      if (more) load(t + kManyStep, next);
      __syncthreads();
      const T *k = lds + buf * kTile, *v = k + kManyStep * kKLd;
      f32x16 s[2];
      const int ki = 16 * (col >> 2 & 1) + 4 * (col >> 3) + (col & 3);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 16; ++j) s[u][j] = 0.f;
#pragma unroll
      for (int c = 0; c < DP / 16; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          s[u] = mfma32<T>(*reinterpret_cast<const vec<T, 8> *>(k + (32 * u + ki) * kKLd + 16 * c + 8 * h), q[c], s[u]);
      const bool edge = partly(t) || !(inside(now.a) && inside(now.b) && inside(now.c) && inside(now.d));
      const int first = t + 16 * h;
      if (edge) {
        mask16(s[0], first, lo, hi, !inside(h ? now.b : now.a));
        mask16(s[1], first + 32, lo, hi, !inside(h ? now.d : now.c));
      }
      vec<T, 8> w[4];
      st.weigh(s, A.scale);
      st.pack(s, w);
      if (partly(t) && odd_at[buf] == t + 1) {
        const uint32_t sees[2] = {bits_of(hi + 1 - t) & ~bits_of(lo - t), bits_of(hi + 1 - t - 32) & ~bits_of(lo - t - 32)};
#pragma unroll
        for (int mt = 0; mt < DP / 32; ++mt)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(odds + (buf * DP + 32 * mt + 8 * (j / 4) + 4 * h + j % 4) * 16);
            st.add_odd(mt, j, (x[0] & sees[0]) | (x[1] & sees[1]), (x[2] & sees[0]) | (x[3] & sees[1]));
          }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int mt = 0; mt < DP / 32; ++mt)
          st.o[mt] = mfma32<T>(*reinterpret_cast<const vec<T, 8> *>(v + (32 * mt + col) * kVLd + 32 * (j / 2) + 8 * (j % 2) + 16 * h),
                               w[j], st.o[mt]);
      buf ^= 1;
      if (more) store(buf, t + kManyStep);
      now = next, next = later;
    }
  }
  st.finish();
  if (!mine) return;
  const int64_t row = (int64_t)(sq.row + i) * hq + head * g + r % g;
  const bool whole = sp.parts <= 1;
  if (whole) {
    const float inv = st.l == 0.f ? 0.f : 1.f / st.l;
    T *to = reinterpret_cast<T *>(A.out) + row * D + 4 * h;
#pragma unroll
    for (int mt = 0; mt < DP / 32; ++mt)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const float y[4] = {st.o[mt][4 * a] * inv, st.o[mt][4 * a + 1] * inv, st.o[mt][4 * a + 2] * inv, st.o[mt][4 * a + 3] * inv};
        if (32 * mt + 8 * a + 4 * h < D) store_vec<T, 4>(to + 32 * mt + 8 * a, y);
      }
    if (h == 0 && A.lse) A.lse[row] = (st.m + __builtin_amdgcn_logf(st.l)) * kLn2F;
  } else {
    const int64_t at = ((int64_t)unit * A.heads + head) * A.many_rows + r - r0;
    float *to = A.many_o + at * D + 4 * h;
#pragma unroll
    for (int mt = 0; mt < DP / 32; ++mt)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const float y[4] = {st.o[mt][4 * a], st.o[mt][4 * a + 1], st.o[mt][4 * a + 2], st.o[mt][4 * a + 3]};
        if (32 * mt + 8 * a + 4 * h < D) store_vec<float, 4>(to + 32 * mt + 8 * a, y);
      }
    if (h == 0) A.many_ml[2 * at] = st.m, A.many_ml[2 * at + 1] = st.l;
  }
}

// ---- many rows of heads up to 128: a workgroup of eight waves takes 256 rows, 32 a wave, two waves a SIMD.  Tiles of 64
// tokens are copied straight into rings in LDS, two tiles ahead of their use (8 bits: as they are, and widened from
// there into rings of T).  The work on a half tile i is three stages of three halves at a time, which do not wait for
// each other: scores of i + 1, weights of i, the product of i - 1 with its values; so the matrix unit works while the vector unit
// takes exponentials.  One workgroup fills a compute unit: 130 KB of LDS (8 bits: 152) and all registers.

// Copies of 16 bytes a lane from memory to LDS: lane l's land at `to` + 16 l, `to` the same for all lanes.  Instructions of
// their own, as the compiler would wait for every copy before each read of LDS; nothing else in the kernel uses
// m0.  A scalar base is read five wait states after the instruction that wrote it at the earliest.
__device__ __forceinline__ void copy_piece(const void *from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}
__device__ __forceinline__ void copy_piece(const void *base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
}
template <typename H>
__device__ __forceinline__ const H *uniform_pointer(const H *p) {  // one for all lanes, in scalar registers
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const H *>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
                                     (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}
// Waits until at most N of this wave's copies are on their way.
template <int N>
__device__ __forceinline__ void copies_left() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// c += a b with the sums in accumulation registers.  Written as an instruction because the allocator, left the choice,
// moves them between both halves of the register file around every use of a score.  It does not know the
// instruction's latency: sums are used again four products later, and read or written by others only after settle_products
// (at most 18 cycles) and before before_products.
template <typename T>
__device__ __forceinline__ void add_product(f32x16 &c, vec<T, 8> a, vec<T, 8> b) {
  if constexpr (std::is_same<T, bf16_t>::value)
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  else
    asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
// Scores: s = a q, or with the products before them.  The vector unit reads them after one more product and apart(), 8 cycles
// each (11 are asked for).
template <typename T>
__device__ __forceinline__ void score_product(f32x16 &s, vec<T, 8> a, vec<T, 8> q, bool first) {
  if constexpr (std::is_same<T, bf16_t>::value) {
    if (first)
      asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "a"(q));
    else
      asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "a"(q));
  } else {
    if (first)
      asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "a"(q));
    else
      asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "a"(q));
  }
}
template <int N>
__device__ __forceinline__ void settle_products(f32x16 (&o)[N]) {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+a"(o[i]));
}
// Between a product and one that adds to its result, or (behind one more product) what reads it.
__device__ __forceinline__ void apart() { asm volatile("s_nop 7" ::: "memory"); }
__device__ __forceinline__ void settle_scores(f32x16 &s) { asm volatile("s_nop 15\n\ts_nop 15" : "+v"(s)::"memory"); }
template <int N>
__device__ __forceinline__ void before_products(f32x16 (&o)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+a"(o[i]));
  asm volatile("s_nop 7" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Sums times a factor where they are: a use by an ordinary instruction would move all of them at every branch's end.
__device__ __forceinline__ void times_sums(f32x16 &o, float by) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float x = o[i], y;
    asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %1, %2\n\tv_accvgpr_write_b32 %0, %1"
                 : "+a"(x), "=&v"(y) : "v"(by));
    o[i] = x;
  }
}

// Place of piece c (8 entries) of a row in LDS: 16 lanes that read one piece of rows 0-3, 16-19, 4-7, 20-23 (or these + 8) of
// keys, or of 16 rows of values in order, meet all banks.
template <int DP>
__device__ __forceinline__ int key_place(int row, int c) {
  if constexpr (DP == 128) return c ^ ((row & 7) | (row >> 4 & 1) << 3);
  if constexpr (DP == 64) return c ^ ((row >> 1 & 3) | (row >> 4 & 1) << 2);
  const int p = c + ((row >> 2 & 1) | (row >> 4 & 1) << 1);
  return p >= DP / 8 ? p - DP / 8 : p;
}
template <int DP>
__device__ __forceinline__ int key_piece(int row, int place) {  // which piece lies there
  if constexpr (DP != 96) return key_place<DP>(row, place);
  const int c = place - ((row >> 2 & 1) | (row >> 4 & 1) << 1);
  return c < 0 ? c + DP / 8 : c;
}
__device__ __forceinline__ int value_place(int d, int c) { return c ^ (d >> 1 & 7); }

// LDS of the kernel: rings of kRing tiles of keys and of values; 8 bits: three tiles of either as they are in memory and their
// scales; the bits of take_odd.
template <typename T, bool BYTES, int DP>
struct Wide {
  static constexpr int kWaves = kWideRows / 32;                       // of 32 rows
  static constexpr int kRing = BYTES ? 3 : 4, kLead = BYTES ? 4 : 3;  // tiles; how far ahead of its use a tile of keys is copied
  static constexpr int kTile = 64 * DP;                               // entries
  static constexpr int kRaw = BYTES ? (DP + 63) / 64 : 0;             // copies of a wave for a tile as it is, of keys and of values
  static constexpr int kCopies = BYTES ? kRaw + 1 : DP / 32;          // of a wave for a tile of keys or of values, and scales
  static constexpr uint32_t kKeys = 0, kValues = kRing * kTile * 2, kRawKeys = 2 * kValues, kRawValues = kRawKeys + 3 * kRaw * 4096,
                            kScales = kRawValues + 3 * kRaw * 4096, kOdds = kScales + (BYTES ? 3 * 2048 : 0),
                            kOddAt = kOdds + DP * 16, kBytes = kOddAt + 16;
};

template <typename T, bool BYTES, int DP>
__global__ __launch_bounds__(64 * (Wide<T, BYTES, DP>::kWaves), (Wide<T, BYTES, DP>::kWaves) / 4) void attend_wide_kernel(AttendArgs A) {
  typedef std::conditional_t<BYTES, uint8_t, T> H;
  typedef vec<T, 8> Vec8;
  typedef Wide<T, BYTES, DP> W;
  constexpr int kMt = DP / 32, kC = DP / 16, kTile = W::kTile, kLead = W::kLead, kThreads = 64 * W::kWaves;
  extern __shared__ __align__(1024) char shared_bytes[];
  const T *keys = reinterpret_cast<const T *>(shared_bytes + W::kKeys);
  T *values = reinterpret_cast<T *>(shared_bytes + W::kValues);
  uint8_t *odds = reinterpret_cast<uint8_t *>(shared_bytes + W::kOdds);  // as in the kernel above, of one tile
  volatile int *odd_at = reinterpret_cast<volatile int *>(shared_bytes + W::kOddAt);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, h = lane >> 5;
  const uint32_t id = block_id();
  const int head = (int)(id % A.heads);
  const Plan plan = plan_of(A);
  // The last tiles of a chunk see the most and come first, but for workgroups with no unit, which end at once: behind
  // the others they would wait for a compute unit each (2048 rows of 4 in 8 bits over 8192 tokens: 369 us, so 358).
  const uint32_t unit = A.many_units - 1u - id / A.heads;
  int b;
  uint32_t tile;
  Seq sq;
  const int g = A.group, hq = A.heads * g, D = A.dim;
  if (!find_unit(A.s, unit, [&](const Seq &s) { return many_units(A, s, plan.per); }, b, tile, sq)) return;
  const uint32_t parts = many_parts(A, sq, plan.per);
  const int part = (int)(tile % parts);
  tile /= parts;
  const int len = sq.pos + sq.n, rows = sq.n * g;
  const int r0 = (int)tile * kWideRows, r1 = min(r0 + kWideRows, rows);
  const int p0 = sq.pos + r0 / g, p1 = sq.pos + (r1 - 1) / g;
  const Span sp = span_of(A, p0, p1, len, plan.per);
  if (part >= max(sp.parts, 1)) return;
  const int begin = sp.begin + part * plan.per, end = min(sp.end, begin + plan.per);
  const int n = end > begin ? (end - begin + 63) / 64 : 0;  // tiles
  const int all_hi = A.causal ? p0 : len - 1, all_lo = A.window > 0 ? p1 - A.window + 1 : 0;
  const bool active = r0 + wave * 32 < rows;  // of the wave

  Vec8 q[kC];
  const int r = r0 + wave * 32 + col, i = r / g;
  const bool mine = r < rows;
  const int hi = mine ? (A.causal ? sq.pos + i : len - 1) : -1, lo = A.window > 0 ? sq.pos + i - A.window + 1 : 0;
  const T *qp = reinterpret_cast<const T *>(A.q) + (int64_t)(sq.row + i) * A.qt + (int64_t)(head * g + r % g) * A.qh;
#pragma unroll
  for (int c = 0; c < kC; ++c) q[c] = load_q<T>(qp, 16 * c + 8 * h, D, mine, A.wide != 0);

  // ---- copies.  Four waves copy keys and four values.  Keys: the first copies tokens 0 .. 15 of the tile, the next 16 .. 31, ..,
  // which lie in one page; values: a lane's 16 bytes of every row that it copies are of the same tokens.  In pages of 64
  // and more a tile lies in one, and all bases are scalars.
  const int quarter = wave & 3;
  const bool for_keys = wave < 4;
  const int page = 1 << A.s.page_shift, inner = page - 1;
  const bool single = page >= 64;
  typedef Pages4 Pages;
  const TableRow table = table_row(A.s, b);
  auto pages = [&](int j) {
    const int t = begin + 64 * j;
    const uint32_t e = table.entry(t);
    if (single) return Pages{e, e, e, e};
    return Pages{e, table.entry(t + 16), table.entry(t + 32), table.entry(t + 48)};
  };
  auto inside = [&](uint32_t e) { return e < A.s.n_pages; };
  auto outside4 = [&](const Pages &pg) {
    if (single) return inside(pg.a) ? 0u : 15u;
    return (inside(pg.a) ? 0u : 1u) | (inside(pg.b) ? 0u : 2u) | (inside(pg.c) ? 0u : 4u) | (inside(pg.d) ? 0u : 8u);
  };
  auto pick = [&](const Pages &pg, int j) -> int64_t {
    const uint32_t e = single ? pg.a : one_of(pg, j);
    return inside(e) ? e : 0u;
  };
  auto slot = [&](int j) { return W::kRing == 4 ? j & 3 : j % 3; };
  const H *kbase = reinterpret_cast<const H *>(A.k) + (int64_t)head * page * D;
  const H *vbase = reinterpret_cast<const H *>(A.v) + (int64_t)head * page * D;
  constexpr int kRowPieces = DP / (16 / (int)sizeof(H));  // of 16 bytes, of a row of keys in LDS
  constexpr int kPieces = BYTES ? W::kRaw : DP / 32;      // copies of a wave for a tile
  constexpr bool kRagged = BYTES && DP == 96;             // a wave's keys do not fill its copies
  uint32_t off[kPieces];  // bytes from the wave's first token's key (~0: nothing), or from the tokens in the first row of values
  const int value_row = BYTES ? quarter * 16 + lane / 4 : quarter * 8 + lane / 8;
  auto value_tok = [&](int l) { return BYTES ? l % 4 * 16 : 8 * value_place(quarter * 8 + l / 8, l % 8); };
#pragma unroll
  for (int e = 0; e < kPieces; ++e) {
    const int m = e * 64 + lane, row = m / kRowPieces;
    const int d = BYTES ? m % kRowPieces * 16 : 8 * key_piece<DP>(16 * quarter + row, m % kRowPieces);
    // rows of values behind the last entry are copies of it: what comes of them is not stored
    off[e] = for_keys ? (row < 16 && d < D ? (uint32_t)((row * D + d) * sizeof(H)) : ~0u)
                      : (uint32_t)(((int64_t)min(value_row + e * (BYTES ? 64 : 32), D - 1) * page + value_tok(lane)) * sizeof(H));
  }
  auto copy_keys = [&](int j, const Pages &pg) {
    const int t = begin + 64 * j + 16 * quarter;
    const H *base = uniform_pointer(kbase + pick(pg, quarter) * A.kp + (t & inner) * D);
    const uint32_t to = BYTES ? W::kRawKeys + (j % 3) * W::kRaw * 4096 + quarter * W::kRaw * 1024 : W::kKeys + slot(j) * kTile * 2 + quarter * 32 * DP;
    if (D == DP && !kRagged) {
#pragma unroll
      for (int e = 0; e < kPieces; ++e) copy_piece(base, off[e], to + e * 1024);
    } else {
#pragma unroll
      for (int e = 0; e < kPieces; ++e)
        if (off[e] != ~0u) copy_piece(base, off[e], to + e * 1024);
    }
  };
  auto copy_values = [&](int j, const Pages &pg) {
    const int t = begin + 64 * j;
    const uint32_t to = BYTES ? W::kRawValues + (j % 3) * W::kRaw * 4096 + quarter * 1024 : W::kValues + slot(j) * kTile * 2 + quarter * 1024;
    if (single) {
      const H *base = uniform_pointer(vbase + pick(pg, 0) * A.vp + (t & inner));
#pragma unroll
      for (int e = 0; e < kPieces; ++e) copy_piece(base, off[e], to + e * 4096);
    } else {
      int l = lane;
      asm volatile("" : "+v"(l));  // computed here: a register kept for it is one too many, and its reload would wait for all copies
      const int at = value_tok(l) & ~15;  // off counts from the tile's first token
      const char *from = reinterpret_cast<const char *>(vbase + pick(pg, at >> 4) * A.vp + (((t + at) & inner) - at));
#pragma unroll
      for (int e = 0; e < kPieces; ++e) copy_piece(from + off[e], to + e * 4096);
    }
  };
  // 8 bits: scales of the keys of a tile and of the values of the one before it, 64 bytes of either (and again every 64, by every
  // wave of four)
  auto copy_scales = [&](int j, const Pages &pk, const Pages &pv) {
    const Pages pg = for_keys ? pk : pv;
    const uint8_t *base = (for_keys ? A.ks : A.vs) + head * page;
    const int64_t step = for_keys ? A.ksp : A.vsp;
    const int t = begin + 64 * (for_keys ? j : j - 1);
    const uint32_t to = W::kScales + (j % 3) * 2048 + (for_keys ? 0 : 1024);
    int l = lane;
    asm volatile("" : "+v"(l));  // as above
    const int gr = l & 3;
    if (single)
      copy_piece(uniform_pointer(base + pick(pg, 0) * step + (t & inner)), 16 * gr, to);
    else
      copy_piece(base + pick(pg, gr) * step + ((t + 16 * gr) & inner), to);
  };
  // 8 bits: a copied tile to the rings
  auto widen_keys = [&](int j) {
    if constexpr (BYTES) {
#pragma unroll
      for (int m = tid; m < W::kRaw * 256; m += kThreads) {
        const int w = m / (W::kRaw * 64), i = m % (W::kRaw * 64), row = 16 * w + i / kRowPieces, c = i % kRowPieces * 2;
        if (i >= 16 * kRowPieces || 8 * c >= D) continue;
        const u32x4 x = *reinterpret_cast<const u32x4 *>(shared_bytes + W::kRawKeys + (j % 3) * W::kRaw * 4096 + m * 16);
        const float by = scale_of((uint8_t)shared_bytes[W::kScales + (j % 3) * 2048 + row]);
        T *to = const_cast<T *>(keys) + slot(j) * kTile + row * DP;
        *reinterpret_cast<Vec8 *>(to + 8 * key_place<DP>(row, c)) = widen<T>(u32x2{x[0], x[1]}, by);
        *reinterpret_cast<Vec8 *>(to + 8 * key_place<DP>(row, c + 1)) = widen<T>(u32x2{x[2], x[3]}, by);
      }
    }
  };
  auto widen_values = [&](int j) {
    if constexpr (BYTES) {
      const u32x4 by = *reinterpret_cast<const u32x4 *>(shared_bytes + W::kScales + ((j + 1) % 3) * 2048 + 1024 + tid % 4 * 16);
#pragma unroll
      for (int m = tid; m < W::kRaw * 256; m += kThreads) {
        const int d = m / 4, c = m % 4 * 2;
        if (d >= DP) continue;
        const u32x4 x = *reinterpret_cast<const u32x4 *>(shared_bytes + W::kRawValues + (j % 3) * W::kRaw * 4096 + m * 16);
        T *to = values + slot(j) * kTile + d * 64;
        *reinterpret_cast<Vec8 *>(to + 8 * value_place(d, c)) = widen<T>(u32x2{x[0], x[1]}, u32x2{by[0], by[1]});
        *reinterpret_cast<Vec8 *>(to + 8 * value_place(d, c + 1)) = widen<T>(u32x2{x[2], x[3]}, u32x2{by[2], by[3]});
      }
    }
  };

  Rows<T, DP> st;
  st.clear();
  const int ki = 16 * (col >> 2 & 1) + 4 * (col >> 3) + (col & 3);
  int koff[kC], voff[4];
#pragma unroll
  for (int c = 0; c < kC; ++c) koff[c] = ki * DP + 8 * key_place<DP>(ki, 2 * c + h);
#pragma unroll
  for (int c = 0; c < 4; ++c) voff[c] = col * 64 + 8 * value_place(col, 4 * (c / 2) + 2 * h + c % 2);
  auto key_piece_of = [&](const T *k, int u, int c) { return *reinterpret_cast<const Vec8 *>(k + 32 * u * DP + koff[c]); };
  auto value_piece_of = [&](const T *v, int u, int m) {  // of the half's kC products' first operands
    return *reinterpret_cast<const Vec8 *>(v + m / 2 * 32 * 64 + voff[2 * u + m % 2]);
  };
  // One half's stage: weights of s to p, scores of half ku of tile k to next, and half vu of the values v times pp.
  // Every product is followed by its share of the vector instructions, and nothing is moved across: of an entry the
  // argument of the exponential, the exponential, and what uses it behind three products in a row.
  constexpr int kAhead = 2, kHeld = kAhead + 1;  // operands on their way from LDS
  Vec8 first_k[kAhead], first_v[kAhead];         // of the next stage
  auto first_pieces = [&](const T *k, int ku, const T *v, int vu) {
#pragma unroll
    for (int c = 0; c < kAhead; ++c) first_k[c] = key_piece_of(k, ku, c), first_v[c] = value_piece_of(v, vu, c);
  };
  auto stage = [&](const f32x16 &s, Vec8 (&p)[2], f32x16 &next, const T *k, int ku, const T *v, int vu, const Vec8 (&pp)[2],
                   const T *then_k, int then_ku, const T *then_v, int then_vu) {
    constexpr int kSlots = 2 * kC, kFirst = 4, kOver = kSlots - kFirst - 2;  // products; the first kFirst share the maxima
    Vec8 ka[kHeld], va[kHeld];
#pragma unroll
    for (int c = 0; c < kAhead; ++c) ka[c] = first_k[c], va[c] = first_v[c];
    float top[4], to, by, from, sum = 0.f, w[16];
    bool grows = false;
    auto vector_share = [&](int slot) {
      if (slot == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) top[i] = max3(s[4 * i], s[4 * i + 1], s[4 * i + 2]);
      } else if (slot == 1) {
        top[0] = max3(top[0], s[3], s[7]), top[1] = max3(top[1], s[11], s[15]);
        top[0] = max3(top[0], top[2], top[3]);
      } else if (slot == 2) {
        const float t = max3(top[0], top[1], partner(max3(top[0], top[1], top[1]))) * A.scale;
        const bool more = t > st.m + kGrowth<T>;
        grows = grows || more;
        to = more ? t - kBelow<T> : st.m;
        from = to == -__builtin_inff() ? 0.f : to;
      } else if (slot == 3) {
        by = to == st.m ? 1.f : __builtin_amdgcn_exp2f(st.m - to);
        st.m = to;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int at = kFirst + e * kOver / 16;
        if (slot == at + 2) {
          sum += w[e];
          if (e % 2) p[e / 8][e % 8 - 1] = (T)w[e - 1], p[e / 8][e % 8] = (T)w[e];
          if (e % 8 == 7) asm volatile("" : "+v"(p[e / 8]), "+v"(sum));  // here, not behind the branch at the stage's end
        }
        if (slot == at + 1) w[e] = __builtin_amdgcn_exp2f(w[e]);
        if (slot == at) w[e] = fmaf(s[e], A.scale, -from);
      }
    };
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      if (c + kAhead < kC) {
        ka[(c + kAhead) % kHeld] = key_piece_of(k, ku, c + kAhead);
        va[(c + kAhead) % kHeld] = value_piece_of(v, vu, c + kAhead);
      } else {
        first_k[c + kAhead - kC] = key_piece_of(then_k, then_ku, c + kAhead - kC);
        first_v[c + kAhead - kC] = value_piece_of(then_v, then_vu, c + kAhead - kC);
      }
      score_product<T>(next, ka[c % kHeld], q[c], c == 0);
      vector_share(2 * c);
      __builtin_amdgcn_sched_barrier(0);
      add_product<T>(st.o[c / 2], va[c % kHeld], pp[c % 2]);
      vector_share(2 * c + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    st.l = st.l * by + sum;
    apart();  // behind the last score
    if (__any(grows)) {
      settle_products(st.o);
#pragma unroll
      for (int mt = 0; mt < kMt; ++mt) times_sums(st.o[mt], by);
      before_products(st.o);
    }
  };

  before_products(st.o);
#pragma unroll
  for (int c = 0; c < kC; ++c) asm volatile("" : "+a"(q[c]));  // queries stay in accumulation registers too
  if (n > 0) {
    // zeros where no key's entry is written to, and in the tile of values that stands before the first
    constexpr uint32_t kBefore = W::kValues + (W::kRing - 1) * kTile * 2;
    for (uint32_t e = tid * 16; e < (D < DP ? W::kValues : 0u); e += 16 * kThreads) *reinterpret_cast<u32x4 *>(shared_bytes + e) = u32x4{0, 0, 0, 0};
    for (uint32_t e = tid * 16; e < kTile * 2; e += 16 * kThreads) *reinterpret_cast<u32x4 *>(shared_bytes + kBefore + e) = u32x4{0, 0, 0, 0};
    if (tid == 0) *odd_at = 0;
    __syncthreads();
    uint32_t bad = 0;  // bits of 16 tokens each without a page, of this tile and those after it
    Pages pk = pages(0), pv = pk, pn = 1 < n ? pages(1) : pk;  // of the tiles of keys and of values copied next, and after
    auto copy_next = [&](int j) {  // keys of tile j and values of j - 1, whose pages are pk and pv
      if (j < n) {
        if (for_keys) copy_keys(j, pk);
        bad |= outside4(pk) << (4 * kLead);
      }
      if constexpr (BYTES) {
        if (j - 1 < n) copy_scales(j, pk, pv);
      }
      if (!for_keys && j > 0 && j - 1 < n) copy_values(j - 1, pv);
    };
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      copy_next(j);
      pv = pk, pk = pn;
      if (j + 2 < n) pn = pages(j + 2);
      bad >>= 4;
    }
    copies_left<0>();
    __syncthreads();
    if constexpr (BYTES) {  // tiles 0 and 1 of keys and 0 of values; then the next into their places
      widen_keys(0);
      if (n > 1) widen_keys(1);
      widen_values(0);
      __syncthreads();
      copy_next(3);
      pv = pk, pk = pn;
      if (5 < n) pn = pages(5);
      bad >>= 4;
    }
    f32x16 s0, s1;
    Vec8 pa[2], pb[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) pb[j][i] = (T)0.f;
    if (active)
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        score_product<T>(s0, key_piece_of(keys, 0, c), q[c], c == 0);
        apart();
      }
    settle_scores(s0);
    first_pieces(keys, 1, values + (W::kRing - 1) * kTile, 1);
    for (int j = 0; j < n; ++j) {
      const int t = begin + 64 * j;
      // of the copies only those of the iteration before may be on their way
      if (j + kLead - 1 < n)
        copies_left<W::kCopies>();
      else
        copies_left<0>();
      __syncthreads();  // and what is overwritten now has been read
      copy_next(j + kLead);
      const T *k1 = keys + slot(j + 1) * kTile, *k0 = keys + slot(j) * kTile;
      T *v0 = values + slot(j) * kTile;
      const T *v1 = values + slot(j + W::kRing - 1) * kTile;  // tile j - 1
      const bool partly = t + 63 > all_hi || t < all_lo;  // some row does not see all tokens
      if (partly) {
        for (int m = tid; m < D * 8; m += kThreads) {
          const int d = m / 8, c = value_place(d, m % 8);
          u32x4 w = reinterpret_cast<const u32x4 *>(v0)[m];
          uint32_t up, down;
          take_odd<T>(w, up, down);
          odds[d * 16 + c] = (uint8_t)up, odds[d * 16 + 8 + c] = (uint8_t)down;
          if (up | down) {
            reinterpret_cast<u32x4 *>(v0)[m] = w;
            *odd_at = t + 1;
          }
        }
        __syncthreads();
        if (*odd_at == t + 1) {
          int d0 = 4 * h;
          asm volatile("" : "+v"(d0));  // places and bounds of all entries would be kept through the loop
          const uint32_t sees[2] = {bits_of(hi + 1 - t) & ~bits_of(lo - t), bits_of(hi + 1 - t - 32) & ~bits_of(lo - t - 32)};
#pragma unroll
          for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int d = d0 + 32 * mt + 8 * (i / 4) + i % 4;
              const u32x4 w = *reinterpret_cast<const u32x4 *>(odds + d * 16);
              st.add_odd(mt, i, d < D && ((w[0] & sees[0]) | (w[1] & sees[1])), d < D && ((w[2] & sees[0]) | (w[3] & sees[1])));
              __builtin_amdgcn_sched_barrier(0);  // one after the other: seldom run, and not worth registers
            }
        }
      }
      if (active) {
        const bool edge = partly || (bad & 15);
        const int first = t + 16 * h;
        if (edge) mask16(s0, first, lo, hi, bad >> h & 1);
        stage(s0, pa, s1, k0, 1, v1, 1, pb, k1, 0, v0, 0);
        if (edge) mask16(s1, first + 32, lo, hi, bad >> (2 + h) & 1);
        stage(s1, pb, s0, k1, 0, v0, 0, pa, k1, 1, v0, 1);
      }
      if constexpr (BYTES) {
        if (j + 2 < n) widen_keys(j + 2);
        if (j + 1 < n) widen_values(j + 1);
      }
      pv = pk, pk = pn;
      if (j + kLead + 2 < n) pn = pages(j + kLead + 2);  // looked at behind the barrier after next
      bad >>= 4;
    }
    if (active) {
      const T *v = values + slot(n - 1) * kTile;
#pragma unroll
      for (int m = 0; m < kC; ++m) {
        add_product<T>(st.o[m / 2], value_piece_of(v, 1, m), pb[m % 2]);
        apart();
      }
    }
  }
  if (!active) return;
  settle_products(st.o);
  st.finish();
  if (r >= rows) return;
  const int64_t row = (int64_t)(sq.row + i) * hq + head * g + r % g;
  if (sp.parts <= 1) {
    const float inv = st.l == 0.f ? 0.f : 1.f / st.l;
    T *to = reinterpret_cast<T *>(A.out) + row * D + 4 * h;
#pragma unroll
    for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const float y[4] = {st.o[mt][4 * a] * inv, st.o[mt][4 * a + 1] * inv, st.o[mt][4 * a + 2] * inv, st.o[mt][4 * a + 3] * inv};
        if (32 * mt + 8 * a + 4 * h < D) store_vec<T, 4>(to + 32 * mt + 8 * a, y);
      }
    if (h == 0 && A.lse) A.lse[row] = (st.m + __builtin_amdgcn_logf(st.l)) * kLn2F;
  } else {
    const int64_t at = ((int64_t)unit * A.heads + head) * A.many_rows + r - r0;
    float *to = A.many_o + at * D + 4 * h;
#pragma unroll
    for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const float y[4] = {st.o[mt][4 * a], st.o[mt][4 * a + 1], st.o[mt][4 * a + 2], st.o[mt][4 * a + 3]};
        if (32 * mt + 8 * a + 4 * h < D) store_vec<float, 4>(to + 32 * mt + 8 * a, y);
      }
    if (h == 0) A.many_ml[2 * at] = st.m, A.many_ml[2 * at + 1] = st.l;
  }
}

// ---- the parts of a row together, in their order.  The first workgroups take sequences with few rows: 32 times four entries,
// and of each eight threads every eighth part, whose sums meet in LDS.  The others take the tokens of the other
// sequences, whose parts are few: a thread four entries at a time.
constexpr int kJoinQuads = kJoinThreads / 8;

// All threads of a workgroup call it; `there`: this thread's entries are some row's.
template <typename T, int SPLIT>
__device__ __forceinline__ void join_row(const AttendArgs &A, const float *po, const float *pm, int64_t at, int64_t step, int parts,
                                         int64_t row, int d, bool there) {
  constexpr int kQuads = kJoinThreads / SPLIT;
  const int k = threadIdx.x / kQuads, e = threadIdx.x % kQuads;
  float top = -__builtin_inff(), l = 0.f;
  vec<float, 4> o = {0.f, 0.f, 0.f, 0.f};
  if (there) {
    for (int s = k; s < parts; s += SPLIT) top = fmaxf(top, pm[2 * (at + s * step)]);
#pragma unroll 4
    for (int s = k; s < parts; s += SPLIT) {
      const int64_t a = at + s * step;
      const float m = pm[2 * a], by = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
      l += pm[2 * a + 1] * by;
      o += *reinterpret_cast<const vec<float, 4> *>(po + a * A.dim + d) * by;
    }
  }
  if constexpr (SPLIT > 1) {
    __shared__ vec<float, 4> sums[SPLIT][kQuads];
    __shared__ float ml[2][SPLIT][kQuads];
    sums[k][e] = o, ml[0][k][e] = top, ml[1][k][e] = l;
    __syncthreads();
    for (int w = 1; w < SPLIT; ++w) top = fmaxf(top, ml[0][w][e]);
    l = 0.f, o = vec<float, 4>{0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < SPLIT; ++w) {
      const float m = ml[0][w][e], by = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
      l += ml[1][w][e] * by;
      o += sums[w][e] * by;
    }
  }
  if (k != 0 || !there) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const float y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  store_vec<T, 4>(reinterpret_cast<T *>(A.out) + row * A.dim + d, y);
  if (d == 0 && A.lse) A.lse[row] = (top + __builtin_amdgcn_logf(l)) * kLn2F;
}

// Workgroups of a sequence with few rows, and of a token.
inline __host__ __device__ uint32_t few_joins(const AttendArgs &A) {
  return (uint32_t)(((int64_t)A.heads * A.few_rows * (A.dim / 4) + kJoinQuads - 1) / kJoinQuads);
}
inline __host__ __device__ uint32_t many_joins(const AttendArgs &A) {
  return (uint32_t)(((int64_t)A.heads * A.group * (A.dim / 4) + kJoinThreads - 1) / kJoinThreads);
}
// All of them: below 2^31, so that the kernel counts them in 32 bits (a call with more is refused).
inline int64_t joins_of(const AttendArgs &A) { return (A.joined ? (int64_t)few_joins(A) * A.s.n_seqs : 0) + A.many_joined; }

template <typename T>
__global__ __launch_bounds__(kJoinThreads) void attend_join_kernel(AttendArgs A) {
  const int g = A.group, hq = A.heads * g, quads = A.dim / 4;
  uint32_t id = block_id();
  const uint32_t few = few_joins(A), few_all = A.joined ? few * A.s.n_seqs : 0u;
  int b;
  if (id < few_all) {
    b = (int)(id / few);
    const Seq sq = seq_of(A.s, b);
    const Few f = few_of(A, sq);
    if (!f.few || f.tokens <= A.few_least) return;
    const int per = few_per(A), parts = (f.tokens + per - 1) / per;
    if (parts <= 1) return;
    const uint32_t unit = units_before(A.s, b, [&](const Seq &s) { return few_parts(A, s, per); });
    const int rows = sq.n * g, e = (int)(id % few) * kJoinQuads + threadIdx.x % kJoinQuads;
    const int r = e / quads % rows, head = e / quads / rows;
    join_row<T, 8>(A, A.few_o, A.few_ml, ((int64_t)unit * A.heads + head) * A.few_rows + r, (int64_t)A.heads * A.few_rows, parts,
                (int64_t)(sq.row + r / g) * hq + head * g + r % g, e % quads * 4, head < A.heads);
    return;
  }
  id -= few_all;
  if (id >= (uint32_t)A.many_joined) return;
  const Plan plan = plan_of(A);
  if (plan.per == kUncut) return;
  const uint32_t many = many_joins(A);
  for (int64_t at = id; at < A.s.n_tokens * many; at += A.many_joined) {
    uint32_t k;
    Seq sq;
    // the rows that are some sequence's are counted, as what starts before the call's rows is none
    if (!find_unit(A.s, (uint32_t)(at / many), [](const Seq &s) { return (uint32_t)s.n; }, b, k, sq)) continue;
    if (!many_tiles(A, sq)) continue;
    const uint32_t unit = units_before(A.s, b, [&](const Seq &s) { return many_units(A, s, plan.per); });
    const int len = sq.pos + sq.n, rows = sq.n * g, e = (int)(at % many) * kJoinThreads + threadIdx.x;
    const int head = min(e / quads, hq - 1), i = (int)k, r = i * g + head % g;
    const int tile = r / A.many_rows, r0 = tile * A.many_rows, r1 = min(r0 + A.many_rows, rows);
    const Span sp = span_of(A, sq.pos + r0 / g, sq.pos + (r1 - 1) / g, len, plan.per);
    const int64_t first = unit + (int64_t)tile * many_parts(A, sq, plan.per);
    join_row<T, 1>(A, A.many_o, A.many_ml, (first * A.heads + head / g) * A.many_rows + r - r0, (int64_t)A.heads * A.many_rows, sp.parts,
                   (int64_t)(sq.row + i) * hq + head, e % quads * 4, sp.parts > 1 && e < hq * quads);
  }
}

template <typename T, bool BYTES, int DP>
hipError_t attend_run(const AttendArgs &A, hipStream_t st) {
  constexpr int kTokenDim = BYTES && DP == 96 ? 128 : DP;  // keys of 8 bits are read 64 entries at a time
  const bool token = A.few_rows <= kTokenRows;
  const int waves = token ? kTokenWaves : 4;
  const size_t few = (size_t)waves * 4 * (token ? std::max(A.few_rows * (kTokenDim + 4), 4 * kTokenDim) : std::max(A.few_rows * (DP + 4), 2 * DP));
  const size_t many = DP <= kWideDim ? (size_t)Wide<T, BYTES, DP>::kBytes
                                     : (size_t)2 * (kManyStep * (DP + 8) + DP * (kManyStep + 8)) * 2 + 2 * DP * 16 + 16;
  void (*few_kernel)(AttendArgs) = attend_few_kernel<T, BYTES, DP>;
  if (token) few_kernel = attend_token_kernel<T, BYTES, kTokenDim>;
  void (*many_kernel)(AttendArgs);
  int many_threads = 256;
  if constexpr (DP <= kWideDim)
    many_kernel = attend_wide_kernel<T, BYTES, DP>, many_threads = 64 * Wide<T, BYTES, DP>::kWaves;
  else
    many_kernel = attend_many_kernel<T, BYTES, DP>;
  for (int i = 0; i < 2; ++i)  // LDS beyond 64 KiB is asked for
    if ((i ? many : few) > 65536 && (i == 0 || A.tiles)) {
      const hipError_t e = hipFuncSetAttribute(i ? reinterpret_cast<const void *>(many_kernel) : reinterpret_cast<const void *>(few_kernel),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)(i ? many : few));
      if (e != hipSuccess) return e;
    }
  few_kernel<<<grid_of((int64_t)A.few_units * A.heads), 64 * waves, few, st>>>(A);
  if (A.tiles) many_kernel<<<grid_of((int64_t)A.many_units * A.heads), many_threads, many, st>>>(A);
  const int64_t joins = joins_of(A);
  if (joins) attend_join_kernel<T><<<grid_of(joins), kJoinThreads, 0, st>>>(A);
  return hipGetLastError();
}

template <typename T, bool BYTES>
hipError_t attend_dim(const AttendArgs &A, hipStream_t st) {
  if (A.dim <= 64) return attend_run<T, BYTES, 64>(A, st);
  if (A.dim <= 96) return attend_run<T, BYTES, 96>(A, st);
  if (A.dim <= 128) return attend_run<T, BYTES, 128>(A, st);
  if (A.dim <= 192) return attend_run<T, BYTES, 192>(A, st);
  return attend_run<T, BYTES, 256>(A, st);
}

#endif  // __HIPCC__

}  // namespace cfp
