// The experts' products and their gradient.
//
// For an assignment a of token t to expert e with weight w (A assignments, in the
// order of their expert):
//     [g u] = x_t W1_e^T,  s = silu(g) u,  o = s W2_e^T,  y_t = sum over t's a of w o.
// Backwards, with silu'(g) = sg (1 + g (1 - sg)), sg = 1 / (1 + exp(-g)):
//     p = dy_t W2_e,  dw = s . p,  dg = w p u silu'(g),  du = w p silu(g),
//     dx_t = sum over t's a of [dg du] W1_e,
//     dW1_e = sum over e's a of [dg du]^T x_t,  dW2_e = sum over e's a of dy_t^T (w s).
// All six products run on the matrix units with 32-bit sums.  Rounded to 16 bits
// between products: s, [dg du] and w s, which the next product takes as operands.
// Kept in 32 bits: g and u for the backward pass (the gradients and dw are computed
// from them), and the experts' outputs and the rows of dx, which wait for the sum over a token's experts.
// float16 holds too few magnitudes for what lies between the products (s is a product of two sums, gradients are often
// below 2^-14 where its bits run out), so there s, [dg du] and w s are first written in 32 bits and then rounded
// under a power of two for every vector that a product sums over, which the product's result is multiplied by.
// Nothing is added through memory in an order that could change: a token's rows are
// gathered and summed by the token.
//
// Measured, bfloat16, rates of the products alone (the card's library reaches 1.5 to 1.6 PFLOP/s on one large
// product of rows by rows, 1.0 to 1.4 where an operand is transposed):
//     16384 tokens to 4 of 32 experts, 4096 wide, 1536 inside: up 1580 us (1.04 PFLOP/s), down 973 (0.85),
//     p = dy W2 1089 (0.76), rows of dx 1629 (1.01), dW1 1645 (1.00), dW2 853 us (0.97);
//     16384 tokens to 8 of 64, 2048 wide, 768 inside: up 820 us (1.01), down 626 (0.66);
//     4096 tokens to 2 of 16, 2048 wide, 1536 inside: 159, 105, 115, 193, 193 and 106 us (0.4 to 0.6).
// The large ones wait for the copies of a stage, which are issued when the stage before has landed; how much of that
// more copies on their way would hide has not been measured.  Down and the rows of dx also write their sums in 32
// bits.  The small ones have fewer tiles than the chip takes at a time, or not many more.
#include <algorithm>
#include <type_traits>

#include "block_common.h"

namespace cfp {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(1))) const void global_void;

// c += a b on the matrix unit, the sums in accumulation registers.  Written as an
// instruction because the register allocator, given 256 sums a lane, moves them between both
// halves of the register file inside the loop; it neither knows nor has to know the
// instruction's latency, as a sum is used again only FF * FR instructions later and
// read after settle().
template <typename T>
__device__ __forceinline__ void mfma(i16x8 a, i16x8 b, f32x4 &c) {
  if constexpr (std::is_same<T, bf16_t>::value)
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  else
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}

// Between vector instructions that write operands or sums and the matrix instructions that read them.
__device__ __forceinline__ void written() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 7" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Waits until every matrix instruction has written its sums (at most 18 cycles).
template <int M, int N>
__device__ __forceinline__ void settle(f32x4 (&acc)[M][N]) {
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int a = 0; a < M; ++a)
#pragma unroll
    for (int b = 0; b < N; ++b) asm volatile("" : "+a"(acc[a][b]));
}

constexpr int kStep = 64;  // entries of the sum's axis in a stage, 128 bytes: whole lines of the caches

// ---------------------------------------------------------------- operands --
//
// A stage of an operand is EXT vectors of 64 entries of the sum's axis, 16-byte
// pieces copied from memory straight into LDS.  An operand whose sum's axis is
// contiguous in memory ("along") lies as [EXT][8 pieces], piece c of vector r at
// place c ^ (r & 7), so that eight lanes that read one piece of eight vectors
// meet all 64 banks; one whose vectors' axis is contiguous ("across") lies as
// [64][EXT / 8 pieces] and is transposed by the read (ds_read_b64_tr_b16), with the
// places permuted so that the 16 rows of one read meet different banks.  Each
// wave copies kLoads pieces a lane; copy<I>() makes one of them.

template <int EXT>
__device__ __forceinline__ int across_place(int krow, int c) {
  return c ^ ((((krow & 3) | ((krow >> 3 & 1) << 2)) << 1) & (EXT / 8 - 1));
}

// Copies of 16 bytes a lane from memory to LDS: lane l's land at the byte set by copy_to, plus (I mod 4) KiB,
// plus 16 l.  Instructions of their own, as the compiler would wait for every copy before each
// transposing read; their only registers are read when they are issued, and nothing else in the
// kernel uses m0.  The instruction adds (I mod 4) KiB to the memory address as well, so
// that the addresses given are that much lower.  The waits are product_kernel's.
__device__ __forceinline__ void copy_to(uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" ::"s"(at) : "memory");
}
template <int I>
__device__ __forceinline__ void copy16(const char *from) {
  asm volatile("global_load_lds_dwordx4 %0, off offset:%1" ::"v"(from), "n"(I % 4 * 1024) : "memory");
}
// base: of the wave.  A memory instruction reads a scalar register that a vector instruction has written five wait
// states later at the earliest; the compiler, which keeps that distance for its own, does not know this one.
template <int I>
__device__ __forceinline__ void copy16(const char *base, uint32_t off) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1 offset:%2" ::"v"(off), "s"(base), "n"(I % 4 * 1024) : "memory");
}
// A value that is the same for all lanes, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ const char *uniform(const char *p) {
  return reinterpret_cast<const char *>(uniform(reinterpret_cast<int64_t>(p)));
}
constexpr int kBack = 4096;  // what wave bases lie lower, so that lane offsets stay positive

template <int N, typename F>
__device__ __forceinline__ void each(F f) {  // f(0) .. f(N - 1), the index a constant
  if constexpr (N > 0) {
    each<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// Rows in a run, from a base that all lanes share ("run"), or each with an address of its own.
template <int EXT, int WAVES, bool RUN>
struct Along {
  static constexpr int kLoads = EXT * 8 / (WAVES * 64);
  const char *base, *start;                                 // run: of the next stage and of the first, kBack lower
  std::conditional_t<RUN, uint32_t, const char *> p[kLoads];  // run: offset from base; each of the vector's first entry
  int k;         // first entry of this lane's pieces
  uint32_t off;  // what this lane adds for the stage
  // row(r): offset of vector r from `from`, or its address; the offsets stay below 2^31
  template <typename F>
  __device__ __forceinline__ void init(const char *from, F row) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    k = ((lane & 7) ^ (lane >> 3)) * 8;
    start = base = uniform(from) - kBack;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if constexpr (RUN)
        p[i] = (uint32_t)row((w * kLoads + i) * 8 + lane / 8) + kBack - i % 4 * 1024;
      else
        p[i] = row((w * kLoads + i) * 8 + lane / 8) - i % 4 * 1024;
    }
  }
  // pieces past the end of the sum's axis are the vector's first ones, which the reader masks
  __device__ __forceinline__ void begin(int k0, int K) {
    if constexpr (RUN) {
      off = k < K - k0 ? k * 2 : 0;
      if (k0 >= K) base = start;
    } else {
      off = k < K - k0 ? (uint32_t)(k0 + k) * 2 : 0;
    }
  }
  template <int I>
  __device__ __forceinline__ void copy() {
    if constexpr (RUN)
      copy16<I>(base, p[I] + off);
    else
      copy16<I>(p[I] + off);
  }
  __device__ __forceinline__ void end() {
    if constexpr (RUN) base += kStep * 2;
  }
};

template <int EXT, int WAVES>
struct AcrossPlace {
  static constexpr int kPer = EXT / 8;              // pieces of a row
  static constexpr int kRows = 64 / kPer;           // rows of a wave's load
  static constexpr int kLoads = kStep / (WAVES * kRows);
  static_assert(kLoads * WAVES * kRows == kStep, "");
  __device__ __forceinline__ static int row(int wave, int i) {
    return (wave * kLoads + i) * kRows + (int)(threadIdx.x & 63) / kPer;
  }
  // first vector of a load's piece; vectors past the end repeat the first ones and are not written
  __device__ __forceinline__ static int col(int wave, int i, int ext) {
    const int c = across_place<EXT>(row(wave, i), (int)(threadIdx.x & 63) % kPer) * 8;
    return c < ext ? c : 0;
  }
};

// Rows at one distance (64 of them within 2^31 bytes).  Rows past the end of the sum's axis are the
// first one, which the reader masks.
template <int EXT, int WAVES>
struct Across : AcrossPlace<EXT, WAVES> {
  using B = AcrossPlace<EXT, WAVES>;
  const char *base, *start;
  uint32_t p[B::kLoads], far[B::kLoads];  // offset of the column, and of the row
  int64_t step;
  int left, row0;
  __device__ __forceinline__ void init(const char *first, int64_t ld, int ext) {
    const int wave = threadIdx.x >> 6;
    start = base = uniform(first) - kBack;
#pragma unroll
    for (int i = 0; i < B::kLoads; ++i) {
      p[i] = B::col(wave, i, ext) * 2 + kBack - i % 4 * 1024;
      far[i] = p[i] + B::row(wave, i) * (uint32_t)ld;
    }
    row0 = B::row(wave, 0);
    step = kStep * uniform(ld);
  }
  __device__ __forceinline__ void begin(int k0, int K) {
    left = K - k0;
    if (left <= 0) base = start;
  }
  template <int I>
  __device__ __forceinline__ void copy() {
    copy16<I>(base, row0 + I * B::kRows < left ? far[I] : p[I]);
  }
  __device__ __forceinline__ void end() { base += step; }
};

// Rows by a list of assignments, whose entries a wave reads in scalar loads before it copies.
template <int EXT, int WAVES>
struct AcrossList : AcrossPlace<EXT, WAVES> {
  using B = AcrossPlace<EXT, WAVES>;
  typedef __attribute__((address_space(4))) const int32_t scalar_int;
  static constexpr int kEach = B::kLoads * B::kRows;  // rows of a wave
  static_assert(kEach <= CFP_PLAN_PAD, "");
  const char *p[B::kLoads];
  int64_t ld;
  scalar_int *list;
  uint32_t magic, shift;
  int32_t now[kEach];
  int first;
  __device__ __forceinline__ void init(const char *base, int64_t ld_, int ext, const int32_t *list_, uint32_t m,
                                       uint32_t sh, int wave) {
#pragma unroll
    for (int i = 0; i < B::kLoads; ++i) p[i] = base + B::col(wave, i, ext) * 2 - i % 4 * 1024;
    ld = uniform(ld_), list = (scalar_int *)uniform(reinterpret_cast<const char *>(list_)), magic = m, shift = sh;
    first = wave * kEach;
  }
  // The list goes on for CFP_PLAN_PAD entries behind its last.  Those past the end of the sum's axis are
  // another expert's or -1, taken as 0: rows that exist, which the reader masks.
  __device__ __forceinline__ void begin(int k0, int K) {
    scalar_int *at = list + min(k0 + first, K);
#pragma unroll
    for (int i = 0; i < kEach; ++i) now[i] = at[i];
  }
  __device__ __forceinline__ int64_t offset(int32_t a) const {
    return (int64_t)((uint64_t)(uint32_t)max(__builtin_amdgcn_readfirstlane(a), 0) * magic >> shift) * ld;
  }
  template <int I>
  __device__ __forceinline__ void copy() {
    const int sub = (int)(threadIdx.x & 63) / B::kPer;
    int64_t off = offset(now[I * B::kRows]);
#pragma unroll
    for (int x = 1; x < B::kRows; ++x) {
      const int64_t o = offset(now[I * B::kRows + x]);
      off = sub == x ? o : off;
    }
    copy16<I>(p[I] + off);
  }
  __device__ __forceinline__ void end() {}
};

// Zeros from entry `have` on.
__device__ __forceinline__ void mask(i16x8 &v, int have) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < have ? v[i] : (short)0;
}

// What the matrix instructions take from a stage: the vectors from r0 on, 16 an instruction.
template <int EXT, bool ACROSS, int N>
struct Reader {
  uint32_t at[ACROSS ? N : 2];  // byte of this lane's entries in a stage, for each 16 vectors (along: for each half)
  static constexpr int kReads = ACROSS ? 2 : 1;
  __device__ __forceinline__ void init(int r0) {
    const int l = threadIdx.x & 63, j = l & 15, g = l >> 4;
    if constexpr (!ACROSS) {
      at[0] = (r0 + j) * 128 + ((g ^ (j & 7)) << 4);
      at[1] = at[0] ^ 64;
    } else {
      const int kr = g * 8 + (j >> 2);
#pragma unroll
      for (int b = 0; b < N; ++b) {
        const int c = r0 + b * 16 + (j & 3) * 4;
        at[b] = kr * (EXT * 2) + (across_place<EXT>(kr, c >> 3) << 4) + (c & 7) * 2;
      }
    }
  }
  // one of kReads parts of the operand of vectors r0 + 16 B on, entries 32 HALF on, from the stage at `lds`
  template <int B, int HALF, int PART>
  __device__ __forceinline__ void read(const char *lds, i16x8 &v) const {
    if constexpr (!ACROSS) {
      v = *reinterpret_cast<const i16x8 *>(lds + at[HALF] + B * 2048);
    } else {
      const i16x4 x =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + at[B] + (HALF * 32 + PART * 4) * EXT * 2));
#pragma unroll
      for (int i = 0; i < 4; ++i) v[PART * 4 + i] = x[i];
    }
  }
};

// ------------------------------------------------------------------- tiles --

enum Product { kUp, kDown, kBackUp, kBackDown, kGradW1, kGradW2 };

// The experts' outputs before the weighted sum.
struct Outputs {
  float *out;  // [rows][ld]
  int64_t ld;
};

// Whether operands between the products are rounded under powers of two (see above).
template <typename T>
constexpr bool kScaled = std::is_same<T, f16_t>::value;
// The power of two of a vector whose largest finite magnitude is m, as the exponent that m has as a float: m in
// [2^e, 2^(e + 1)) goes to [2^14, 2^15).  Entries that are not finite stay so; those 2^28 below m begin to lose bits.
__device__ __forceinline__ float finite(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }
__device__ __forceinline__ int exponent(float m) { return (int)(__float_as_uint(m) >> 23); }
__device__ __forceinline__ float scale_down(float x, int e) { return ldexpf(x, 141 - e); }
__device__ __forceinline__ float scale_up(float x, int e) { return ldexpf(x, e - 141); }

struct Args {
  // operands: rows of the tile (assignments, or output rows of a weight gradient), and features
  const char *row, *feat;
  int64_t ld_row, ld_feat;     // bytes
  int64_t feat_expert;         // bytes between experts
  const int32_t *offsets, *rows;
  int32_t experts;
  uint32_t magic, shift;       // token of an assignment a: a * magic >> shift
  int32_t K;                   // length of the sum's axis (of the grouped rows: the products over assignments ignore it)
  int32_t n_row, n_feat;       // extents of the output (n_row: weight gradients)
  int32_t F, Fp;               // inner width, and as laid out
  int32_t deal_rows;           // weight gradients: blocks of row tiles that eight dies divide, 1, 2, 4 or 8
  // epilogues
  void *out;                   // 16-bit rows; float rows of operands to be scaled
  int64_t ld_out;              // elements
  float *h;                    // g and u in blocks of 16 assignments of an expert x 16 features, gate block then up block, each
                               // in the order of the lanes that make and take it; expert e's from block row first / 16 + e on
  const float *weight;         // [T * k]
  void *out2;                  // w s, rows like those of out, ld_out2 elements apart
  int64_t ld_out2;
  const uint8_t *exps;         // weight gradients from scaled operands: exponents of an expert's Fp + Fp + Fp columns
  Outputs outputs;             // kDown, kBackDown
  float *dot;                  // [A][dot_tiles]: s . p over a feature tile
  int32_t dot_tiles;
};

// Which expert and tile the workgroup takes: tiles of all experts in a row, dealt in
// eight runs, one for each die, whose workgroups then meet the same weights in its cache.
struct Place {
  int expert, tile, first, count;  // first and count: the expert's assignments
};

__device__ __forceinline__ int dealt(int i, int total) {
  const int x = i & 7, q = total >> 3, r = total & 7;
  return x * q + min(x, r) + (i >> 3);
}

// All lanes of a wave; tiles of BR assignments; nt feature tiles each.  An expert's tiles go in groups of
// kGroup row tiles, a group's rows first, so that the workgroups that a die runs at a time form a
// block of tiles with few different rows and features (large training step, groups of 1, 4 and 8: up 1.74, 1.66
// and 1.62 ms, L2 misses 50, 36 and 36 million).
constexpr int kGroup = 8;

template <int BR>
__device__ __forceinline__ bool find(const Args &A, uint32_t block, int nt, Place &p, int &ft) {
  const int lane = threadIdx.x & 63;
  int total = 0;
  for (int e0 = 0; e0 < A.experts; e0 += 64) {
    const int e = e0 + lane;
    int c = e < A.experts ? (A.offsets[e + 1] - A.offsets[e] + BR - 1) / BR : 0;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) c += __shfl_xor(c, off, 64);
    total += __builtin_amdgcn_readfirstlane(c);
  }
  if ((int64_t)block >= (int64_t)total * nt) return false;
  const int id = dealt(block, total * nt);
  const int tile = id / nt;
  int before = 0;
  for (int e0 = 0; e0 < A.experts; e0 += 64) {
    const int e = e0 + lane;
    const int lo = e < A.experts ? A.offsets[e] : 0, hi = e < A.experts ? A.offsets[e + 1] : 0;
    const int own = (hi - lo + BR - 1) / BR;
    int c = own;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int y = __shfl_up(c, off, 64);
      if (lane >= off) c += y;
    }
    const uint64_t past = __ballot(before + c <= tile);
    const int k = __popcll(past);
    if (k < 64) {
      const int rows = __builtin_amdgcn_readfirstlane(__shfl(own, k, 64));
      const int local = id - (before + __builtin_amdgcn_readfirstlane(__shfl(c, k, 64)) - rows) * nt;  // among the expert's
      const int group = local / (kGroup * nt), in = local - group * kGroup * nt, wide = min(kGroup, rows - group * kGroup);
      ft = in / wide;
      p.expert = e0 + k;
      p.tile = group * kGroup + in - ft * wide;
      p.first = __builtin_amdgcn_readfirstlane(__shfl(lo, k, 64));
      p.count = __builtin_amdgcn_readfirstlane(__shfl(hi, k, 64)) - p.first;
      return true;
    }
    before += __builtin_amdgcn_readfirstlane(__shfl(c, 63, 64));
  }
  return false;
}

// 1 / (1 + 2^t), t = -x log2(e), within four units of the last place.  The rounding of the product t alone would be
// |x| units of 2^t: its rest r, in two parts of log2(e), is taken up as 2^(t + r) = 2^t (1 + r ln 2).  Past |x| = 100
// the value is 1 or, below 2^-126 already at x = -88, 0.
__device__ __forceinline__ float sigmoid(float x) {
  constexpr float kHigh = -1.44269502f, kLow = -1.92596299e-8f, kLn2 = 0.693147181f;
  x = fminf(fmaxf(x, -100.f), 100.f);
  const float t = x * kHigh, r = fmaf(x, kLow, fmaf(x, kHigh, -t));
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(t) * fmaf(r, kLn2, 1.f));
}

// BR rows x BF features by WR x WF waves.  The features are the matrix instruction's
// first operand, so that a lane holds four consecutive features of one row.
//
// Two stages of 64 entries of the sum's axis lie in LDS; a matrix instruction takes half of one.  While
// the matrix units work on the first half of stage s, whose operands are in registers, those of its
// second half are read from LDS; then one barrier, after which every wave has read stage s and stage
// s + 1 has landed; while they work on the second half, the first operands of stage s + 1 are read and
// stage s + 2 is copied over stage s.  Reads and copies are spread between the matrix instructions.
// Copies go on past the end of the sum, over rows that exist.
//
// A tile of 256 x 256 copies least for its products (64 KiB for 2048 cycles of the matrix units) and has 256 sums
// a lane, all of the accumulation registers, so one workgroup a compute unit; of 128 x 128 two run and of 64 x 128
// three, whose parts outside the loop overlap.
template <typename T, int P, int BR, int BF, int WR, int WF>
__device__ __forceinline__ void product_tile(const Args &A, uint32_t block) {
  constexpr int WAVES = WR * WF, THREADS = WAVES * 64;
  constexpr int TR = BR / WR, TF = BF / WF, FR = TR / 16, FF = TF / 16;
  constexpr bool kGrad = P == kGradW1 || P == kGradW2;
  constexpr bool kRowAcross = kGrad, kFeatAcross = kGrad || P == kBackUp || P == kBackDown;
  constexpr int kFeatTile = P == kUp ? BF / 2 : BF;  // kUp: half gate, half up
  constexpr int kBytes = (BR + BF) * kStep * 2;
  extern __shared__ __align__(16) char smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / WF, wf = wave % WF;
  const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;

  Place pl;
  int ft, rt = 0, K;
  if constexpr (kGrad) {
    const int nf = (A.n_feat + BF - 1) / BF, nr = (A.n_row + BR - 1) / BR;
    // every die takes a block of each expert's tiles, as the experts' sums differ in length
    const int x = block & 7, i = block >> 3, br = (nr + A.deal_rows - 1) / A.deal_rows,
              bf = (nf * A.deal_rows + 7) / 8;
    pl.expert = i / (br * bf);
    if (pl.expert >= A.experts) return;
    const int in = i - pl.expert * br * bf;
    rt = x % A.deal_rows * br + in % br;
    ft = x / A.deal_rows * bf + in / br;
    if (rt >= nr || ft >= nf) return;
    pl.first = __builtin_amdgcn_readfirstlane(A.offsets[pl.expert]);
    pl.count = __builtin_amdgcn_readfirstlane(A.offsets[pl.expert + 1]) - pl.first;
    K = pl.count;
  } else {
    const int nt = ((P == kUp ? A.F : A.n_feat) + kFeatTile - 1) / kFeatTile;
    if (!find<BR>(A, block, nt, pl, ft)) return;
    rt = pl.tile;
    K = A.K;
  }
  const int r0 = rt * BR, f0 = ft * kFeatTile;
  const int n_rows = kGrad ? A.n_row : pl.count;

  constexpr bool kRowList = P == kGradW2, kFeatList = P == kGradW1;
  constexpr bool kGather = P == kUp || P == kBackUp;
  using RowLoad = std::conditional_t<!kRowAcross, Along<BR, WAVES, !kGather>,
                                     std::conditional_t<kRowList, AcrossList<BR, WAVES>, Across<BR, WAVES>>>;
  using FeatLoad = std::conditional_t<!kFeatAcross, Along<BF, WAVES, true>,
                                      std::conditional_t<kFeatList, AcrossList<BF, WAVES>, Across<BF, WAVES>>>;
  RowLoad rl;
  FeatLoad fl;
  if constexpr (kRowList) {
    rl.init(A.row + (int64_t)r0 * 2, A.ld_row, A.n_row - r0, A.rows + pl.first, A.magic, A.shift, wave);
  } else if constexpr (kRowAcross) {
    rl.init(A.row + pl.first * A.ld_row + (int64_t)r0 * 2, A.ld_row, A.n_row - r0);
  } else {
    // rows past the end repeat the last one and are not written
    if constexpr (kGather)
      rl.init(nullptr, [&](int r) {
        const int64_t a = A.rows[pl.first + min(r0 + r, n_rows - 1)];
        return A.row + (int64_t)((uint64_t)a * A.magic >> A.shift) * A.ld_row;
      });
    else
      rl.init(A.row + (int64_t)(pl.first + r0) * A.ld_row,
              [&](int r) { return (uint32_t)min(r, n_rows - 1 - r0) * (uint32_t)A.ld_row; });
  }
  if constexpr (kFeatList) {
    fl.init(A.feat + (int64_t)f0 * 2, A.ld_feat, A.n_feat - f0, A.rows + pl.first, A.magic, A.shift, wave);
  } else if constexpr (kFeatAcross) {
    fl.init(A.feat + (kGrad ? pl.first * A.ld_feat : pl.expert * A.feat_expert) + (int64_t)f0 * 2, A.ld_feat,
            A.n_feat - f0);
  } else {
    fl.init(A.feat + pl.expert * A.feat_expert + (int64_t)f0 * A.ld_feat, [&](int n) {
      if constexpr (P == kUp) {
        const int w = n / TF, x = n % TF, f = min(w * (TF / 2) + x % (TF / 2), A.F - 1 - f0);
        return (uint32_t)(f + (x < TF / 2 ? 0 : A.Fp)) * (uint32_t)A.ld_feat;
      } else {
        return (uint32_t)min(n, A.n_feat - 1 - f0) * (uint32_t)A.ld_feat;
      }
    });
  }
  constexpr int kRowLoads = RowLoad::kLoads, kFeatLoads = FeatLoad::kLoads, kLoads = kRowLoads + kFeatLoads;
  // where this wave's copies of a stage begin
  const uint32_t row_to = (uint32_t)(uintptr_t)(lds_void *)smem + wave * kRowLoads * 1024;
  const uint32_t feat_to = (uint32_t)(uintptr_t)(lds_void *)smem + BR * kStep * 2 + wave * kFeatLoads * 1024;
  // copy i of a stage that lies `at` bytes behind the first
  auto copy = [&](auto i, uint32_t at) {
    if constexpr (i.value < kRowLoads && i.value % 4 == 0) copy_to(row_to + at + i.value * 1024);
    if constexpr (i.value >= kRowLoads && (i.value - kRowLoads) % 4 == 0)
      copy_to(feat_to + at + (i.value - kRowLoads) * 1024);
    if constexpr (i.value < kRowLoads)
      rl.template copy<i.value>();
    else
      fl.template copy<i.value - kRowLoads>();
  };
  Reader<BF, kFeatAcross, FF> fread;
  Reader<BR, kRowAcross, FR> rread;
  fread.init(wf * TF);
  rread.init(wr * TR);

  f32x4 acc[FF][FR];
#pragma unroll
  for (int a = 0; a < FF; ++a)
#pragma unroll
    for (int b = 0; b < FR; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  written();
  const int steps = (K + kStep - 1) / kStep;
  if (steps > 0) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      rl.begin(s * kStep, K);
      fl.begin(s * kStep, K);
      each<kLoads>([&](auto i) { copy(i, s * kBytes); });
      rl.end();
      fl.end();
    }
    i16x8 fo[2][FF], ro[2][FR];
    constexpr int kFeatReads = FF * fread.kReads, kReads = kFeatReads + FR * rread.kReads, kMfma = FF * FR;
    // read number r of half h of the stage at `lds`
    auto read = [&](auto r, auto h, const char *lds) {
      if constexpr (r.value < kFeatReads) {
        constexpr int x = r.value / fread.kReads;
        fread.template read<x, h.value, r.value % fread.kReads>(lds + BR * kStep * 2, fo[h.value][x]);
      } else {
        constexpr int x = (r.value - kFeatReads) / rread.kReads;
        rread.template read<x, h.value, (r.value - kFeatReads) % rread.kReads>(lds, ro[h.value][x]);
      }
    };
    // The FF * FR instructions of half h, with the reads of the other half from `lds` and COPIES copies to `to` between them.
    auto half = [&](auto h, const char *lds, auto n_copies, uint32_t to, int have) {
      constexpr int kCopies = n_copies.value;
      if (have < 32) {  // the sum ends in this half: entries behind its end count for nothing in either operand
        each<FF>([&](auto a) { mask(fo[h.value][a.value], have - g * 8); });
        each<FR>([&](auto b) { mask(ro[h.value][b.value], have - g * 8); });
        written();
      }
      each<kMfma>([&](auto m) {
        constexpr int a = m.value / FR, b = m.value % FR;
        mfma<T>(fo[h.value][a], ro[h.value][b], acc[a][b]);
        // evenly: copies in a row at the start of the half meet a full queue of the vector cache (up 1.79 against 1.66 ms)
        constexpr int kOps = kReads + kCopies;
        constexpr int o0 = m.value * kOps / kMfma, o1 = (m.value + 1) * kOps / kMfma;
        each<o1 - o0>([&](auto oc) {
          constexpr int o = o0 + oc.value, copies = (o + 1) * kCopies / kOps;  // up to and with this operation
          if constexpr (copies > o * kCopies / kOps)
            copy(std::integral_constant<int, copies - 1>{}, to);
          else
            read(std::integral_constant<int, o - copies>{}, std::integral_constant<int, 1 - h.value>{}, lds);
        });
        if constexpr (o1 > o0) __builtin_amdgcn_sched_barrier(0);
      });
    };
    const std::integral_constant<int, 0> zero;
    const std::integral_constant<int, 1> one;
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLoads) : "memory");
    each<kReads>([&](auto r) { read(r, zero, smem); });
    uint32_t slot = 0;
    for (int s = 0; s < steps; ++s) {
      const int have = K - s * kStep;
      __builtin_amdgcn_sched_barrier(0);
      rl.begin((s + 2) * kStep, K);
      fl.begin((s + 2) * kStep, K);
      half(zero, smem + slot, zero, 0, have);
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      const uint32_t old = slot;
      slot = kBytes - slot;
      half(one, smem + slot, std::integral_constant<int, kLoads>{}, old, have - 32);
      rl.end();
      fl.end();
      // a copy of a sum that the register allocator might place here reads it written
      asm volatile("s_nop 10");
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // copies still on their way end before the LDS is used again
    settle(acc);
  }

  // ---- epilogues: lane (j, g) holds features 4 g .. 4 g + 3 of row j of each 16 x 16 block.  Stores of
  // such pieces touch 16 lines each and took 60 cycles apiece, half of the 31 thousand cycles of a weight gradient's
  // tile of two stages.  So 16-bit results pass through LDS, a part of its own for each wave, and leave in whole
  // rows of that (4096 tokens to 2 of 16 experts, 2048 wide, 1536 inside, tiles of 256 x 256: dW1 from 185 to 170 us,
  // dW2 from 105 to 97 us); what is kept in 32 bits is laid out by blocks in the lanes' order, and other results in 32
  // bits go out as 64 bytes of each row.
  const int width = P == kUp || P == kBackUp ? A.F : P == kDown || P == kBackDown ? (int)A.outputs.ld : (int)A.ld_out;
  const bool inside = f0 + kFeatTile <= width && r0 + BR <= n_rows && (P != kGradW1 || A.F == A.Fp);
  constexpr int kCols = P == kUp ? TF / 2 : TF, kPieces = kCols / 8;  // a wave's results of a row
  constexpr int kHold = P == kBackUp ? 48 : TR;               // rows of its part
  static_assert(kHold * kCols * 2 * WAVES <= 2 * kBytes && 16 * kPieces % 64 == 0, "");
  char *mine = smem + wave * kHold * kCols * 2;
  auto put = [&](int row, int col, const vec<T, 4> &v) {
    *reinterpret_cast<vec<T, 4> *>(mine + row * kCols * 2 + ((col >> 3 ^ (row & (kPieces - 1))) << 4) + (col & 4) * 2) = v;
  };
  // `rows` rows from row `from` of the wave's part, to to(row): where the wave's first result of that row of the part
  // goes, or null; `limit` results of a row exist
  auto flush = [&](auto rows, int from, auto to, int limit) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int i = 0; i < rows.value * kPieces / 64; ++i) {
      const int row = i * (64 / kPieces) + lane / kPieces, c = lane % kPieces;
      const vec<T, 8> v =
          *reinterpret_cast<const vec<T, 8> *>(mine + (from + row) * kCols * 2 + ((c ^ (row & (kPieces - 1))) << 4));
      T *at = to(row);
      if (at == nullptr || c * 8 >= limit) continue;
      if (!kGrad || c * 8 + 8 <= limit) {  // the others have a multiple of 8 results in a row
        __builtin_memcpy(at + c * 8, &v, 16);  // at any address: rows of an odd width
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c * 8 + e < limit) at[c * 8 + e] = v[e];
      }
    }
  };
  constexpr std::integral_constant<int, TR> kAll{};
  __syncthreads();  // every wave has read its last stage
  auto finish = [&](auto whole) {
    constexpr bool kWhole = whole.value;
    const int i0 = r0 + wr * TR;       // the wave's first row
    const int c0 = f0 + wf * kCols;    // and first feature
    const int64_t a0 = pl.first + i0;  // its assignment, where rows are assignments
    // the row's place in `base`, ld results a row
    auto rows_of = [&](void *base, int64_t ld) {
      return [=](int row) -> T * {
        return kWhole || i0 + row < n_rows ? reinterpret_cast<T *>(base) + (a0 + row) * ld + c0 : nullptr;
      };
    };
    using Between = std::conditional_t<kScaled<T>, float, T>;
    // this lane's four entries of the block of rows b and features q in rows of floats
    auto wide = [&](void *base, int64_t ld, int b, int q) {
      return reinterpret_cast<float *>(base) + (a0 + b * 16 + j) * ld + c0 + q * 16 + g * 4;
    };
    const int Fb = (A.F + 15) / 16;
    // this lane's part of the block of rows b and features q of what is kept: gate, and 256 entries on, up
    auto kept = [&](int b, int q) {
      return A.h + ((int64_t)(pl.first / 16 + pl.expert + i0 / 16 + b) * Fb + c0 / 16 + q) * 512 + lane * 4;
    };
    if constexpr (P == kUp) {
#pragma unroll
      for (int b = 0; b < FR; ++b) {
        if (!kWhole && i0 + b * 16 >= n_rows) continue;
#pragma unroll
        for (int q = 0; q < FF / 2; ++q) {
          if (!kWhole && c0 + q * 16 >= A.F) continue;
          f32x4 ga, up;
          vec<Between, 4> s;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool in = kWhole || c0 + q * 16 + g * 4 + e < A.F;
            ga[e] = in ? acc[q][b][e] : 0.f;
            up[e] = in ? acc[q + FF / 2][b][e] : 0.f;
            s[e] = (Between)(ga[e] * sigmoid(ga[e]) * up[e]);
          }
          if constexpr (!kScaled<T>)
            put(b * 16 + j, q * 16 + g * 4, s);
          else if (kWhole || (i0 + b * 16 + j < n_rows && c0 + q * 16 + g * 4 < A.Fp))
            *reinterpret_cast<f32x4 *>(wide(A.out, A.ld_out, b, q)) = s;
          if (A.h != nullptr) {
            *reinterpret_cast<f32x4 *>(kept(b, q)) = ga;
            *reinterpret_cast<f32x4 *>(kept(b, q) + 256) = up;
          }
        }
      }
      if constexpr (!kScaled<T>) flush(kAll, 0, rows_of(A.out, A.ld_out), A.Fp - c0);
    } else if constexpr (P == kDown || P == kBackDown) {
#pragma unroll
      for (int b = 0; b < FR; ++b) {
        if (!kWhole && i0 + b * 16 + j >= n_rows) continue;
        float *to = A.outputs.out + (a0 + b * 16 + j) * A.outputs.ld + c0 + g * 4;
#pragma unroll
        for (int q = 0; q < FF; ++q)
          if (kWhole || c0 + q * 16 + g * 4 < width) *reinterpret_cast<f32x4 *>(to + q * 16) = acc[q][b];
      }
    } else if constexpr (P == kBackUp) {
      float dots[FR];
      constexpr std::integral_constant<int, 16> kBlock{};
      float weight[2];
      f32x4 gate[2][FF], value[2][FF];
      auto fetch = [&](auto at) {  // what a block of 16 rows takes, on its way while the block before is worked on
        constexpr int b = at.value;
        if (!kWhole && i0 + b * 16 >= n_rows) return;
        weight[b & 1] = kWhole || i0 + b * 16 + j < n_rows ? A.weight[A.rows[a0 + b * 16 + j]] : 0.f;
#pragma unroll
        for (int q = 0; q < FF; ++q) {
          if (!kWhole && c0 + q * 16 >= A.F) continue;
          gate[b & 1][q] = *reinterpret_cast<const f32x4 *>(kept(b, q));
          value[b & 1][q] = *reinterpret_cast<const f32x4 *>(kept(b, q) + 256);
        }
        __builtin_amdgcn_sched_barrier(0);
      };
      fetch(std::integral_constant<int, 0>{});
      each<FR>([&](auto at) {  // 16 rows at a time: dg, du and w s
        constexpr int b = at.value;
        dots[b] = 0.f;
        if constexpr (b + 1 < FR) fetch(std::integral_constant<int, b + 1>{});
        if (!kWhole && i0 + b * 16 >= n_rows) return;
        const float w = weight[b & 1];
#pragma unroll
        for (int q = 0; q < FF; ++q) {
          if (!kWhole && c0 + q * 16 >= A.F) continue;
          const f32x4 ga = gate[b & 1][q], up = value[b & 1][q];
          vec<Between, 4> dg, du, ws;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool in = kWhole || c0 + q * 16 + g * 4 + e < A.F;
            const float p = in ? acc[q][b][e] : 0.f;
            const float sg = sigmoid(ga[e]), si = ga[e] * sg, s = si * up[e];
            dots[b] += in ? s * p : 0.f;
            dg[e] = (Between)(w * p * up[e] * sg * (1.f + ga[e] * (1.f - sg)));
            du[e] = (Between)(w * p * si);
            ws[e] = (Between)(in ? w * s : 0.f);
          }
          if constexpr (!kScaled<T>) {
            put(j, q * 16 + g * 4, dg);
            put(16 + j, q * 16 + g * 4, du);
            put(32 + j, q * 16 + g * 4, ws);
          } else if (kWhole || (i0 + b * 16 + j < n_rows && c0 + q * 16 + g * 4 < A.Fp)) {
            float *to = wide(A.out, A.ld_out, b, q);
            *reinterpret_cast<f32x4 *>(to) = dg;
            *reinterpret_cast<f32x4 *>(to + A.Fp) = du;
            *reinterpret_cast<f32x4 *>(wide(A.out2, A.ld_out2, b, q)) = ws;
          }
        }
        if constexpr (kScaled<T>) return;
        auto rows_of = [&](void *base, int64_t ld) {
          return [=](int row) -> T * {
            const int i = i0 + b * 16 + row;
            return kWhole || i < n_rows ? reinterpret_cast<T *>(base) + (pl.first + (int64_t)i) * ld + c0 : nullptr;
          };
        };
        flush(kBlock, 0, rows_of(A.out, A.ld_out), A.Fp - c0);
        flush(kBlock, 16, rows_of(reinterpret_cast<T *>(A.out) + A.Fp, A.ld_out), A.Fp - c0);
        flush(kBlock, 32, rows_of(A.out2, A.ld_out2), A.Fp - c0);
      });
      float *part = reinterpret_cast<float *>(smem);  // [WF][BR]
      __syncthreads();
#pragma unroll
      for (int b = 0; b < FR; ++b) {
        float v = dots[b];
        v += __shfl_xor(v, 16, 64);
        v += __shfl_xor(v, 32, 64);
        if (g == 0) part[wf * BR + wr * TR + b * 16 + j] = v;
      }
      __syncthreads();
      for (int r = threadIdx.x; r < BR; r += THREADS) {
        if (!kWhole && r0 + r >= n_rows) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WF; ++w) v += part[w * BR + r];
        A.dot[(int64_t)(pl.first + r0 + r) * A.dot_tiles + ft] = v;
      }
    } else {  // gradients of the weights
#pragma unroll
      for (int b = 0; b < FR; ++b)
#pragma unroll
        for (int q = 0; q < FF; ++q) {
          f32x4 v = acc[q][b];
          if (kScaled<T> && pl.count > 0) {  // an expert's exponents: of gate, up and w s (not there without any row)
            const uint8_t *exps = A.exps + pl.expert * (int64_t)(3 * A.Fp);
            if constexpr (P == kGradW1) {
              const int by = exps[min(i0 + b * 16 + j, A.n_row - 1)];
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = scale_up(v[e], by);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = scale_up(v[e], exps[2 * A.Fp + min(c0 + q * 16 + g * 4 + e, A.Fp - 1)]);
            }
          }
          put(b * 16 + j, q * 16 + g * 4, vec<T, 4>{(T)v[0], (T)v[1], (T)v[2], (T)v[3]});
        }
      const int64_t per = P == kGradW1 ? 2 * A.F : A.n_row;
      T *o0 = reinterpret_cast<T *>(A.out) + (pl.expert * per + i0) * A.ld_out + c0;
      flush(
          kAll, 0,
          [&](int row) -> T * {
            if constexpr (kWhole) return o0 + row * A.ld_out;
            const int i = i0 + row, half = P == kGradW1 && i >= A.Fp;  // gate and up rows, each Fp as laid out
            if (i >= n_rows || (P == kGradW1 && i - half * A.Fp >= A.F)) return nullptr;
            return o0 + (row - half * (int64_t)(A.Fp - A.F)) * A.ld_out;
          },
          width - c0);
    }
  };
  if (inside)
    finish(std::true_type{});
  else
    finish(std::false_type{});
}

template <typename T, int P, int BR, int BF, int WR, int WF, int PER_CU>
__global__ __launch_bounds__(WR *WF * 64, PER_CU *WR *WF / 4) void product_kernel(Args A) {
  product_tile<T, P, BR, BF, WR, WF>(A, block_id());
}

// What follows from p = dy W2 in one launch: rows of dx, dW1 and dW2.  For steps whose products do not fill the
// chip one by one.
template <typename T>
__global__ __launch_bounds__(256, 3) void gradients_kernel(Args dx, Args dw1, Args dw2, uint32_t from1, uint32_t from2) {
  if (blockIdx.x < from1)
    product_tile<T, kBackDown, 64, 128, 2, 2>(dx, blockIdx.x);
  else if (blockIdx.x < from2)
    product_tile<T, kGradW1, 64, 128, 2, 2>(dw1, blockIdx.x - from1);
  else
    product_tile<T, kGradW2, 64, 128, 2, 2>(dw2, blockIdx.x - from2);
}

// ------------------------------------------------------------- few tokens --
//
// Where an expert has a few tokens the products are bound by reading its weights once.  A workgroup takes
// 32 rows of them (16 gate rows and their 16 up rows, or 32 rows of W2) for 16 NT tokens, and its four
// waves a quarter of the sum's axis each: the weights go from memory to the registers that the
// matrix instructions take them from, kMost steps of 2 KiB a wave ahead, and only the four partial
// sums meet in LDS.  Rows need no alignment (a piece of 8 entries is one load of 16 bytes at any
// address), so odd widths are read in place.
// 384 assignments to 64 experts, 2048 wide, 1024 inside: up 100 us (5.4 TB/s), down 57 us (4.7 TB/s); one token to 6:
// 14 and 8 us, bound by the latency of a launch and two or three rounds of loads.  Twice the steps on their way
// leaves half the waves: 110 and 68 us.

constexpr int kFewWaves = 4;

// Entries k .. k + 7 of a row of K, zeros behind its end, in two steps: one load of 16 bytes that ends with the
// row at the latest, then a shift by what it began too early.  (Entries tested one by one cost a wait each.)
__device__ __forceinline__ i16x8 piece_load(const char *row, int k, int K) {
  i16x8 v = {};
  if (K >= 8) {
    __builtin_memcpy(&v, row + (int64_t)min(k, K - 8) * 2, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k + i < K) v[i] = reinterpret_cast<const short *>(row)[k + i];
  }
  return v;
}
__device__ __forceinline__ i16x8 piece_shift(i16x8 v, int k, int K) {
  const int by = K >= 8 ? k - min(k, K - 8) : 0;
  unsigned __int128 x = __builtin_bit_cast(unsigned __int128, v);
  x = by < 8 ? x >> (by * 16) : 0;
  return __builtin_bit_cast(i16x8, x);
}

template <typename T>
__device__ __forceinline__ f32x4 mfma_v(i16x8 a, i16x8 b, f32x4 c) {  // with waits by the compiler
  if constexpr (std::is_same<T, bf16_t>::value)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <typename T, int P, int NT>
__global__ __launch_bounds__(kFewWaves * 64) void few_kernel(Args A) {
  constexpr int kMost = NT == 1 ? 8 : 4;  // steps of a wave on their way at once
  constexpr int kTile = P == kUp ? 16 : 32;  // features of a workgroup
  __shared__ f32x4 part[kFewWaves][NT * 2][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
  const int n_feat = P == kUp ? A.F : A.n_feat;
  Place pl;
  int ft;
  if (!find<16 * NT>(A, block_id(), (n_feat + kTile - 1) / kTile, pl, ft)) return;
  const int r0 = pl.tile * 16 * NT, f0 = ft * kTile, K = A.K;
  const char *base = A.feat + pl.expert * A.feat_expert;
  // rows past the end repeat the last one and are not written
  const char *w0 = base + (int64_t)min(f0 + j, n_feat - 1) * A.ld_feat;
  const char *w1 = P == kUp ? base + (int64_t)(min(f0 + j, n_feat - 1) + A.F) * A.ld_feat
                            : base + (int64_t)min(f0 + 16 + j, n_feat - 1) * A.ld_feat;
  const char *x[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    int64_t row = pl.first + min(r0 + t * 16 + j, pl.count - 1);
    if constexpr (P == kUp) row = (uint64_t)(uint32_t)A.rows[row] * A.magic >> A.shift;
    x[t] = A.row + row * A.ld_row;
  }
  const int steps = (K + 31) / 32, each = (steps + kFewWaves - 1) / kFewWaves;
  const int from = wave * each, to = min(from + each, steps);
  f32x4 acc[2][NT] = {};
  auto run = [&](int s, auto whole) {
    constexpr int kAhead = whole.value ? kMost : kMost / 2;  // the shifts at the end need registers of their own
    i16x8 a[2][kAhead], b[NT][kAhead];
    auto place = [&](int i) { return s + i < to ? (s + i) * 32 + g * 8 : K; };  // past this wave's part: zeros
    auto load = [&](const char *row, int i) {
      if constexpr (whole.value) {
        i16x8 v;
        __builtin_memcpy(&v, row + (int64_t)(s * 32 + g * 8) * 2 + i * 64, 16);
        return v;
      } else {
        return piece_load(row, place(i), K);
      }
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      a[0][i] = load(w0, i);
      a[1][i] = load(w1, i);
#pragma unroll
      for (int t = 0; t < NT; ++t) b[t][i] = load(x[t], i);
    }
    __builtin_amdgcn_sched_barrier(0);  // every load is on its way before the first is waited for
    if constexpr (!whole.value) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        a[0][i] = piece_shift(a[0][i], place(i), K);
        a[1][i] = piece_shift(a[1][i], place(i), K);
#pragma unroll
        for (int t = 0; t < NT; ++t) b[t][i] = piece_shift(b[t][i], place(i), K);
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        acc[0][t] = mfma_v<T>(a[0][i], b[t][i], acc[0][t]);
        acc[1][t] = mfma_v<T>(a[1][i], b[t][i], acc[1][t]);
      }
  };
  int s = from;
  for (; s + kMost <= to && (s + kMost) * 32 <= K; s += kMost) run(s, std::true_type{});
  for (; s < to; s += kMost / 2) run(s, std::false_type{});
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    part[wave][2 * t][lane] = acc[0][t];
    part[wave][2 * t + 1][lane] = acc[1][t];
  }
  __syncthreads();
  // lane (j, g) of the sum: features 4 g .. 4 g + 3 of token j
  for (int t = wave; t < NT; t += kFewWaves) {
    f32x4 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      v[h] = part[0][2 * t + h][lane];
#pragma unroll
      for (int w = 1; w < kFewWaves; ++w) v[h] += part[w][2 * t + h][lane];
    }
    const int i = r0 + t * 16 + j;
    if (i >= pl.count) continue;
    const int64_t at = pl.first + i;
    if constexpr (P == kUp) {
      const int f = f0 + g * 4;
      if (f >= A.Fp) continue;
      float s[4], ga[4], up[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = f + e < A.F;
        ga[e] = in ? v[0][e] : 0.f;
        up[e] = in ? v[1][e] : 0.f;
        s[e] = ga[e] * sigmoid(ga[e]) * up[e];
      }
      using Between = std::conditional_t<kScaled<T>, float, T>;
      store_vec<Between, 4>(reinterpret_cast<Between *>(A.out) + at * A.ld_out + f, s);
      if (A.h != nullptr) {  // the block of what is kept, in the lanes' order
        float *h = A.h + ((int64_t)(pl.first / 16 + pl.expert + r0 / 16 + t) * ((A.F + 15) / 16) + ft) * 512 + lane * 4;
        store_vec<float, 4>(h, ga);
        store_vec<float, 4>(h + 256, up);
      }
    } else {
      const Outputs &S = A.outputs;
      const int f = f0 + g * 4;
      float *to = S.out + at * S.ld + f;
      if (f < S.ld) *reinterpret_cast<f32x4 *>(to) = v[0];
      if (f + 16 < S.ld) *reinterpret_cast<f32x4 *>(to + 16) = v[1];
    }
  }
}

// ------------------------------------------------------ around the products --

// Rows of `in` [rows][ld_in], `cols` (a multiple of 4) of each, rounded under a power of two for each row: a wave a
// row, read twice (the second time from the caches).  Positions behind the last one kept are left out.  Bound by its
// bytes; 1166 rows of 368: 4 us, the launch.
__global__ __launch_bounds__(256) void scale_rows_kernel(const float *in, int64_t ld_in, int cols, f16_t *out,
                                                         uint8_t *exps, const int32_t *offsets, int experts) {
  const int64_t row = (int64_t)block_id() * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= offsets[experts]) return;
  const float *from = in + row * ld_in;
  float m = 0.f;
  for (int c = lane * 4; c < cols; c += 256) {
    float x[4];
    load_vec<float, 4>(from + c, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, finite(x[i]));
  }
  const int e = exponent(group_max<64>(m));
  for (int c = lane * 4; c < cols; c += 256) {
    float x[4];
    load_vec<float, 4>(from + c, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = scale_down(x[i], e);
    store_vec<f16_t, 4>(out + row * cols + c, x);
  }
  if (lane == 0) exps[row] = (uint8_t)e;
}

// The same for each column of an expert's rows.  A workgroup takes 64 columns (blockIdx.x) of an expert
// (blockIdx.y) and the blockIdx.z-th part of its rows; with more than one part their largest magnitudes come from a
// launch before (ROUND false), part [parts][experts][cols].  Bound by its bytes, where there are few rows by two
// rounds of loads (7 experts of about 170 rows, 1104 columns: 10 us, 256 threads 16).
constexpr int kColThreads = 1024;
template <bool ROUND>
__global__ __launch_bounds__(kColThreads) void scale_cols_kernel(const float *in, int cols, f16_t *out, uint8_t *exps,
                                                                 float *part, const int32_t *offsets) {
  constexpr int kRows = kColThreads / 16;
  __shared__ float most[kColThreads / 64][64];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 64 + x * 4, e = blockIdx.y;
  const int lo = offsets[e], hi = offsets[e + 1], parts = gridDim.z, each = (hi - lo + parts - 1) / parts;
  const int64_t from = lo + (int64_t)blockIdx.z * each, to = min(from + each, (int64_t)hi);
  float m[4] = {0.f, 0.f, 0.f, 0.f};
  if (!ROUND || parts == 1) {
    if (c < cols)
#pragma unroll 4
      for (int64_t r = from + y; r < to; r += kRows) {
        float v[4];
        load_vec<float, 4>(in + r * cols + c, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = fmaxf(m[i], finite(v[i]));
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // a wave holds four rows of threads
      m[i] = fmaxf(m[i], __shfl_xor(m[i], 16, 64));
      most[y >> 2][x * 4 + i] = fmaxf(m[i], __shfl_xor(m[i], 32, 64));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
      for (int k = 0; k < kColThreads / 64; ++k) m[i] = fmaxf(m[i], most[k][x * 4 + i]);
  } else if (c < cols) {
    for (int z = 0; z < parts; ++z) {
      float v[4];
      load_vec<float, 4>(part + ((int64_t)z * gridDim.y + e) * cols + c, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = fmaxf(m[i], v[i]);
    }
  }
  if (c >= cols) return;
  if constexpr (!ROUND) {
    if (y == 0) store_vec<float, 4>(part + ((int64_t)blockIdx.z * gridDim.y + e) * cols + c, m);
  } else {
    int by[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) by[i] = exponent(m[i]);
    if (y == 0 && blockIdx.z == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) exps[(int64_t)e * cols + c + i] = (uint8_t)by[i];
#pragma unroll 4
    for (int64_t r = from + y; r < to; r += kRows) {
      float v[4];
      load_vec<float, 4>(in + r * cols + c, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = scale_down(v[i], by[i]);
      store_vec<f16_t, 4>(out + r * cols + c, v);
    }
  }
}

// y_t = sum over the token's assignments of w o (weight null: of o; exps: of the rows that o was made from, where they
// were scaled), and the gradient of the weights from the feature tiles' sums.  Bound by the bytes of o: 8 entries a load.
// (65536 outputs of 4096: 247 us, 4.9 TB/s.)
template <typename T>
__global__ __launch_bounds__(256) void combine_kernel(Outputs o, const uint8_t *exps, const float *weight,
                                                      const int32_t *slot, int64_t n_tokens, int per_token, int H, T *y,
                                                      const float *dot, int nt, float *dweight) {
  const int64_t t = block_id();
  if (t >= n_tokens) return;
  const int32_t *sl = slot + t * per_token;
  if (dweight != nullptr && blockIdx.z == 0)
    for (int q = threadIdx.x; q < per_token; q += 256) {
      float v = 0.f;
      if (sl[q] >= 0)
        for (int i = 0; i < nt; ++i) v += dot[(int64_t)sl[q] * nt + i];
      dweight[t * per_token + q] = v;
    }
  const int c = (blockIdx.z * 256 + threadIdx.x) * 8;
  if (c >= H) return;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.f;
  for (int q = 0; q < per_token; ++q) {
    const int64_t a = sl[q];
    if (a < 0) continue;
    const float w = weight ? weight[t * per_token + q] : 1.f;
    float x[8];
    load_vec<float, 8>(o.out + a * o.ld + c, x);
    if constexpr (kScaled<T>) {
      const int e = exps[a];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = scale_up(x[i], e);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += w * x[i];
  }
  T *to = y + t * H + c;
  if (c + 8 <= H) {  // at any address: rows of an odd width
    vec<T, 8> w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (T)v[i];
    __builtin_memcpy(to, &w, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < H) to[i] = (T)v[i];
  }
}

// Copy of [n][rows][cols] with both inner extents padded by zeros (16-bit elements).  `halves`: the rows
// are two runs of rows / halves that are padded each.  Bound by its bytes: a workgroup makes kPadPieces pieces of
// 16 bytes of the copy in a row, whatever the width, four loads a thread on their way at once (216 MB: 38 us, 5.6 TB/s).
constexpr int kPadPieces = 1024;
__global__ __launch_bounds__(256) void pad_kernel(const uint16_t *in, int64_t ld, int rows, int cols, int halves,
                                                  uint16_t *out, int out_rows, int out_cols, int64_t n) {
  const int per = out_rows / halves, src = rows / halves, width = out_cols / 8;  // out_cols is a multiple of 8
  const int64_t pieces = n * out_rows * width, from = block_id() * (int64_t)kPadPieces;
  if (from >= pieces) return;
  const int64_t r0 = from / width, e0 = r0 / out_rows;
  const int y0 = (int)(r0 - e0 * out_rows), c0 = (int)(from - r0 * width);
  i16x8 v[4];
  int k[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t at = c0 + i * 256 + threadIdx.x, dr = at / (uint32_t)width, y = y0 + dr, de = y / (uint32_t)out_rows;
    const int row = (int)(y - de * out_rows), half = row >= per, x = row - half * per;
    k[i] = x < src ? (int)(at - dr * width) * 8 : cols;
    const int64_t e = min(e0 + (int64_t)de, n - 1);
    v[i] = piece_load(reinterpret_cast<const char *>(in + (e * rows + half * src + min(x, src - 1)) * ld), k[i], cols);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at = from + i * 256 + threadIdx.x;
    if (at < pieces) *reinterpret_cast<i16x8 *>(out + at * 8) = piece_shift(v[i], k[i], cols);
  }
}

inline int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// Where the parts of the workspace lie.  Copies of operands whose rows do not start on
// 16 bytes are made for the call.
struct Region {
  size_t x = 0, dy = 0, w1 = 0, w2 = 0;  // copies
  size_t act = 0;                         // s, or w s backwards [A][Fp]; scaled, backwards: [dg du w s] by columns [A][3 Fp]
  size_t out = 0;                         // o, or the rows of dx [A][Hp] float
  size_t dgu = 0;                         // [A][2 Fp]
  size_t wide = 0;                        // scaled: s, or [dg du w s], float [A][Fp] or [A][3 Fp]
  size_t exps = 0, col_exps = 0;          // and the exponents of rows [A] and of columns [E][3 Fp]
  size_t part = 0;                        // [parts][E][3 Fp] float
  size_t dot = 0;                         // [A][feature tiles]
  size_t total = 0;
};

bool on16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

constexpr int kMinFeatTile = 128;

// Parts that an expert's rows are taken in by scale_cols_kernel, of 512 in the mean.
int column_parts(const cfp_experts_desc &d) {
  return (int)std::min<int64_t>(64, std::max<int64_t>(1, d.n_tokens * d.k / (d.n_experts * (int64_t)512)));
}

Region region(const cfp_experts_desc &d, bool bwd, bool pad_x, bool pad_dy, bool pad_w1, bool pad_w2) {
  const size_t A = (size_t)d.n_tokens * d.k, Hp = up(d.hidden, 8), Fp = up(d.inner, 8), E = d.n_experts;
  Region r;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = up(off + bytes, 256);
    return at;
  };
  if (pad_x) r.x = take((size_t)d.n_tokens * Hp * 2);
  if (pad_dy) r.dy = take((size_t)d.n_tokens * Hp * 2);
  if (pad_w1) r.w1 = take(E * 2 * Fp * Hp * 2);
  if (pad_w2) r.w2 = take(E * d.hidden * Fp * 2);
  const bool scaled = d.dtype == CFP_DT_F16;
  r.act = take(A * Fp * (scaled && bwd ? 6 : 2));
  if (scaled) r.wide = take(A * Fp * (bwd ? 12 : 4)), r.exps = take(A);
  if (scaled && bwd) {
    r.col_exps = take(E * 3 * Fp);
    if (column_parts(d) > 1) r.part = take((size_t)column_parts(d) * E * 3 * Fp * 4);
  }
  r.out = take(A * Hp * 4);
  if (bwd) {
    r.dgu = take(A * 2 * Fp * 2);
    r.dot = take(A * ((d.inner + kMinFeatTile - 1) / kMinFeatTile) * 4);
  }
  r.total = off;
  return r;
}

bool pads_x(const cfp_experts_desc &d, const void *x, int64_t stride) {
  return d.hidden % 8 != 0 || !on16(x) || (stride % 8 != 0 && d.n_tokens > 1);
}
bool pads_w1(const cfp_experts_desc &d) { return d.hidden % 8 != 0 || d.inner % 8 != 0 || !on16(d.w1); }
bool pads_w2(const cfp_experts_desc &d) { return d.inner % 8 != 0 || !on16(d.w2); }

void pad(const void *in, int64_t ld, int64_t rows, int cols, int halves, void *out, int64_t out_rows, int out_cols,
         int64_t n, hipStream_t st) {
  const int64_t grid = (n * out_rows * (out_cols / 8) + kPadPieces - 1) / kPadPieces;
  pad_kernel<<<grid_of(grid), 256, 0, st>>>(static_cast<const uint16_t *>(in), ld, (int)rows, cols, halves,
                                   static_cast<uint16_t *>(out), (int)out_rows, out_cols, n);
}

// Workgroups of a product; for gradients of weights also how the dies share an expert's tiles (A.deal_rows).
template <int P, int BR, int BF>
int64_t workgroups(Args &A, int64_t n_assign) {
  constexpr int kFeatTile = P == kUp ? BF / 2 : BF;
  const int64_t nt = ((P == kUp ? A.F : A.n_feat) + kFeatTile - 1) / kFeatTile;
  if (P != kGradW1 && P != kGradW2) return nt * (n_assign / BR + std::min<int64_t>(A.experts, n_assign));
  int64_t grid = 0, best = 0;
  const int64_t nr = (A.n_row + BR - 1) / BR;
  for (int r = 1; r <= 8; r *= 2) {  // the fewest idle workgroups, then the squarest blocks
    const int64_t br = (nr + r - 1) / r, bf = (nt * r + 7) / 8, cost = br * bf * 1024 + br + bf;
    if (grid == 0 || cost < best) best = cost, A.deal_rows = r, grid = 8 * br * bf * A.experts;
  }
  return grid;
}

template <typename T, int P, int BR, int BF, int WR, int WF, int PER_CU>
hipError_t run_product(Args A, int64_t n_assign, hipStream_t st) {
  constexpr size_t lds = 2 * (BR + BF) * kStep * 2;
  const int64_t grid = workgroups<P, BR, BF>(A, n_assign);
  if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
  auto *kernel = product_kernel<T, P, BR, BF, WR, WF, PER_CU>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<grid_of(grid), WR * WF * 64, lds, st>>>(A);
  return hipGetLastError();
}

// Few tokens an expert: the products are bound by the weights' bytes.
bool few_tokens(int64_t n_assign, int experts) { return n_assign <= (int64_t)experts * 32 || n_assign <= 64; }

template <typename T, int P>
hipError_t few(const Args &A, int64_t n_assign, hipStream_t st) {
  const auto go = [&](auto nt) {
    constexpr int kTile = P == kUp ? 16 : 32;
    const int64_t tiles = ((P == kUp ? A.F : A.n_feat) + kTile - 1) / kTile;
    const int64_t grid = tiles * (n_assign / (16 * nt.value) + std::min<int64_t>(A.experts, n_assign));
    if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
    few_kernel<T, P, nt.value><<<grid_of(grid), kFewWaves * 64, 0, st>>>(A);
    return hipGetLastError();
  };
  return n_assign <= (int64_t)A.experts * 8 ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, 4>{});
}

// The tile of a product, rows x features: the one of least time by a model of it, as the tiles that a compute unit
// works through, and half of one more for the end, times a tile's fixed part and its stages.  Fitted to eleven
// training steps of 180 to 81 thousand assignments; the tile it picks takes 1.02 times the best one's time in the mean.
// (256 x 256 against 128 x 128 and 64 x 128: 32768 assignments of 8 experts, 2048 wide, 1408 inside, up 456, 522 and
// 577 us; 16384 of 32, 1024 wide, 512 inside, up 92, 75 and 74 us; 1860 of 16, 536 wide, 1184 inside, down 31, 20 and
// 17 us.)  p = dy W2 has no tile of 256 x 256, as its epilogue needs more registers than that leaves: 485 us where 128 x
// 128 took 340 in the first of these.
struct Tile {
  int rows, feats;
};
Tile tile_of(int p, const Args &A, int64_t n_assign) {
  const bool grad = p == kGradW1 || p == kGradW2;
  const double stages = (double)((grad ? n_assign / A.experts : A.K) + kStep - 1) / kStep;
  const auto time = [&](int br, int bf, int per_cu, double fixed, double stage) {
    const double nt = ((p == kUp ? 2 * (int64_t)A.F : (int64_t)A.n_feat) + bf - 1) / bf;
    const double nr = grad ? (double)((A.n_row + br - 1) / br) * A.experts  // else an expert's last tile is half full
                           : (double)n_assign / br + std::min<int64_t>(A.experts, n_assign) / 2;
    return std::max(1., nt * nr / (256 * per_cu) + .5) * (fixed + stages * stage);
  };
  const double t256 = p == kBackUp ? INFINITY : time(256, 256, 1, 18, 1.75), t128 = time(128, 128, 2, 5, 1.3),
               t64 = time(64, 128, 3, 4, 1.2);
  return t256 < std::min(t128, t64) ? Tile{256, 256} : t128 < t64 ? Tile{128, 128} : Tile{64, 128};
}

template <typename T, int P>
hipError_t product(const Args &A, int64_t n_assign, hipStream_t st) {
  const Tile t = tile_of(P, A, n_assign);
  if constexpr (P != kBackUp)
    if (t.rows == 256) return run_product<T, P, 256, 256, 2, 2, 1>(A, n_assign, st);
  if (t.rows == 128) return run_product<T, P, 128, 128, 2, 2, 2>(A, n_assign, st);
  return run_product<T, P, 64, 128, 2, 2, 3>(A, n_assign, st);
}

// The three products that follow from p = dy W2: in one launch of 64 x 128 tiles up to kTogether workgroups of it,
// else one by one in the tiles of each.  (Sum of the three against the one: 777 tokens to 7 of 12 experts, 1000 wide,
// 364 inside, 1352 workgroups, 48 and 28 us; 6000 to 2 of 8, 1024 wide, 512 inside, 3096, 129 and 111 us; 1024 to 2 of
// 16, 2048 wide, 512 inside, 6912, 75 and 69 us.  Above, tiles of 256 x 256 are worth more.)
constexpr int64_t kTogether = 8192;
template <typename T>
hipError_t gradients(Args dx, Args dw1, Args dw2, int64_t n_assign, hipStream_t st) {
  // a multiple of 8 each, as eight dies take workgroups in turn
  const int64_t n0 = n_assign > 0 ? up(workgroups<kBackDown, 64, 128>(dx, n_assign), 8) : 0;
  const int64_t n1 = workgroups<kGradW1, 64, 128>(dw1, n_assign), n2 = workgroups<kGradW2, 64, 128>(dw2, n_assign);
  if (n0 + n1 + n2 <= kTogether) {
    gradients_kernel<T><<<(unsigned)(n0 + n1 + n2), 256, 2 * (64 + 128) * kStep * 2, st>>>(dx, dw1, dw2, (uint32_t)n0,
                                                                                         (uint32_t)(n0 + n1));
    return hipGetLastError();
  }
  hipError_t e = hipSuccess;
  if (n_assign > 0) e = product<T, kBackDown>(dx, n_assign, st);
  if (e == hipSuccess) e = product<T, kGradW1>(dw1, n_assign, st);
  return e == hipSuccess ? product<T, kGradW2>(dw2, n_assign, st) : e;
}

Args base_args(const cfp_experts_desc &d) {
  Args A{};
  A.offsets = d.offsets, A.rows = d.rows, A.experts = d.n_experts;
  // a / k for 0 <= a < 2^31: with 2^c >= k, magic = ceil(2^(31 + c) / k) < 2^32 exceeds the quotient by less than
  // k / 2^(31 + c) relative to 1 / k, and a times that is below 1 / k
  int c = 0;
  while ((1 << c) < d.k) ++c;
  A.shift = 31 + c, A.magic = (uint32_t)((((uint64_t)1 << A.shift) + d.k - 1) / d.k);
  A.F = d.inner, A.Fp = (int)up(d.inner, 8), A.weight = d.weight;
  return A;
}

Outputs outputs_of(const cfp_experts_desc &d, const Region &r, uint8_t *ws) {
  return {reinterpret_cast<float *>(ws + r.out), up(d.hidden, 8)};
}

template <typename T>
hipError_t combine(const cfp_experts_desc &d, const Outputs &o, const uint8_t *exps, const float *weight, void *y,
                   const float *dot, int nt, float *dweight, hipStream_t st) {
  dim3 grid = grid_of(d.n_tokens);
  grid.z = (d.hidden + 2047) / 2048;
  combine_kernel<T><<<grid, 256, 0, st>>>(o, exps, weight, d.slot, d.n_tokens, d.k, d.hidden, static_cast<T *>(y), dot,
                                          nt, dweight);
  return hipGetLastError();
}

struct Laid {  // operands as the products take them
  const char *x, *dy, *w1, *w2;
  int64_t ld_x, ld_dy, Hp, Fp;
};

Laid lay_out(const cfp_experts_desc &d, const void *dy, int64_t dy_stride, const Region &r, bool px, bool pdy, bool pw1,
             bool pw2, uint8_t *ws, hipStream_t st) {
  const int Hp = (int)up(d.hidden, 8), Fp = (int)up(d.inner, 8);
  Laid L{static_cast<const char *>(d.x), static_cast<const char *>(dy), static_cast<const char *>(d.w1),
         static_cast<const char *>(d.w2), d.x_stride * 2, dy_stride * 2, Hp, Fp};
  if (px) {
    pad(d.x, d.x_stride, d.n_tokens, d.hidden, 1, ws + r.x, d.n_tokens, Hp, 1, st);
    L.x = reinterpret_cast<const char *>(ws + r.x), L.ld_x = Hp * 2;
  }
  if (pdy) {
    pad(dy, dy_stride, d.n_tokens, d.hidden, 1, ws + r.dy, d.n_tokens, Hp, 1, st);
    L.dy = reinterpret_cast<const char *>(ws + r.dy), L.ld_dy = Hp * 2;
  }
  if (pw1) {
    pad(d.w1, d.hidden, 2 * (int64_t)d.inner, d.hidden, 2, ws + r.w1, 2 * (int64_t)Fp, Hp, d.n_experts, st);
    L.w1 = reinterpret_cast<const char *>(ws + r.w1);
  }
  if (pw2) {
    pad(d.w2, d.inner, d.hidden, d.inner, 1, ws + r.w2, d.hidden, Fp, d.n_experts, st);
    L.w2 = reinterpret_cast<const char *>(ws + r.w2);
  }
  return L;
}

// The first `cols` of the ld entries of the wide rows, under a power of two for each row, to `out` [A][cols].
hipError_t scale_rows(const cfp_experts_desc &d, const Region &r, uint8_t *ws, int64_t ld, int64_t cols, void *out,
                      hipStream_t st) {
  scale_rows_kernel<<<grid_of((d.n_tokens * d.k + 3) / 4), 256, 0, st>>>(
      reinterpret_cast<const float *>(ws + r.wide), ld, (int)cols, static_cast<f16_t *>(out), ws + r.exps, d.offsets,
      d.n_experts);
  return hipGetLastError();
}

// All 3 Fp columns of the wide rows, under a power of two for each column of an expert, to r.act.
hipError_t scale_cols(const cfp_experts_desc &d, const Region &r, uint8_t *ws, int64_t cols, hipStream_t st) {
  const dim3 grid((unsigned)((cols + 63) / 64), d.n_experts, column_parts(d));
  const float *in = reinterpret_cast<const float *>(ws + r.wide);
  f16_t *out = reinterpret_cast<f16_t *>(ws + r.act);
  float *part = reinterpret_cast<float *>(ws + r.part);
  uint8_t *exps = ws + r.col_exps;
  if (grid.z > 1) scale_cols_kernel<false><<<grid, kColThreads, 0, st>>>(in, (int)cols, out, exps, part, d.offsets);
  scale_cols_kernel<true><<<grid, kColThreads, 0, st>>>(in, (int)cols, out, exps, part, d.offsets);
  return hipGetLastError();
}

template <typename T>
hipError_t forward(const cfp_experts_desc &d, void *y, float *h, uint8_t *ws, hipStream_t st) {
  const int64_t n = d.n_tokens * d.k;
  const bool small = few_tokens(n, d.n_experts);  // reads rows of any alignment in place
  const bool px = !small && pads_x(d, d.x, d.x_stride), pw1 = !small && pads_w1(d), pw2 = !small && pads_w2(d);
  const Region r = region(d, false, px, false, pw1, pw2);
  const Laid L = lay_out(d, nullptr, 0, r, px, false, pw1, pw2, ws, st);
  const int64_t H = small ? d.hidden : L.Hp, F = small ? d.inner : L.Fp;  // widths of the weights' rows
  Args A = base_args(d);
  A.row = L.x, A.ld_row = L.ld_x, A.feat = L.w1, A.ld_feat = H * 2, A.feat_expert = 2 * F * H * 2;
  A.K = (int)H, A.n_feat = d.inner, A.out = ws + (kScaled<T> ? r.wide : r.act), A.ld_out = L.Fp, A.h = h;
  hipError_t e = small ? few<T, kUp>(A, n, st) : product<T, kUp>(A, n, st);
  if (e == hipSuccess && kScaled<T>) e = scale_rows(d, r, ws, L.Fp, L.Fp, ws + r.act, st);
  if (e != hipSuccess) return e;
  A = base_args(d);
  A.row = reinterpret_cast<const char *>(ws + r.act), A.ld_row = L.Fp * 2;
  A.feat = L.w2, A.ld_feat = F * 2, A.feat_expert = (int64_t)d.hidden * F * 2;
  A.K = (int)F, A.n_feat = d.hidden, A.outputs = outputs_of(d, r, ws);
  if ((e = small ? few<T, kDown>(A, n, st) : product<T, kDown>(A, n, st)) != hipSuccess) return e;
  return combine<T>(d, A.outputs, ws + r.exps, d.weight, y, nullptr, 0, nullptr, st);
}

template <typename T>
hipError_t backward(const cfp_experts_desc &d, const void *dy, int64_t dy_stride, const float *h, void *dx, void *dw1,
                    void *dw2, float *dweight, uint8_t *ws, hipStream_t st) {
  const bool some = d.n_tokens > 0;  // without tokens only the gradients of the weights are written, with zeros
  const bool px = some && pads_x(d, d.x, d.x_stride), pdy = some && pads_x(d, dy, dy_stride);
  const bool pw1 = some && pads_w1(d), pw2 = some && pads_w2(d);
  const Region r = region(d, true, px, pdy, pw1, pw2);
  const Laid L = lay_out(d, dy, dy_stride, r, px, pdy, pw1, pw2, ws, st);
  const int64_t n = d.n_tokens * d.k;
  Args A = base_args(d);
  hipError_t e = hipSuccess;
  int dots = 0;
  if (n > 0) {
    // p = dy W2, and what follows from it
    A.row = L.dy, A.ld_row = L.ld_dy, A.feat = L.w2, A.ld_feat = L.Fp * 2, A.feat_expert = (int64_t)d.hidden * L.Fp * 2;
    A.K = d.hidden, A.n_feat = (int)L.Fp, A.h = const_cast<float *>(h);
    if constexpr (kScaled<T>) {
      A.out = ws + r.wide, A.ld_out = A.ld_out2 = 3 * L.Fp, A.out2 = ws + r.wide + 2 * L.Fp * sizeof(float);
    } else {
      A.out = ws + r.dgu, A.ld_out = 2 * L.Fp, A.out2 = ws + r.act, A.ld_out2 = L.Fp;
    }
    A.dot = reinterpret_cast<float *>(ws + r.dot);
    const int dot_tile = tile_of(kBackUp, A, n).feats;
    A.dot_tiles = dots = (int)((L.Fp + dot_tile - 1) / dot_tile);
    if ((e = product<T, kBackUp>(A, n, st)) != hipSuccess) return e;
    if constexpr (kScaled<T>) {
      if ((e = scale_rows(d, r, ws, 3 * L.Fp, 2 * L.Fp, ws + r.dgu, st)) != hipSuccess) return e;
      if ((e = scale_cols(d, r, ws, 3 * L.Fp, st)) != hipSuccess) return e;
    }
  }
  Args X = base_args(d);  // rows of dx
  X.row = reinterpret_cast<const char *>(ws + r.dgu), X.ld_row = 2 * L.Fp * 2;
  X.feat = L.w1, X.ld_feat = L.Hp * 2, X.feat_expert = 2 * L.Fp * L.Hp * 2;
  X.K = (int)(2 * L.Fp), X.n_feat = (int)L.Hp, X.outputs = outputs_of(d, r, ws);
  Args W1 = base_args(d), W2 = W1;  // dW1 = [dg du]^T x
  W1.row = reinterpret_cast<const char *>(ws + (kScaled<T> ? r.act : r.dgu)), W1.ld_row = (kScaled<T> ? 3 : 2) * L.Fp * 2;
  W1.exps = W2.exps = ws + r.col_exps, W1.n_row = (int)(2 * L.Fp);
  W1.feat = L.x, W1.ld_feat = L.ld_x, W1.n_feat = d.hidden, W1.out = dw1, W1.ld_out = d.hidden;
  // dW2 = dy^T (w s)
  W2.row = L.dy, W2.ld_row = L.ld_dy, W2.n_row = d.hidden;
  W2.feat = reinterpret_cast<const char *>(ws + r.act + (kScaled<T> ? 2 * L.Fp * 2 : 0));
  W2.ld_feat = (kScaled<T> ? 3 : 1) * L.Fp * 2, W2.n_feat = d.inner, W2.out = dw2;
  W2.ld_out = d.inner;
  if ((e = gradients<T>(X, W1, W2, n, st)) != hipSuccess || n == 0) return e;
  return combine<T>(d, outputs_of(d, r, ws), ws + r.exps, nullptr, dx,
                    reinterpret_cast<const float *>(ws + r.dot), dots, dweight, st);
}

}  // namespace

size_t experts_kept_bytes(const cfp_experts_desc &d) {
  // floor(first / 16) + e leaves each expert room for its last, partial block
  return ((size_t)d.n_tokens * d.k / 16 + d.n_experts) * ((d.inner + 15) / 16) * 512 * 4;
}

size_t experts_bytes(const cfp_experts_desc &d, bool bwd) {
  // dy is checked only when it is given: room for its copy is taken with x's
  const bool small = !bwd && few_tokens(d.n_tokens * d.k, d.n_experts), px = !small && pads_x(d, d.x, d.x_stride);
  return region(d, bwd, px || bwd, bwd, !small && pads_w1(d), !small && pads_w2(d)).total;
}

hipError_t launch_experts(const cfp_experts_desc &d, void *y, float *h, uint8_t *ws, hipStream_t st) {
  return d.dtype == CFP_DT_BF16 ? forward<bf16_t>(d, y, h, ws, st) : forward<f16_t>(d, y, h, ws, st);
}

hipError_t launch_experts_bwd(const cfp_experts_desc &d, const void *dy, int64_t dy_stride, const float *h, void *dx,
                              void *dw1, void *dw2, float *dweight, uint8_t *ws, hipStream_t st) {
  return d.dtype == CFP_DT_BF16 ? backward<bf16_t>(d, dy, dy_stride, h, dx, dw1, dw2, dweight, ws, st)
                                : backward<f16_t>(d, dy, dy_stride, h, dx, dw1, dw2, dweight, ws, st);
}

}  // namespace cfp
