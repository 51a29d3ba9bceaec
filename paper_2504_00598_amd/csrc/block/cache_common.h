// What the operators over a paged cache share: sequences, pages and the 8-bit floats.
#pragma once

#include "block_common.h"

namespace cfp {

struct SeqArgs {
  const int32_t *table, *starts, *lengths;
  int64_t table_stride, n_tokens;  // n_tokens: rows of the call
  int32_t n_seqs, width, page_shift;
  uint32_t n_pages;
};

inline SeqArgs seq_args(const cfp_cache_desc &c, const cfp_sequences_desc &s, int64_t n_tokens) {
  SeqArgs a{};
  a.table = s.table, a.starts = s.starts, a.lengths = s.lengths;
  a.table_stride = s.table_stride, a.n_tokens = n_tokens;
  a.n_seqs = s.n_seqs, a.width = s.width, a.n_pages = (uint32_t)c.n_pages;
  while ((1 << a.page_shift) < c.page) ++a.page_shift;
  return a;
}

// Rows of sequence b: first row, how many, and the token that the first one is.  What lies outside the call's rows
// is no sequence's.
struct Seq {
  int32_t row, n, pos;
};
__device__ __forceinline__ Seq seq_of(const SeqArgs &S, int b) {
  const int64_t from = S.starts[b], to = S.starts[b + 1];
  const int32_t length = S.lengths[b];
  Seq q;
  q.row = (int32_t)from;
  q.n = from >= 0 && to > from && to <= S.n_tokens ? (int32_t)(to - from) : 0;
  q.pos = max(length, 0) - q.n;
  return q;
}
__device__ __forceinline__ Seq seq_of_lane(const Seq &q, int lane) {
  return {__builtin_amdgcn_readlane(q.row, lane), __builtin_amdgcn_readlane(q.n, lane), __builtin_amdgcn_readlane(q.pos, lane)};
}

// The page of token p >= 0 of sequence b, and whether it is one of the cache's (else page 0).
__device__ __forceinline__ uint32_t page_of(const SeqArgs &S, int b, int p, bool &ok) {
  const int at = p >> S.page_shift;
  ok = at < S.width;
  const uint32_t pg = ok ? (uint32_t)S.table[b * S.table_stride + at] : 0u;
  ok = ok && pg < S.n_pages;
  return ok ? pg : 0u;
}

// Entries of a sequence's row of the table, read as constants (by scalar loads: the index is the same for all lanes).  They
// are loaded a tile or two before they are looked at.
typedef const __attribute__((address_space(4))) int32_t const_i32;
struct TableRow {
  const_i32 *row;
  int32_t last, shift;
  // Of the page that token p >= 0 lies in; of the last one for tokens behind the table, which no row sees.
  __device__ __forceinline__ uint32_t entry(int p) const { return (uint32_t)row[min(p >> shift, last)]; }
};
__device__ __forceinline__ TableRow table_row(const SeqArgs &S, int b) {  // of a sequence with tokens that fit its row
  return {reinterpret_cast<const_i32 *>(reinterpret_cast<uintptr_t>(S.table + b * S.table_stride)), S.width - 1, S.page_shift};
}

// Sums over the lanes up to this one.
__device__ __forceinline__ uint32_t lanes_before(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false);  // row_shr: 1, 2, 4, 8
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);  // row_bcast: 15 to rows 1 and 3
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);  // 31 to rows 2 and 3
  return v;
}

// Which sequence the unit `id` belongs to, and the how-manieth of its units it is, where a sequence q has units(q) of
// them in a row.  All 64 lanes of a wave call it; false where there is no such unit.
template <typename F>
__device__ __forceinline__ bool find_unit(const SeqArgs &S, uint32_t id, F units, int &b, uint32_t &k, Seq &q) {
  const int lane = threadIdx.x & 63;
  uint32_t before = 0;
  for (int first = 0; first < S.n_seqs; first += 64) {
    Seq s = {0, 0, 0};
    if (first + lane < S.n_seqs) s = seq_of(S, first + lane);
    const uint32_t own = first + lane < S.n_seqs ? units(s) : 0u;
    const uint32_t sum = lanes_before(own);
    const uint64_t past = __ballot(before + sum > id);
    if (past) {
      const int l = __builtin_ctzll(past);
      b = first + l;
      q = seq_of_lane(s, l);
      k = id - before - (uint32_t)__builtin_amdgcn_readlane((int)(sum - own), l);
      return true;
    }
    before += (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
  }
  return false;
}

// Units of the sequences before b.  All 64 lanes call it.
template <typename F>
__device__ __forceinline__ uint32_t units_before(const SeqArgs &S, int b, F units) {
  const int lane = threadIdx.x & 63;
  uint32_t before = 0;
  for (int first = 0; first < b; first += 64)
    before += (uint32_t)__builtin_amdgcn_readlane((int)lanes_before(first + lane < b ? units(seq_of(S, first + lane)) : 0u), 63);
  return before;
}

// 2^(scale - 127) of a scale from 1 to 254
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s << 23); }

hipError_t launch_cache_write(const cfp_cache_desc &c, const cfp_sequences_desc &s, int64_t n_tokens, int dtype, const void *k,
                              HeadStrides sk, const void *v, HeadStrides sv, hipStream_t st);
hipError_t launch_cache_read(const cfp_cache_desc &c, const cfp_sequences_desc &s, int64_t n_tokens, int dtype, void *k,
                             void *v, hipStream_t st);

// Whether the workgroups that join parts can be numbered.
bool attend_fits(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s);
size_t attend_bytes(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s);
hipError_t launch_attend(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s, void *out, float *lse,
                         void *ws, hipStream_t st);

}  // namespace cfp
