// Attention over a paged cache: how a call is cut into parts, and its workspace.
#include <algorithm>

#include "attend.h"

namespace cfp {
namespace {

// How the work is laid out: bounds from what the host knows; the device cuts by the lengths that it finds.  Sequences with few
// rows are cut into about kFewParts equal parts over all (512 workgroups are at work at a time).
void parts_of(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s, AttendArgs &A) {
  const int64_t g = a.n_q / c.heads, most_len = (int64_t)s.width * c.page;
  const int64_t new_rows = std::min<int64_t>(s.max_new, a.n_tokens) * g;
  // all sequences have few rows, or those that have go with the narrow kernel and the others with the one for many
  A.few_rows = (int32_t)(new_rows <= kFewRows ? new_rows : g <= kTokenRows ? kTokenRows : kFewRows);
  A.few_least = A.few_rows <= kTokenRows ? kTokenLeast : kFewLeast;
  A.joined = most_len > A.few_least;
  A.few_target = (int32_t)std::max<int64_t>(kFewParts / c.heads, 1);
  A.few_units = s.n_seqs + (A.joined ? (int32_t)std::min<int64_t>(A.few_target, most_len / A.few_least * s.n_seqs) : 0);
  A.many_rows = c.dim <= kWideDim ? kWideRows : kManyRows;
  A.tiles = 0, A.many_parts = 1;
  if (new_rows > A.few_rows) {
    A.tiles = (uint32_t)std::min<int64_t>(a.n_tokens * g / A.many_rows + s.n_seqs, (a.n_tokens * g + A.few_rows) / (A.few_rows + 1));
    // Time in tiles: rounds of the chip (a workgroup a compute unit; sixteen more are not counted as a round) times a
    // part's tiles and about five that a workgroup takes before its first and behind its last; a launch more joins the
    // parts (three).  The sequences are taken to be alike; as they may not be, one part stays where others save little.
    const int64_t each = a.n_tokens * g / s.n_seqs;
    const int64_t groups = c.heads * (each > A.few_rows ? s.n_seqs * ((each + A.many_rows - 1) / A.many_rows)
                                                        : (a.n_tokens * g + A.many_rows - 1) / A.many_rows);
    const int64_t most_tiles = (most_len + kManyStep - 1) / kManyStep;
    int64_t least = 0;
    for (int parts = 1; parts <= 64 && (parts == 1 || most_tiles * kManyStep >= (int64_t)parts * kManyLeast); ++parts) {
      const int64_t rounds = (std::max<int64_t>(groups * parts - 16, 1) + 255) / 256;
      const int64_t time = rounds * ((most_tiles + parts - 1) / parts + 5) + (parts > 1 ? 3 : 0);
      if (parts == 1)
        least = time * 7 / 8;
      else if (time < least)
        least = time, A.many_parts = parts;
    }
  }
}

size_t few_slots(const cfp_cache_desc &c, const AttendArgs &A) {
  return A.joined ? (size_t)A.few_units * c.heads * A.few_rows : 0;
}
size_t many_slots(const cfp_attend_desc &a, const AttendArgs &A) {
  return A.many_parts > 1 ? (size_t)a.n_tokens * a.n_q * A.many_parts : 0;
}

}  // namespace

size_t attend_bytes(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s) {
  AttendArgs A{};
  parts_of(a, c, s, A);
  return (few_slots(c, A) + many_slots(a, A)) * (c.dim + 2) * 4;
}

hipError_t launch_attend(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s, void *out, float *lse,
                         void *ws, hipStream_t st) {
  AttendArgs A{};
  parts_of(a, c, s, A);
  A.s = seq_args(c, s, a.n_tokens);
  A.q = a.q, A.k = c.k, A.v = c.v, A.ks = c.k_scale, A.vs = c.v_scale;
  A.kp = c.k_page_stride, A.vp = c.v_page_stride, A.ksp = c.k_scale_page_stride, A.vsp = c.v_scale_page_stride;
  A.qt = a.q_token_stride, A.qh = a.q_head_stride;
  A.out = out, A.lse = lse;
  const size_t few = few_slots(c, A), many = many_slots(a, A);
  A.few_o = (float *)ws, A.many_o = A.few_o + few * c.dim;
  A.few_ml = A.many_o + many * c.dim, A.many_ml = A.few_ml + 2 * few;
  A.heads = c.heads, A.group = a.n_q / c.heads, A.dim = c.dim, A.max_new = s.max_new;
  A.causal = a.causal != 0, A.window = std::min(a.window, 1 << 30);
  A.wide = reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_token_stride % 8 == 0 && a.q_head_stride % 8 == 0;
  A.scale = a.scale * 1.44269504088896341f;
  return a.dtype == CFP_DT_F16 ? attend_f16(A, c.dtype == CFP_DT_E4M3, st) : attend_bf16(A, c.dtype == CFP_DT_E4M3, st);
}

}  // namespace cfp
