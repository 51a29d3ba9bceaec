// Attention over a paged cache: how a call is cut into parts, and its workspace.
#include <algorithm>

#include "attend.h"

namespace cfp {
namespace {

// How the work is laid out: bounds from what the host knows; the device cuts by the lengths that it finds.  Sequences with few
// rows are cut into about kFewParts equal parts over all (512 workgroups are at work at a time).
void parts_of(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s, AttendArgs &A) {
  A.s = seq_args(c, s, a.n_tokens);
  A.heads = c.heads, A.group = a.n_q / c.heads, A.dim = c.dim;
  const int64_t g = A.group, most_len = (int64_t)s.width * c.page;
  const int64_t new_rows = std::min<int64_t>(s.max_new, a.n_tokens) * g;
  // all sequences have few rows, or those that have go with the narrow kernel and the others with the one for many
  A.few_rows = (int32_t)(new_rows <= kFewRows ? new_rows : g <= kTokenRows ? kTokenRows : kFewRows);
  A.few_least = A.few_rows <= kTokenRows ? kTokenLeast : kFewLeast;
  A.joined = most_len > A.few_least;
  A.few_target = (int32_t)std::max<int64_t>(kFewParts / c.heads, 1);
  A.few_units = s.n_seqs + (A.joined ? (int32_t)std::min<int64_t>(A.few_target, most_len / A.few_least * s.n_seqs) : 0);
  A.many_rows = c.dim <= kWideDim ? kWideRows : kManyRows;
  A.tiles = A.many_units = A.many_most = 0, A.many_joined = 0;
  if (new_rows > A.few_rows) {
    const int64_t rows = a.n_tokens * g;
    const int64_t most_span = a.causal && a.window > 0 ? std::min<int64_t>(most_len, a.window + A.many_rows / g + kManyStep) : most_len;
    A.tiles = (uint32_t)std::min<int64_t>(rows / A.many_rows + s.n_seqs, (rows + A.few_rows) / (A.few_rows + 1));
    // The device cuts tiles into parts where there are few, and where they see so much that parts may save something.  There are
    // these at least, if all rows are some sequence's:
    const int64_t least = std::max<int64_t>((rows - (int64_t)s.n_seqs * A.few_rows + A.many_rows - 1) / A.many_rows, 1);
    if (least * c.heads <= kManyRounds * kGroups + kSpare && most_span > 2 * kManyLeast + kManyStep) {
      const int64_t rounds = std::min<int64_t>(((int64_t)A.tiles * c.heads + kGroups - 1) / kGroups, kManyRounds);
      A.many_most = (uint32_t)std::min<int64_t>(rounds * kGroups / c.heads, A.tiles * ((most_len + kManyLeast - 1) / kManyLeast));
      A.many_joined = (int32_t)std::min<int64_t>(a.n_tokens * ((a.n_q * (int64_t)c.dim / 4 + kJoinThreads - 1) / kJoinThreads), 2048);
    }
    A.many_units = std::max(A.tiles, A.many_most);
  }
}

size_t few_slots(const cfp_cache_desc &c, const AttendArgs &A) {
  return A.joined ? (size_t)A.few_units * c.heads * A.few_rows : 0;
}
size_t many_slots(const cfp_cache_desc &c, const AttendArgs &A) { return (size_t)A.many_most * c.heads * A.many_rows; }
constexpr size_t kPlanBytes = 16;

}  // namespace

bool attend_fits(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s) {
  AttendArgs A{};
  parts_of(a, c, s, A);
  return joins_of(A) < (int64_t)1 << 31;
}

size_t attend_bytes(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s) {
  AttendArgs A{};
  parts_of(a, c, s, A);
  return (few_slots(c, A) + many_slots(c, A)) * (c.dim + 2) * 4 + (A.tiles ? kPlanBytes : 0);
}

hipError_t launch_attend(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s, void *out, float *lse,
                         void *ws, hipStream_t st) {
  AttendArgs A{};
  parts_of(a, c, s, A);
  A.q = a.q, A.k = c.k, A.v = c.v, A.ks = c.k_scale, A.vs = c.v_scale;
  A.kp = c.k_page_stride, A.vp = c.v_page_stride, A.ksp = c.k_scale_page_stride, A.vsp = c.v_scale_page_stride;
  A.qt = a.q_token_stride, A.qh = a.q_head_stride;
  A.out = out, A.lse = lse;
  const size_t few = few_slots(c, A), many = many_slots(c, A);
  A.plan = (int32_t *)ws;
  A.few_o = (float *)((char *)ws + (A.tiles ? kPlanBytes : 0)), A.many_o = A.few_o + few * c.dim;
  A.few_ml = A.many_o + many * c.dim, A.many_ml = A.few_ml + 2 * few;
  A.max_new = s.max_new;
  A.causal = a.causal != 0, A.window = std::min(a.window, 1 << 30);
  A.wide = reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_token_stride % 8 == 0 && a.q_head_stride % 8 == 0;
  A.scale = a.scale * 1.44269504088896341f;
  return a.dtype == CFP_DT_F16 ? attend_f16(A, c.dtype == CFP_DT_E4M3, st) : attend_bf16(A, c.dtype == CFP_DT_E4M3, st);
}

}  // namespace cfp
