// Attention over a paged cache: how a call is cut into parts, and its workspace.
#include <algorithm>

#include "attend.h"

namespace cfp {
namespace {

// Parts that the tokens of a sequence are cut into at most (a short one is cut into fewer on the device).
void parts_of(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s, AttendArgs &A) {
  const int64_t g = a.n_q / c.heads, most_len = (int64_t)s.width * c.page;
  const int64_t new_rows = std::min<int64_t>(s.max_new, a.n_tokens) * g;
  const int64_t pairs = (int64_t)s.n_seqs * c.heads;
  A.few_rows = (int32_t)std::min<int64_t>(kFewRows, new_rows);
  A.few_parts = (int32_t)std::clamp<int64_t>(std::min<int64_t>(2048 / pairs, most_len / kFewLeast), 1, 64);
  A.tiles = 0, A.many_parts = 1;
  if (new_rows > kFewRows) {
    A.tiles = (uint32_t)std::min<int64_t>(a.n_tokens * g / kManyRows + s.n_seqs, (a.n_tokens * g + kFewRows) / (kFewRows + 1));
    const int64_t groups = (int64_t)A.tiles * c.heads;
    if (groups < 512) A.many_parts = (int32_t)std::clamp<int64_t>(std::min<int64_t>(1024 / groups, most_len / kManyLeast), 1, 16);
  }
}

size_t few_floats(const cfp_cache_desc &c, const cfp_sequences_desc &s, const AttendArgs &A) {
  return A.few_parts > 1 ? (size_t)s.n_seqs * c.heads * A.few_parts * A.few_rows : 0;
}
size_t many_floats(const cfp_attend_desc &a, const AttendArgs &A) {
  return A.many_parts > 1 ? (size_t)a.n_tokens * a.n_q * A.many_parts : 0;
}

}  // namespace

size_t attend_bytes(const cfp_attend_desc &a, const cfp_cache_desc &c, const cfp_sequences_desc &s) {
  AttendArgs A{};
  parts_of(a, c, s, A);
  return (few_floats(c, s, A) + many_floats(a, A)) * (c.dim + 2) * 4;
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
  const size_t few = few_floats(c, s, A), many = many_floats(a, A);
  A.few_o = (float *)ws, A.many_o = A.few_o + few * c.dim;
  A.few_ml = A.many_o + many * c.dim, A.many_ml = A.few_ml + 2 * few;
  A.heads = c.heads, A.group = a.n_q / c.heads, A.dim = c.dim, A.max_new = s.max_new;
  A.causal = a.causal != 0, A.window = std::min(a.window, 1 << 30);
  A.wide = reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_token_stride % 8 == 0 && a.q_head_stride % 8 == 0;
  A.scale = a.scale * 1.44269504088896341f;
  return a.dtype == CFP_DT_F16 ? attend_f16(A, c.dtype == CFP_DT_E4M3, st) : attend_bf16(A, c.dtype == CFP_DT_E4M3, st);
}

}  // namespace cfp
