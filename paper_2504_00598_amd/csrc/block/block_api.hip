// Exported C ABI of libcfp_block: argument checks and launches.  Every check is
// made on the host before the first HIP call.
#include <cmath>

#include "cache_common.h"

namespace cfp {
namespace {

constexpr int64_t kMaxTokens = (int64_t)1 << 31;  // counts of rows and of assignments stay below 2^31

bool dtype_ok(int t) { return t == CFP_DT_F32 || t == CFP_DT_F16 || t == CFP_DT_BF16; }

bool on(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

int status(hipError_t e) { return e == hipSuccess ? CFP_OK : CFP_ERR_HIP; }

int check_qk(const cfp_qk_desc *d) {
  if (!d || d->n_tokens < 0 || d->n_q < 0 || d->n_k < 0 || d->dim < 1 || d->rot < 0 || d->rot > d->dim || d->rot % 2 ||
      !dtype_ok(d->dtype) || !dtype_ok(d->wdtype) || !(d->eps >= 0.f) || d->n_pos < 0)
    return CFP_ERR_ARG;
  if (d->dim > CFP_QK_MAX_DIM || d->n_tokens * ((int64_t)d->n_q + d->n_k) >= kMaxTokens || d->n_tokens >= kMaxTokens)
    return CFP_ERR_UNSUPPORTED;
  if (d->n_tokens == 0 || d->n_q + d->n_k == 0) return CFP_OK;
  if ((d->n_q && !d->q) || (d->n_k && !d->k)) return CFP_ERR_ARG;
  if (d->rot && (!d->cos || !d->sin || (!d->pos && d->n_tokens > d->n_pos))) return CFP_ERR_ARG;
  return CFP_OK;
}

int check_axes(const cfp_qk_desc *d, const uint8_t *axis, int n_axes) {
  if (int e = check_qk(d)) return e;
  if (n_axes < 1 || (d->rot && !axis) || (d->n_tokens > 0 && d->rot && !d->pos)) return CFP_ERR_ARG;
  if (n_axes > CFP_QK_MAX_AXES) return CFP_ERR_UNSUPPORTED;
  for (int i = 0; i < d->rot / 2; ++i)
    if (axis[i] >= n_axes) return CFP_ERR_ARG;
  return CFP_OK;
}

int qk_fwd(const cfp_qk_desc &d, const uint8_t *axis, void *yq, void *yk, void *stream) {
  if (d.n_tokens == 0 || d.n_q + d.n_k == 0) return CFP_OK;
  if ((d.n_q && !yq) || (d.n_k && !yk)) return CFP_ERR_ARG;
  return status(launch_qk_fwd(d, d.rot ? axis : nullptr, yq, yk, (hipStream_t)stream));
}

int qk_bwd(const cfp_qk_desc &d, const uint8_t *axis, const void *dyq, HeadStrides sq, const void *dyk,
           HeadStrides sk, void *dq, void *dk, float *dwq, float *dwk, void *ws, size_t ws_bytes, void *stream) {
  const bool none = d.n_tokens == 0;
  if (!none && ((d.n_q && (!dyq || !dq)) || (d.n_k && (!dyk || !dk)))) return CFP_ERR_ARG;
  const size_t need = none || d.n_q + d.n_k == 0 ? 0 : qk_bwd_bytes(d);
  if (need && (!ws || ws_bytes < need)) return CFP_ERR_WORKSPACE;
  if (need && !on(ws, 4)) return CFP_ERR_ARG;
  return status(launch_qk_bwd(d, d.rot ? axis : nullptr, dyq, dyk, sq, sk, dq, dk, dwq, dwk, (float *)ws,
                              (hipStream_t)stream));
}

int check_route(const cfp_route_desc *d) {
  if (!d || d->n_tokens < 0 || d->n_experts < 1 || d->k < 1 || d->k > d->n_experts || d->groups < 1 ||
      d->top_groups < 1 || d->top_groups > d->groups || d->n_experts % d->groups || !dtype_ok(d->dtype) ||
      (d->score != CFP_SCORE_SOFTMAX && d->score != CFP_SCORE_SIGMOID) ||
      (d->group_score != CFP_GROUP_MAX && d->group_score != CFP_GROUP_TOP_TWO) ||
      (d->group_score == CFP_GROUP_TOP_TWO && d->groups > 1 && d->n_experts / d->groups < 2))
    return CFP_ERR_ARG;
  if (d->n_experts > CFP_ROUTE_MAX_EXPERTS || d->k > CFP_ROUTE_MAX_K || d->n_tokens * d->k >= kMaxTokens)
    return CFP_ERR_UNSUPPORTED;
  if (d->n_tokens > 0 && (!d->logits || (d->n_tokens > 1 && d->stride < d->n_experts))) return CFP_ERR_ARG;
  return CFP_OK;
}

int check_plan(const cfp_plan_desc *d) {
  if (!d || d->n_tokens < 0 || d->k < 1 || d->n_experts < 1 || d->first < 0) return CFP_ERR_ARG;
  if (d->n_experts > CFP_ROUTE_MAX_EXPERTS || d->k > CFP_EXPERTS_MAX_K || d->n_tokens >= kMaxTokens ||
      d->n_tokens * d->k >= kMaxTokens)
    return CFP_ERR_UNSUPPORTED;
  return d->n_tokens > 0 && !d->index ? CFP_ERR_ARG : CFP_OK;
}

int check_experts(const cfp_experts_desc *d) {
  if (!d || d->n_tokens < 0 || d->k < 1 || d->n_experts < 1 || d->hidden < 1 || d->inner < 1 ||
      (d->dtype != CFP_DT_F16 && d->dtype != CFP_DT_BF16))
    return CFP_ERR_ARG;
  if (d->n_experts > CFP_ROUTE_MAX_EXPERTS || d->k > CFP_EXPERTS_MAX_K || d->hidden > CFP_EXPERTS_MAX_DIM ||
      d->inner > CFP_EXPERTS_MAX_DIM || d->n_tokens >= kMaxTokens || d->n_tokens * d->k >= kMaxTokens)
    return CFP_ERR_UNSUPPORTED;
  if (!d->w1 || !d->w2 || !d->offsets) return CFP_ERR_ARG;
  if (d->n_tokens > 0 && (!d->x || !d->weight || !d->rows || !d->slot || (d->n_tokens > 1 && d->x_stride < d->hidden)))
    return CFP_ERR_ARG;
  return CFP_OK;
}

bool half_type(int t) { return t == CFP_DT_F16 || t == CFP_DT_BF16; }

int check_cache(const cfp_cache_desc *c) {
  if (!c || c->n_pages < 1 || c->page < 1 || c->heads < 1 || c->dim < 1 || !c->k || !c->v ||
      (!half_type(c->dtype) && c->dtype != CFP_DT_E4M3))
    return CFP_ERR_ARG;
  if (c->n_pages > 0x7fffffff || c->page < 16 || c->page > CFP_CACHE_MAX_PAGE || (c->page & (c->page - 1)) ||
      c->dim > CFP_CACHE_MAX_DIM || c->dim % 16 || (int64_t)c->heads * c->dim * c->page >= kMaxTokens)
    return CFP_ERR_UNSUPPORTED;
  const int64_t inner = (int64_t)c->heads * c->page * c->dim, scales = (int64_t)c->heads * c->page;
  const bool several = c->n_pages > 1;
  if (!on(c->k, 16) || !on(c->v, 16) || (several && (c->k_page_stride < inner || c->v_page_stride < inner ||
                                                      c->k_page_stride % 16 || c->v_page_stride % 16)))
    return CFP_ERR_ARG;
  if (c->dtype == CFP_DT_E4M3 &&
      (!c->k_scale || !c->v_scale || !on(c->k_scale, 16) || !on(c->v_scale, 16) ||
       (several && (c->k_scale_page_stride < scales || c->v_scale_page_stride < scales || c->k_scale_page_stride % 16 ||
                    c->v_scale_page_stride % 16))))
    return CFP_ERR_ARG;
  return CFP_OK;
}

int check_sequences(const cfp_sequences_desc *s, const cfp_cache_desc &c, int64_t n_tokens) {
  if (!s || s->n_seqs < 0 || s->width < 0 || n_tokens < 0 || s->max_new < 0) return CFP_ERR_ARG;
  if (n_tokens >= kMaxTokens || n_tokens * c.heads >= kMaxTokens || s->n_seqs > CFP_MAX_SEQUENCES || (int64_t)s->n_seqs * c.heads >= kMaxTokens / 16 ||
      (int64_t)s->width * c.page >= (int64_t)1 << 30)
    return CFP_ERR_UNSUPPORTED;
  if (s->n_seqs > 0 && n_tokens > 0 &&
      (!s->starts || !s->lengths || (s->width && !s->table) || (s->n_seqs > 1 && s->table_stride < s->width)))
    return CFP_ERR_ARG;
  return CFP_OK;
}

int check_rows(const cfp_cache_desc *c, const cfp_sequences_desc *s, int64_t n_tokens, int dtype) {
  if (int e = check_cache(c)) return e;
  if (int e = check_sequences(s, *c, n_tokens)) return e;
  if (!half_type(dtype)) return CFP_ERR_ARG;
  return c->dtype != CFP_DT_E4M3 && c->dtype != dtype ? CFP_ERR_UNSUPPORTED : CFP_OK;
}

int check_attend(const cfp_attend_desc *a, const cfp_cache_desc *c, const cfp_sequences_desc *s) {
  if (!a) return CFP_ERR_ARG;
  if (int e = check_rows(c, s, a->n_tokens, a->dtype)) return e;
  if (a->n_q < 1 || a->n_q % c->heads || !(a->scale > 0.f) || !std::isfinite(a->scale) || a->window < 0) return CFP_ERR_ARG;
  // a row's entries are counted in 32 bits where a workgroup's are
  if (a->n_tokens * a->n_q >= kMaxTokens || (int64_t)a->n_q * c->dim >= kMaxTokens ||
      a->n_tokens * (((int64_t)a->n_q * c->dim / 4 + 31) / 32) >= kMaxTokens)
    return CFP_ERR_UNSUPPORTED;
  if (!attend_fits(*a, *c, *s)) return CFP_ERR_UNSUPPORTED;
  return a->n_tokens > 0 && !a->q ? CFP_ERR_ARG : CFP_OK;
}

bool nothing(const cfp_sequences_desc &s, int64_t n_tokens) { return n_tokens == 0 || s.n_seqs == 0; }

}  // namespace
}  // namespace cfp

using namespace cfp;

#pragma GCC visibility push(default)
extern "C" {

int cfp_qk_norm_rope(const cfp_qk_desc *d, void *yq, void *yk, void *stream) {
  if (int e = check_qk(d)) return e;
  return qk_fwd(*d, nullptr, yq, yk, stream);
}

size_t cfp_qk_workspace_bytes(const cfp_qk_desc *d) {
  if (check_qk(d) || d->n_tokens == 0 || d->n_q + d->n_k == 0) return 0;
  return qk_bwd_bytes(*d);
}

int cfp_qk_norm_rope_bwd(const cfp_qk_desc *d, const void *dyq, int64_t dyq_token_stride, int64_t dyq_head_stride,
                         const void *dyk, int64_t dyk_token_stride, int64_t dyk_head_stride, void *dq, void *dk,
                         float *dwq, float *dwk, void *ws, size_t ws_bytes, void *stream) {
  if (int e = check_qk(d)) return e;
  return qk_bwd(*d, nullptr, dyq, {dyq_token_stride, dyq_head_stride}, dyk, {dyk_token_stride, dyk_head_stride}, dq, dk,
                dwq, dwk, ws, ws_bytes, stream);
}

int cfp_qk_norm_rope_axes(const cfp_qk_desc *d, const uint8_t *axis, int32_t n_axes, void *yq, void *yk, void *stream) {
  if (int e = check_axes(d, axis, n_axes)) return e;
  return qk_fwd(*d, axis, yq, yk, stream);
}

int cfp_qk_norm_rope_axes_bwd(const cfp_qk_desc *d, const uint8_t *axis, int32_t n_axes, const void *dyq,
                              int64_t dyq_token_stride, int64_t dyq_head_stride, const void *dyk, int64_t dyk_token_stride,
                              int64_t dyk_head_stride, void *dq, void *dk, float *dwq, float *dwk, void *ws,
                              size_t ws_bytes, void *stream) {
  if (int e = check_axes(d, axis, n_axes)) return e;
  return qk_bwd(*d, axis, dyq, {dyq_token_stride, dyq_head_stride}, dyk, {dyk_token_stride, dyk_head_stride}, dq, dk,
                dwq, dwk, ws, ws_bytes, stream);
}

int cfp_route(const cfp_route_desc *d, float *weight, int32_t *index, void *stream) {
  if (int e = check_route(d)) return e;
  if (d->n_tokens == 0) return CFP_OK;
  if (!weight || !index) return CFP_ERR_ARG;
  return status(launch_route(*d, weight, index, (hipStream_t)stream));
}

int cfp_route_bwd(const cfp_route_desc *d, const int32_t *index, const float *dweight, void *dlogits, void *stream) {
  if (int e = check_route(d)) return e;
  if (d->n_tokens == 0) return CFP_OK;
  if (!index || !dweight || !dlogits) return CFP_ERR_ARG;
  return status(launch_route_bwd(*d, index, dweight, dlogits, (hipStream_t)stream));
}

size_t cfp_expert_plan_workspace_bytes(const cfp_plan_desc *d) {
  return check_plan(d) ? 0 : plan_bytes(d->n_tokens * d->k, d->n_experts);
}

int cfp_expert_plan(const cfp_plan_desc *d, int32_t *offsets, int32_t *rows, int32_t *slot, void *ws, size_t ws_bytes,
                    void *stream) {
  if (int e = check_plan(d)) return e;
  if (!offsets || !rows || (d->n_tokens > 0 && !slot)) return CFP_ERR_ARG;
  const size_t need = plan_bytes(d->n_tokens * d->k, d->n_experts);
  if (need && (!ws || ws_bytes < need)) return CFP_ERR_WORKSPACE;
  if (need && !on(ws, 4)) return CFP_ERR_ARG;
  return status(launch_expert_plan(*d, offsets, rows, slot, (int32_t *)ws, (hipStream_t)stream));
}

size_t cfp_experts_kept_bytes(const cfp_experts_desc *d) {
  return check_experts(d) ? 0 : experts_kept_bytes(*d);
}

size_t cfp_experts_workspace_bytes(const cfp_experts_desc *d, int32_t backward) {
  return check_experts(d) ? 0 : experts_bytes(*d, backward != 0);
}

int cfp_experts(const cfp_experts_desc *d, void *y, void *kept, void *ws, size_t ws_bytes, void *stream) {
  if (int e = check_experts(d)) return e;
  if (d->n_tokens == 0) return CFP_OK;
  if (!y) return CFP_ERR_ARG;
  if (!ws || ws_bytes < experts_bytes(*d, false)) return CFP_ERR_WORKSPACE;
  if (!on(ws, 16) || !on(kept, 16)) return CFP_ERR_ARG;
  return status(launch_experts(*d, y, (float *)kept, (uint8_t *)ws, (hipStream_t)stream));
}

int cfp_experts_bwd(const cfp_experts_desc *d, const void *dy, int64_t dy_stride, const void *kept, void *dx, void *dw1,
                    void *dw2, float *dweight, void *ws, size_t ws_bytes, void *stream) {
  if (int e = check_experts(d)) return e;
  if (!dw1 || !dw2) return CFP_ERR_ARG;
  if (d->n_tokens > 0) {
    if (!dy || !kept || !dx || !dweight || (d->n_tokens > 1 && dy_stride < d->hidden)) return CFP_ERR_ARG;
    if (!ws || ws_bytes < experts_bytes(*d, true)) return CFP_ERR_WORKSPACE;
    if (!on(ws, 16) || !on(kept, 16)) return CFP_ERR_ARG;
  }
  return status(launch_experts_bwd(*d, dy, dy_stride, (const float *)kept, dx, dw1, dw2, dweight, (uint8_t *)ws,
                                   (hipStream_t)stream));
}

int cfp_cache_write(const cfp_cache_desc *c, const cfp_sequences_desc *s, int64_t n_tokens, int32_t dtype, const void *k,
                    int64_t k_token_stride, int64_t k_head_stride, const void *v, int64_t v_token_stride,
                    int64_t v_head_stride, void *stream) {
  if (int e = check_rows(c, s, n_tokens, dtype)) return e;
  if (nothing(*s, n_tokens)) return CFP_OK;
  if (!k || !v) return CFP_ERR_ARG;
  return status(launch_cache_write(*c, *s, n_tokens, dtype, k, {k_token_stride, k_head_stride}, v,
                                   {v_token_stride, v_head_stride}, (hipStream_t)stream));
}

int cfp_cache_read(const cfp_cache_desc *c, const cfp_sequences_desc *s, int64_t n_tokens, int32_t dtype, void *k, void *v,
                   void *stream) {
  if (int e = check_rows(c, s, n_tokens, dtype)) return e;
  if (nothing(*s, n_tokens)) return CFP_OK;
  if (!k || !v || !on(k, 16) || !on(v, 16)) return CFP_ERR_ARG;
  return status(launch_cache_read(*c, *s, n_tokens, dtype, k, v, (hipStream_t)stream));
}

size_t cfp_attend_workspace_bytes(const cfp_attend_desc *a, const cfp_cache_desc *c, const cfp_sequences_desc *s) {
  return check_attend(a, c, s) || nothing(*s, a->n_tokens) ? 0 : attend_bytes(*a, *c, *s);
}

int cfp_attend(const cfp_attend_desc *a, const cfp_cache_desc *c, const cfp_sequences_desc *s, void *out, float *lse, void *ws,
               size_t ws_bytes, void *stream) {
  if (int e = check_attend(a, c, s)) return e;
  if (nothing(*s, a->n_tokens)) return CFP_OK;
  if (!out || !on(out, 16)) return CFP_ERR_ARG;
  const size_t need = attend_bytes(*a, *c, *s);
  if (need && (!ws || ws_bytes < need)) return CFP_ERR_WORKSPACE;
  if (need && !on(ws, 16)) return CFP_ERR_ARG;
  return status(launch_attend(*a, *c, *s, out, lse, ws, (hipStream_t)stream));
}

}  // extern "C"
#pragma GCC visibility pop
