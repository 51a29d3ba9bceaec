// Exported C ABI of libcfp_block: argument checks and launches.  Every check is
// made on the host before the first HIP call.
#include "block_common.h"

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

}  // namespace
}  // namespace cfp

using namespace cfp;

#pragma GCC visibility push(default)
extern "C" {

int cfp_qk_norm_rope(const cfp_qk_desc *d, void *yq, void *yk, void *stream) {
  if (int e = check_qk(d)) return e;
  if (d->n_tokens == 0 || d->n_q + d->n_k == 0) return CFP_OK;
  if ((d->n_q && !yq) || (d->n_k && !yk)) return CFP_ERR_ARG;
  return status(launch_qk_fwd(*d, yq, yk, (hipStream_t)stream));
}

size_t cfp_qk_workspace_bytes(const cfp_qk_desc *d) {
  if (check_qk(d) || d->n_tokens == 0 || d->n_q + d->n_k == 0) return 0;
  return qk_bwd_bytes(*d);
}

int cfp_qk_norm_rope_bwd(const cfp_qk_desc *d, const void *dyq, int64_t dyq_token_stride, int64_t dyq_head_stride,
                         const void *dyk, int64_t dyk_token_stride, int64_t dyk_head_stride, void *dq, void *dk,
                         float *dwq, float *dwk, void *ws, size_t ws_bytes, void *stream) {
  if (int e = check_qk(d)) return e;
  const bool none = d->n_tokens == 0;
  if (!none && ((d->n_q && (!dyq || !dq)) || (d->n_k && (!dyk || !dk)))) return CFP_ERR_ARG;
  const size_t need = cfp_qk_workspace_bytes(d);
  if (need && (!ws || ws_bytes < need)) return CFP_ERR_WORKSPACE;
  if (need && !on(ws, 4)) return CFP_ERR_ARG;
  return status(launch_qk_bwd(*d, dyq, dyk, {dyq_token_stride, dyq_head_stride}, {dyk_token_stride, dyk_head_stride}, dq,
                              dk, dwq, dwk, (float *)ws, (hipStream_t)stream));
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

}  // extern "C"
#pragma GCC visibility pop
