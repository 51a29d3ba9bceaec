// Helpers shared by the operators of a decoder block: 16-bit and 32-bit element
// types, vector loads and the launchers' declarations.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "cfp_block.h"

namespace cfp {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

template <typename T, int N>
using vec = T __attribute__((ext_vector_type(N)));

// N elements from memory aligned to N elements or 16 bytes, in pieces of up to 16 bytes.
template <typename T, int N>
__device__ __forceinline__ void load_vec(const T *p, float (&v)[N]) {
  constexpr int M = N * sizeof(T) > 16 ? 16 / (int)sizeof(T) : N;
#pragma unroll
  for (int j = 0; j < N; j += M) {
    const vec<T, M> x = *reinterpret_cast<const vec<T, M> *>(p + j);
#pragma unroll
    for (int i = 0; i < M; ++i) v[j + i] = (float)x[i];
  }
}

template <typename T, int N>
__device__ __forceinline__ void store_vec(T *p, const float (&v)[N]) {
  constexpr int M = N * sizeof(T) > 16 ? 16 / (int)sizeof(T) : N;
#pragma unroll
  for (int j = 0; j < N; j += M) {
    vec<T, M> x;
#pragma unroll
    for (int i = 0; i < M; ++i) x[i] = (T)v[j + i];
    *reinterpret_cast<vec<T, M> *>(p + j) = x;
  }
}

// op over aligned groups of G lanes; every lane gets the result.  Inside a row of 16 the
// other operand comes by data-parallel moves (quads, then mirrored halves and rows of what is
// already equal in them), beyond it by row swaps.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
template <int G, typename Op>
__device__ __forceinline__ uint32_t group_reduce(uint32_t v, Op op) {
  if constexpr (G > 1) v = op(v, moved<0xB1>(v));   // quad_perm [1, 0, 3, 2]
  if constexpr (G > 2) v = op(v, moved<0x4E>(v));   // quad_perm [2, 3, 0, 1]
  if constexpr (G > 4) v = op(v, moved<0x141>(v));  // row_half_mirror
  if constexpr (G > 8) v = op(v, moved<0x140>(v));  // row_mirror
  if constexpr (G > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = op(r[0], r[1]);
  }
  if constexpr (G > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = op(r[0], r[1]);
  }
  return v;
}

template <int G>
__device__ __forceinline__ float group_sum(float v) {
  return __uint_as_float(group_reduce<G>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}

template <int G>
__device__ __forceinline__ float group_max(float v) {
  return __uint_as_float(group_reduce<G>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}

template <int G>
__device__ __forceinline__ uint32_t group_umax(uint32_t v) {
  return group_reduce<G>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// n workgroups (below 2^31), numbered by block_id().  A launch of 2^32 threads or more in one dimension starts only
// some of them and reports no error, so they lie in rows of kGridRow; those behind the n-th have nothing to do.
constexpr int64_t kGridRow = 1 << 20;
inline dim3 grid_of(int64_t n) {
  return n <= kGridRow ? dim3((unsigned)n) : dim3((unsigned)kGridRow, (unsigned)((n + kGridRow - 1) / kGridRow));
}
__device__ __forceinline__ uint32_t block_id() { return blockIdx.y * gridDim.x + blockIdx.x; }

inline int elem_bytes(int dtype) { return dtype == CFP_DT_F32 ? 4 : 2; }

// Strides in elements of a [tokens][heads][dim] array whose last dimension is contiguous.
struct HeadStrides {
  int64_t tok, head;
};

// axis: that of each rotated pair, below CFP_QK_MAX_AXES, a row of d.pos [axes][n_tokens]; or NULL
hipError_t launch_qk_fwd(const cfp_qk_desc &d, const uint8_t *axis, void *yq, void *yk, hipStream_t st);
size_t qk_bwd_bytes(const cfp_qk_desc &d);
hipError_t launch_qk_bwd(const cfp_qk_desc &d, const uint8_t *axis, const void *dyq, const void *dyk,
                         HeadStrides sq, HeadStrides sk, void *dq, void *dk, float *dwq, float *dwk, float *part,
                         hipStream_t st);

hipError_t launch_route(const cfp_route_desc &d, float *weight, int32_t *index, hipStream_t st);
hipError_t launch_route_bwd(const cfp_route_desc &d, const int32_t *index, const float *dweight, void *dlogits,
                            hipStream_t st);

size_t plan_bytes(int64_t n_assign, int n_experts);
hipError_t launch_expert_plan(const cfp_plan_desc &d, int32_t *offsets, int32_t *rows, int32_t *slot, int32_t *scratch,
                              hipStream_t st);

size_t experts_kept_bytes(const cfp_experts_desc &d);
size_t experts_bytes(const cfp_experts_desc &d, bool backward);
hipError_t launch_experts(const cfp_experts_desc &d, void *y, float *h, uint8_t *ws, hipStream_t st);
hipError_t launch_experts_bwd(const cfp_experts_desc &d, const void *dy, int64_t dy_stride, const float *h, void *dx,
                              void *dw1, void *dw2, float *dweight, uint8_t *ws, hipStream_t st);

}  // namespace cfp
