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

// Sum and maximum over aligned groups of G lanes; every lane gets the result.
template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int off = G / 2; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

template <int G>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int off = G / 2; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
  return v;
}

inline int elem_bytes(int dtype) { return dtype == CFP_DT_F32 ? 4 : 2; }

// Strides in elements of a [tokens][heads][dim] array whose last dimension is contiguous.
struct HeadStrides {
  int64_t tok, head;
};

hipError_t launch_qk_fwd(const cfp_qk_desc &d, void *yq, void *yk, hipStream_t st);
size_t qk_bwd_bytes(const cfp_qk_desc &d);
hipError_t launch_qk_bwd(const cfp_qk_desc &d, const void *dyq, const void *dyk, HeadStrides sq, HeadStrides sk, void *dq,
                         void *dk, float *dwq, float *dwk, float *part, hipStream_t st);

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
