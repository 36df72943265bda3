// Device helpers of the model-end kernels (k_embed.cu, k_norm.cu, k_loss.cu):
// element conversion, row addressing and block-wide sums in a fixed order.
#pragma once

#include <cuda_bf16.h>

#include "eogp_dev.cuh"
#include "eogp_internal.h"

namespace eogp {

using bf16 = __nv_bfloat16;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 from_f32<bf16>(float v) { return __float2bfloat16_rn(v); }

// A weight or bias of either type; NULL reads as `none`.
__device__ __forceinline__ float param_at(const void* p, bool is_bf16, int c, float none) {
  if (!p) return none;
  return is_bf16 ? to_f32(static_cast<const bf16*>(p)[c]) : static_cast<const float*>(p)[c];
}

template <typename T>
__device__ __forceinline__ const T* row_of(const RowView& v, int b, int t) {
  return static_cast<const T*>(v.p) + b * v.bs + t * v.ld;
}
template <typename T>
__device__ __forceinline__ T* row_out(const RowView& v, int b, int t) {
  return const_cast<T*>(static_cast<const T*>(v.p)) + b * v.bs + t * v.ld;
}

__device__ __forceinline__ long long token_at(const TokenView& v, int b, int t) {
  return v.i64 ? static_cast<const long long*>(v.p)[b * v.bs + t] : static_cast<const int*>(v.p)[b * v.bs + t];
}

__device__ __forceinline__ bool row_kept(const RowSet& rs, int b, int t) {
  return !rs.lengths || t < rs.lengths[b];
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over the block, the same in every thread. `part` has NW floats; the
// caller keeps a __syncthreads between two uses of the same `part`.
template <int NW>
__device__ __forceinline__ float block_sum(float v, float* part) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) s += part[w];
  return s;
}

}  // namespace eogp
