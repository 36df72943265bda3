// Device helpers of the model-end kernels (k_embed.cu, k_norm.cu, k_loss.cu, k_head.cu,
// k_head_tc.cu, k_distill.cu): element conversion, row addressing, exponentials and block-wide
// sums in a fixed order.
#pragma once

#include <cuda_bf16.h>

#include "eogp_dev.cuh"
#include "eogp_internal.h"

namespace eogp {

using bf16 = __nv_bfloat16;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLargest = 3.402823466e38f, kLowest = -kLargest;

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

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

// Example and token of row r; one example needs no division.
__device__ __forceinline__ void locate(const RowSet& rs, int r, int& b, int& t) {
  b = rs.B == 1 ? 0 : r / rs.T;
  t = r - b * rs.T;
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

// N contiguous elements as raw words: 16 bytes, two elements, or one.
template <typename T, int N>
struct Raw {
  uint4 w;
  static_assert(sizeof(T) * N == 16, "a vector is 16 bytes");
};
template <>
struct Raw<bf16, 2> {
  uint32_t w;
};
template <>
struct Raw<float, 2> {
  uint2 w;
};
template <typename T>
struct Raw<T, 1> {
  T w;
};

// Streaming load (global data that is read once).
template <typename T, int N>
__device__ __forceinline__ Raw<T, N> ld_raw(const T* p) {
  Raw<T, N> r;
  if constexpr (N == 1)
    r.w = *p;
  else
    r.w = __ldcs(reinterpret_cast<const decltype(r.w)*>(p));
  return r;
}

// The same for data that other blocks read again, through the read-only path.
template <typename T, int N>
__device__ __forceinline__ Raw<T, N> ld_keep(const T* p) {
  Raw<T, N> r;
  if constexpr (N == 1)
    r.w = *p;
  else
    r.w = __ldg(reinterpret_cast<const decltype(r.w)*>(p));
  return r;
}

// Asynchronous copy of N elements into shared memory; of two bytes, which have no
// such copy, a plain one.
template <typename T, int N>
__device__ __forceinline__ void copy_async(Raw<T, N>* dst, const T* src) {
  constexpr int B = N * sizeof(T);
  if constexpr (B == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
  else if constexpr (B >= 4)
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(dst)), "l"(src), "n"(B) : "memory");
  else
    dst->w = *src;
}
__device__ __forceinline__ void commit_async() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_async() {
  asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// The N values in fp32: pairs, for the paired instructions, or a single one.
template <int N>
struct Vals {
  using E = float2;
  static constexpr int P = N / 2;
  E p[P];
  __device__ __forceinline__ float get(int i) const { return i & 1 ? p[i / 2].y : p[i / 2].x; }
  __device__ __forceinline__ void set(int i, float x) { (i & 1 ? p[i / 2].y : p[i / 2].x) = x; }
  static __device__ __forceinline__ E all(float x) { return make_float2(x, x); }
};
template <>
struct Vals<1> {
  using E = float;
  static constexpr int P = 1;
  E p[P];
  __device__ __forceinline__ float get(int) const { return p[0]; }
  __device__ __forceinline__ void set(int, float x) { p[0] = x; }
  static __device__ __forceinline__ E all(float x) { return x; }
};

template <typename T, int N>
__device__ __forceinline__ Vals<N> unpack(const Raw<T, N>& r) {
  Vals<N> v;
  if constexpr (N == 1) {
    v.p[0] = to_f32(r.w);
  } else if constexpr (sizeof(T) == 4) {
    v.p[0] = make_float2(__uint_as_float(r.w.x), __uint_as_float(r.w.y));
    if constexpr (N == 4) v.p[1] = make_float2(__uint_as_float(r.w.z), __uint_as_float(r.w.w));
  } else {
    uint32_t u[N / 2];
    if constexpr (N == 2) {
      u[0] = r.w;
    } else {
      u[0] = r.w.x;
      u[1] = r.w.y;
      u[2] = r.w.z;
      u[3] = r.w.w;
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i)
      v.p[i] = make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
  }
  return v;
}

__device__ __forceinline__ uint32_t pack_bf16(float2 v) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// The values rounded to T, as raw words of 16 bytes.
template <typename T, int N>
__device__ __forceinline__ Raw<T, N> pack_raw(const Vals<N>& v) {
  Raw<T, N> r;
  if constexpr (sizeof(T) == 4)
    r.w = make_uint4(__float_as_uint(v.p[0].x), __float_as_uint(v.p[0].y), __float_as_uint(v.p[1].x),
                     __float_as_uint(v.p[1].y));
  else
    r.w = make_uint4(pack_bf16(v.p[0]), pack_bf16(v.p[1]), pack_bf16(v.p[2]), pack_bf16(v.p[3]));
  return r;
}

// Streaming store, rounded once to T.
template <typename T, int N>
__device__ __forceinline__ void st_vals(T* p, const Vals<N>& v) {
  if constexpr (N == 1) {
    *p = from_f32<T>(v.p[0]);
  } else if constexpr (sizeof(T) == 4) {
    if constexpr (N == 4)
      __stcs(reinterpret_cast<float4*>(p), make_float4(v.p[0].x, v.p[0].y, v.p[1].x, v.p[1].y));
    else
      __stcs(reinterpret_cast<float2*>(p), v.p[0]);
  } else if constexpr (N == 2) {
    __stcs(reinterpret_cast<unsigned*>(p), pack_bf16(v.p[0]));
  } else {
    __stcs(reinterpret_cast<uint4*>(p),
           make_uint4(pack_bf16(v.p[0]), pack_bf16(v.p[1]), pack_bf16(v.p[2]), pack_bf16(v.p[3])));
  }
}

// The same for a type whose N elements may take two accesses, or half of one.
template <typename G, int N>
__device__ __forceinline__ void st_wide(G* p, const Vals<N>& v) {
  if constexpr (sizeof(G) * N == 32) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(v.p[0].x, v.p[0].y, v.p[1].x, v.p[1].y));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v.p[2].x, v.p[2].y, v.p[3].x, v.p[3].y));
  } else if constexpr (sizeof(G) == 2 && N == 4) {
    __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack_bf16(v.p[0]), pack_bf16(v.p[1])));
  } else {
    st_vals<G, N>(p, v);
  }
}

// N floats, aligned to min(N, 4) of them.
template <int N>
__device__ __forceinline__ Vals<N> ld_floats(const float* p) {
  Vals<N> v;
  if constexpr (N == 1) {
    v.p[0] = *p;
  } else if constexpr (N == 2) {
    v.p[0] = *reinterpret_cast<const float2*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const float4 f = *(reinterpret_cast<const float4*>(p) + i);
      v.p[2 * i] = make_float2(f.x, f.y);
      v.p[2 * i + 1] = make_float2(f.z, f.w);
    }
  }
  return v;
}
template <int N>
__device__ __forceinline__ void st_floats(float* p, const Vals<N>& v) {
  if constexpr (N == 1) {
    *p = v.p[0];
  } else if constexpr (N == 2) {
    *reinterpret_cast<float2*>(p) = v.p[0];
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      *(reinterpret_cast<float4*>(p) + i) = make_float4(v.p[2 * i].x, v.p[2 * i].y, v.p[2 * i + 1].x, v.p[2 * i + 1].y);
  }
}

// N elements of G, as st_wide writes them.
template <typename G, int N>
__device__ __forceinline__ Vals<N> ld_wide(const G* p) {
  if constexpr (sizeof(G) == 4) {
    return ld_floats<N>(p);
  } else if constexpr (N == 4) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    Vals<4> v;
    v.p[0] = make_float2(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u));
    v.p[1] = make_float2(__uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
    return v;
  } else {
    return unpack<G, N>(*reinterpret_cast<const Raw<G, N>*>(p));
  }
}

template <int N>
__device__ __forceinline__ Vals<N> fill(float x) {
  Vals<N> v;
#pragma unroll
  for (int i = 0; i < Vals<N>::P; ++i) v.p[i] = Vals<N>::all(x);
  return v;
}

// N weights or biases from channel c on, of either type; `none` where p is NULL
// (N = 2: p and c aligned to two
// elements; N > 2: p to 16 bytes).
template <int N>
__device__ __forceinline__ Vals<N> ld_param(const void* p, bool is_bf16, int c, float none) {
  Vals<N> v;
  if (!p) {
    v = fill<N>(none);
  } else if constexpr (N == 1) {
    v.p[0] = param_at(p, is_bf16, c, none);
  } else if (is_bf16) {
    const bf16* q = static_cast<const bf16*>(p) + c;
    if constexpr (N == 8) {
      v = unpack<bf16, 8>(Raw<bf16, 8>{__ldg(reinterpret_cast<const uint4*>(q))});
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const uint32_t u = __ldg(reinterpret_cast<const unsigned*>(q) + i);
        v.p[i] = make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
      }
    }
  } else {
    const float* q = static_cast<const float*>(p) + c;
    if constexpr (N >= 4) {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        const float4 f = __ldg(reinterpret_cast<const float4*>(q) + i);
        v.p[2 * i] = make_float2(f.x, f.y);
        v.p[2 * i + 1] = make_float2(f.z, f.w);
      }
    } else {
      v.p[0] = __ldg(reinterpret_cast<const float2*>(q));
    }
  }
  return v;
}

__device__ __forceinline__ float2 pair(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float sum2(float2 a) { return a.x + a.y; }
__device__ __forceinline__ float add2(float a, float b) { return a + b; }
__device__ __forceinline__ float mul2(float a, float b) { return a * b; }
__device__ __forceinline__ float fma2(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float sum2(float a) { return a; }

}  // namespace eogp

// Elements per access (16 bytes, two elements or one) that base, strides and width
// of rows of es-byte elements allow.
inline int row_vec(const void* p, long long bs, long long ld, const RowSet& rs, long long n, int es) {
  for (int v = 16 / es; v > 1; v = v > 2 ? 2 : 1)
    if (reinterpret_cast<uintptr_t>(p) % (v * es) == 0 && n % v == 0 && (rs.B == 1 || bs % v == 0) &&
        (rs.T == 1 || ld % v == 0))
      return v;
  return 1;
}
inline int row_vec(const RowView& v, const RowSet& rs, long long n, int es) {
  return row_vec(v.p, v.bs, v.ld, rs, n, es);
}
// Whether example strides continue the token strides, so that B examples of T
// tokens are one run of rows.
inline bool flat(const RowView& v, const RowSet& rs) { return rs.B == 1 || v.bs == v.ld * rs.T; }

// Lets kernel k be launched with `bytes` of dynamic shared memory. The limit belongs to
// the process: calls of several host threads share it, so every call sets the same
// value, which none of them can need more than, and no thread takes from another what
// it has asked for. (227 KB a block, less up to 3 KB of static arrays.)
constexpr size_t kMostDynamicSmem = 224 * 1024;
constexpr size_t kFreeDynamicSmem = 40 * 1024;  // with the static part, below the 48 KB that need no asking
template <typename F>
cudaError_t allow_smem(F k, size_t bytes) {
  if (bytes <= kFreeDynamicSmem) return cudaSuccess;
  if (bytes > kMostDynamicSmem) return cudaErrorInvalidValue;
  return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMostDynamicSmem));
}
