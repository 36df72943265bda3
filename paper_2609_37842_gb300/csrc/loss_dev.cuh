// Device code that the losses on given logits share (k_loss.cu, k_distill.cu): sums of
// exponentials with a running maximum, the vectors of a row that need not start on 16 bytes, and
// the slices of a row by a cluster.
#pragma once

#include <algorithm>

#include "rows_dev.cuh"

namespace eogp {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNearLogit = 134217728.f;  // 2^27: c's last place is 16 at most

// Maximum m and s = sum 2^(x f - ref(m, f)) of some logits, f = log2(e) over the temperature;
// m = -inf: none yet.
struct __align__(8) MaxSum {
  float m, s;
};
// The reference c, rounded: sums are joined right only if every use has the same value,
// so the product is kept from being fused with what follows.
__device__ __forceinline__ float ref(float m, float f = kLog2e) {
  return fmaxf(__fmul_rn(m, f), -kNearLogit * kLog2e);
}
// Over a warp: the maximum first, then one rescaling a lane and a plain sum.
__device__ __forceinline__ MaxSum warp_join(MaxSum v, float f = kLog2e) {
  float m = v.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  return MaxSum{m, warp_sum(v.s * exp2_fast(ref(v.m, f) - ref(m, f)))};
}
// Over n entries of shared memory, in order.
__device__ __forceinline__ MaxSum join_all(const MaxSum* p, int n, float f = kLog2e) {
  float m = p[0].m;
  for (int i = 1; i < n; ++i) m = fmaxf(m, p[i].m);
  const float c = ref(m, f);
  float s = 0.f;
  for (int i = 0; i < n; ++i) s += p[i].s * exp2_fast(ref(p[i].m, f) - c);
  return MaxSum{m, s};
}
// A new maximum of the logits that follow.
__device__ __forceinline__ void raise(MaxSum& v, float m, float f = kLog2e) {
  if (m > v.m) {
    v.s *= exp2_fast(ref(v.m, f) - ref(m, f));
    v.m = m;
  }
}
// Whether the reference of this maximum does for a row.
__device__ __forceinline__ bool near(float m) { return fabsf(m) <= kNearLogit; }

// ---------------------------------------------------------------- vectors of a row
// Vector i of a row covers columns i * N - ph .. + N - 1, ph the elements between the
// last 16-byte boundary and the row's start; vectors [f0, f1) lie in the row, `head`
// elements before them and `tail` after.
template <typename T>
struct RowVecs {
  static constexpr int N = 16 / sizeof(T);
  int ph, f0, f1, head, tail;
  __device__ __forceinline__ RowVecs(const T* row, int V) {
    ph = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    f0 = ph > 0 ? 1 : 0;
    f1 = max(f0, (ph + V) / N);
    head = ph > 0 ? min(V, N - ph) : 0;
    tail = V - head - (f1 - f0) * N;
  }
  __device__ __forceinline__ int col(int i) const { return i * N - ph; }
  // Column of the edge element that thread `tid` has, -1 for none.
  __device__ __forceinline__ int edge(int tid) const {
    if (tid < head) return tid;
    if (tid >= N && tid - N < tail) return head + (f1 - f0) * N + tid - N;
    return -1;
  }
};

template <typename T, int N>
__device__ __forceinline__ float max_of(const Raw<T, N>& r) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t u[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
    __nv_bfloat162 m = *reinterpret_cast<const __nv_bfloat162*>(&u[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __hmax2(m, *reinterpret_cast<const __nv_bfloat162*>(&u[i]));
    return fmaxf(__low2float(m), __high2float(m));
  } else {
    return fmaxf(fmaxf(__uint_as_float(r.w.x), __uint_as_float(r.w.y)),
                 fmaxf(__uint_as_float(r.w.z), __uint_as_float(r.w.w)));
  }
}

// 2^(x f - c) of a vector.
template <typename T, int N>
__device__ __forceinline__ Vals<N> exp_of(const Raw<T, N>& r, float c, float f = kLog2e) {
  Vals<N> v = unpack<T, N>(r);
#pragma unroll
  for (int i = 0; i < Vals<N>::P; ++i) {
    const float2 d = fma2(v.p[i], pair(f), pair(-c));
    v.p[i] = make_float2(exp2_fast(d.x), exp2_fast(d.y));
  }
  return v;
}

// Adds K vectors to a thread's sum.
template <typename T, int N, int K>
__device__ __forceinline__ void add_vecs(MaxSum& v, const Raw<T, N> (&r)[K], float f = kLog2e) {
  float m = max_of<T, N>(r[0]);
#pragma unroll
  for (int k = 1; k < K; ++k) m = fmaxf(m, max_of<T, N>(r[k]));
  raise(v, m, f);
  const float c = ref(v.m, f);
  float2 s = pair(0.f);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const Vals<N> e = exp_of<T, N>(r[k], c, f);
#pragma unroll
    for (int i = 0; i < Vals<N>::P; ++i) s = add2(s, e.p[i]);
  }
  v.s += s.x + s.y;
}
__device__ __forceinline__ void add_one(MaxSum& v, float x, float f = kLog2e) {
  raise(v, x, f);
  v.s += exp2_fast(fmaf(x, f, -ref(v.m, f)));
}

// Gradient of a vector that no target is in: inv 2^(x f - c).
template <typename T, int N>
__device__ __forceinline__ Vals<N> grad_of(const Raw<T, N>& r, float c, float inv, float f = kLog2e) {
  Vals<N> v = exp_of<T, N>(r, c, f);
#pragma unroll
  for (int i = 0; i < Vals<N>::P; ++i) v.p[i] = mul2(v.p[i], pair(inv));
  return v;
}
// Zeros in the row: vectors v0 + tid, + nt, .. below v1, and its edge elements.
template <typename T>
__device__ __forceinline__ void zero_vecs(T* g, const RowVecs<T>& row, int v0, int v1, int tid, int nt, bool edges) {
  constexpr int N = RowVecs<T>::N;
  for (int i = v0 + tid; i < v1; i += nt) st_vals<T, N>(g + row.col(i), fill<N>(0.f));
  if (edges && row.edge(tid) >= 0) g[row.edge(tid)] = from_f32<T>(0.f);
}

// ----------------------------------------------------------------- slices of rows
constexpr int kSliceThreads = 256;  // most threads of a CTA
constexpr int kMaxCluster = 8;

// A store to CTA `rank` of the cluster that its mbarrier counts.
__device__ __forceinline__ void put_peer(const MaxSum* slot, const uint64_t* bar, int rank, MaxSum v) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(
                   mapa_shared(smem_u32(slot), rank)),
               "f"(v.m), "f"(v.s), "r"(mapa_shared(smem_u32(bar), rank))
               : "memory");
}

// Rows of a cluster: as many as leave every multiprocessor about four sets of
// clusters to take in turn, eight at most.
inline int loss_rows(int M, int cs, int threads, int num_sms) {
  const long long resident = std::max(1ll, static_cast<long long>(num_sms) * (1024 / threads) / cs);
  return static_cast<int>(std::max(1ll, std::min(8ll, M / (4 * resident))));
}

}  // namespace eogp
