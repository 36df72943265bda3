// Token loss (cross entropy) and the gradient of its sum. Per row x of V logits,
// with m = max x and s = sum_v exp(x_v - m):
//   lse = m + log s,  loss = w ((m - x_target) + log s),
//   dx  = w (exp(x - m) / s - e_target).
// HBM-bound: a row is read once and its gradient written once.
//
// k_loss: a row is cut into slices of up to about 56 KB, one for each CTA of a
// cluster. A thread copies its vectors of the slice to its own places of shared
// memory, reads them there for the maximum, for the sum and for the gradient, and
// the CTAs exchange their (maximum, sum) once through distributed shared memory.
// Four CTAs share a multiprocessor: the copies of some run while others compute.
// k_loss_warp: short rows, one a warp, held in registers.
// k_loss_rows: rows too long for a cluster's shared memory are read twice.
//
// Rows need not start on 16 bytes (an odd V): vectors are those of the aligned
// addresses, and the row's first and last vector are filled element by element,
// with -inf where they reach beyond the row.
#include <algorithm>

#include "rows_dev.cuh"

using namespace eogp;

namespace {

constexpr int kThreads = 512;  // k_loss_rows
constexpr int kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// exp(x - m). The difference is formed before it is scaled: logits at the type's
// lowest value would overflow if they were scaled first.
__device__ __forceinline__ float exp_diff(float x, float m) { return exp2_fast((x - m) * kLog2e); }

// Maximum m and s = sum exp(x - m). A maximum of -inf stands for "nothing above
// -inf yet"; NaN and +inf stay in s.
struct __align__(8) MaxSum {
  float m, s;
};
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return MaxSum{m, a.s + b.s};
  return MaxSum{m, a.s * exp_diff(a.m, m) + b.s * exp_diff(b.m, m)};
}

// Which row r is, whether it takes part, its target and weight.
struct RowJob {
  int b, t;
  long long target;
  float w;
  bool kept;
};
__device__ __forceinline__ RowJob row_job(const LossArgs& a, int r, unsigned* status, bool flag) {
  RowJob j;
  locate(a.rs, r, j.b, j.t);
  j.target = -1;
  j.w = 1.f;
  j.kept = row_kept(a.rs, j.b, j.t);
  if (j.kept) {
    j.target = token_at(a.targets, j.b, j.t);
    if (a.weights) j.w = a.weights[r];
    j.kept = j.target != a.ignore && j.w != 0.f;
    if (j.kept && (j.target < 0 || j.target >= a.V)) {
      if (flag) flag_status(status, EOGP_ST_DEVICE);
      j.kept = false;
    }
  }
  return j;
}

__device__ __forceinline__ void put_loss(const LossArgs& a, int r, const RowJob& j, MaxSum v, float xt) {
  float loss = 0.f, lse = 0.f;
  if (j.kept) {
    // A row of -inf has no softmax: NaN, as its terms exp(x - lse) are.
    const float ls = v.m == -INFINITY ? NAN : logf(v.s);
    loss = j.w * ((v.m - xt) + ls);  // m - x_target first: exact where the target is the maximum
    lse = v.m + ls;
  }
  a.loss[r] = loss;
  if (a.lse) a.lse[r] = lse;
}

// ------------------------------------------------------- rows too long for a cluster
// One block per row; the sum is formed relative to a running maximum, so the
// statistics take one pass and the gradient a second one.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_loss_rows(const LossArgs a, unsigned* status) {
  __shared__ MaxSum part[kWarps];
  const int r = blockIdx.x;
  const RowJob j = row_job(a, r, status, threadIdx.x == 0);
  T* gr = a.dlogits.p ? row_out<T>(a.dlogits, j.b, j.t) : nullptr;
  if (!j.kept) {
    if (gr)
      for (int c = threadIdx.x; c < a.V; c += kThreads) gr[c] = from_f32<T>(0.f);
    if (threadIdx.x == 0) put_loss(a, r, j, MaxSum{0.f, 1.f}, 0.f);
    return;
  }
  const T* xr = row_of<T>(a.logits, j.b, j.t);
  const float xt = to_f32(xr[j.target]);
  MaxSum v{-INFINITY, 0.f};
  for (int c = threadIdx.x; c < a.V; c += kThreads) {
    const float x = to_f32(xr[c]);
    if (x > v.m) {
      v.s = v.m == -INFINITY ? v.s : v.s * exp_diff(v.m, x);
      v.m = x;
    }
    if (x != -INFINITY) v.s += exp_diff(x, v.m);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    v = join(v, MaxSum{__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o)});
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = part[0];
  for (int i = 1; i < kWarps; ++i) v = join(v, part[i]);
  if (threadIdx.x == 0) put_loss(a, r, j, v, xt);
  if (!gr) return;
  const float inv = j.w / v.s;
  for (int c = threadIdx.x; c < a.V; c += kThreads) {
    float p = exp_diff(to_f32(xr[c]), v.m) * inv;
    if (c == j.target) p -= j.w;
    gr[c] = from_f32<T>(p);
  }
}

// ---------------------------------------------------------------- vectors of a row
// Vector i of a row covers columns i * N - ph .. + N - 1, ph the elements between the
// last 16-byte boundary and the row's start.
template <typename T>
struct RowVecs {
  static constexpr int N = 16 / sizeof(T);
  const T* x;
  int V, ph, count;
  __device__ __forceinline__ RowVecs(const T* row, int v)
      : x(row), V(v), ph(static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T))), count((ph + v + N - 1) / N) {}
  __device__ __forceinline__ int col(int i) const { return i * N - ph; }
  __device__ __forceinline__ bool full(int i) const { return col(i) >= 0 && col(i) + N <= V; }
  // The row's first or last vector, element by element.
  __device__ __forceinline__ Raw<T, N> edge(int i) const {
    Vals<N> v;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = col(i) + k;
      const float e = c >= 0 && c < V ? to_f32(x[c]) : -INFINITY;
      (k & 1 ? v.p[k / 2].y : v.p[k / 2].x) = e;
    }
    return pack_raw<T, N>(v);
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

// exp(x - m) of a vector.
template <typename T, int N>
__device__ __forceinline__ Vals<N> exp_of(const Raw<T, N>& r, float m) {
  Vals<N> v = unpack<T, N>(r);
#pragma unroll
  for (int i = 0; i < Vals<N>::P; ++i) {
    const float2 d = mul2(add2(v.p[i], pair(-m)), pair(kLog2e));
    v.p[i] = make_float2(exp2_fast(d.x), exp2_fast(d.y));
  }
  return v;
}

// Gradient of vector i: w (exp(x - m) / s - e_target), inv = w / s.
template <typename T, int N>
__device__ __forceinline__ Vals<N> grad_of(const Raw<T, N>& r, int col, float m, float inv, float w, int target) {
  Vals<N> v = exp_of<T, N>(r, m);
#pragma unroll
  for (int i = 0; i < Vals<N>::P; ++i) v.p[i] = mul2(v.p[i], pair(inv));
  if (static_cast<unsigned>(target - col) < static_cast<unsigned>(N)) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (col + i == target) (i & 1 ? v.p[i / 2].y : v.p[i / 2].x) -= w;
  }
  return v;
}

template <typename T, int N>
__device__ __forceinline__ void put_vec(T* g, const RowVecs<T>& row, int i, const Vals<N>& v) {
  const int c = row.col(i);
  if (row.full(i)) {
    st_vals<T, N>(g + c, v);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (c + k >= 0 && c + k < row.V) g[c + k] = from_f32<T>(k & 1 ? v.p[k / 2].y : v.p[k / 2].x);
  }
}

// ------------------------------------------------------------------- short rows
template <typename T, int NV>
__global__ void __launch_bounds__(128) k_loss_warp(const LossArgs a, int M, unsigned* status) {
  constexpr int N = 16 / sizeof(T);
  const int lane = threadIdx.x & 31, r = blockIdx.x * 4 + (threadIdx.x >> 5);
  if (r >= M) return;
  const RowJob j = row_job(a, r, status, lane == 0);
  T* const g = a.dlogits.p ? row_out<T>(a.dlogits, j.b, j.t) : nullptr;
  if (!j.kept) {
    if (g) {
      const RowVecs<T> out(g, a.V);
      for (int i = lane; i < out.count; i += 32) put_vec<T, N>(g, out, i, fill<N>(0.f));
    }
    if (lane == 0) put_loss(a, r, j, MaxSum{0.f, 1.f}, 0.f);
    return;
  }
  const T* const x = row_of<T>(a.logits, j.b, j.t);
  const RowVecs<T> row(x, a.V);
  const float xt = to_f32(x[j.target]);
  Raw<T, N> raw[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = k * 32 + lane;
    if (i >= row.count)
      raw[k] = pack_raw<T, N>(fill<N>(-INFINITY));
    else
      raw[k] = row.full(i) ? ld_raw<T, N>(x + row.col(i)) : row.edge(i);
  }
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < NV; ++k) m = fmaxf(m, max_of<T, N>(raw[k]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float at = m == -INFINITY ? 0.f : m;
  float2 s2 = pair(0.f);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const Vals<N> e = exp_of<T, N>(raw[k], at);
#pragma unroll
    for (int i = 0; i < Vals<N>::P; ++i) s2 = add2(s2, e.p[i]);
  }
  const MaxSum v{m, warp_sum(s2.x + s2.y)};
  if (lane == 0) put_loss(a, r, j, v, xt);
  if (!g) return;
  const RowVecs<T> out(g, a.V);
  const float inv = j.w / v.s;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = k * 32 + lane;
    if (i >= row.count) continue;
    const Vals<N> d = grad_of<T, N>(raw[k], row.col(i), m, inv, j.w, static_cast<int>(j.target));
    if (out.ph == row.ph) {
      put_vec<T, N>(g, out, i, d);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int c = row.col(i) + e;
        if (c >= 0 && c < a.V) g[c] = from_f32<T>(e & 1 ? d.p[e / 2].y : d.p[e / 2].x);
      }
    }
  }
}

// ----------------------------------------------------------------- slices of rows
constexpr int kSliceThreads = 256;  // most threads of a CTA
constexpr int kMaxCluster = 8;

template <typename T>
__global__ void __launch_bounds__(kSliceThreads, 4) k_loss(const LossArgs a, int per, int cs, unsigned* status) {
  constexpr int N = 16 / sizeof(T);
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float part[2][kSliceThreads / 32];
  __shared__ MaxSum peers[kMaxCluster];
  const int tid = threadIdx.x, nt = blockDim.x, nw = nt >> 5;
  const int r = blockIdx.x / cs, rank = blockIdx.x - r * cs;
  const RowJob j = row_job(a, r, status, tid == 0 && rank == 0);
  T* const g = a.dlogits.p ? row_out<T>(a.dlogits, j.b, j.t) : nullptr;
  const int v0 = rank * per;
  if (!j.kept) {  // all CTAs of the cluster
    if (g) {
      const RowVecs<T> out(g, a.V);
      const int end = rank == cs - 1 ? out.count : min(out.count, v0 + per);
      for (int i = v0 + tid; i < end; i += nt) put_vec<T, N>(g, out, i, fill<N>(0.f));
    }
    if (tid == 0 && rank == 0) put_loss(a, r, j, MaxSum{0.f, 1.f}, 0.f);
    return;
  }
  if (cs > 1) cluster_arrive();  // waited for before the first store to another CTA
  const T* const x = row_of<T>(a.logits, j.b, j.t);
  const RowVecs<T> row(x, a.V);
  const int n = max(0, min(row.count - v0, per));  // vectors of this slice
  Raw<T, N>* const slice = reinterpret_cast<Raw<T, N>*>(smem);
  for (int i = tid; i < n; i += nt) {
    if (row.full(v0 + i))
      copy_async<T, N>(slice + i, x + row.col(v0 + i));
    else
      slice[i] = row.edge(v0 + i);
  }
  commit_async();
  const float xt = tid == 0 && rank == 0 ? to_f32(x[j.target]) : 0.f;
  wait_async<0>();
  // Maximum and sum of the slice.
  float m = -INFINITY;
#pragma unroll 4
  for (int i = tid; i < n; i += nt) m = fmaxf(m, max_of<T, N>(slice[i]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if ((tid & 31) == 0) part[0][tid >> 5] = m;
  __syncthreads();
  m = part[0][0];
  for (int w = 1; w < nw; ++w) m = fmaxf(m, part[0][w]);
  const float at = m == -INFINITY ? 0.f : m;
  float2 s2 = pair(0.f);
#pragma unroll 2
  for (int i = tid; i < n; i += nt) {
    const Vals<N> e = exp_of<T, N>(slice[i], at);
#pragma unroll
    for (int k = 0; k < Vals<N>::P; ++k) s2 = add2(s2, e.p[k]);
  }
  const float ws = warp_sum(s2.x + s2.y);
  if ((tid & 31) == 0) part[1][tid >> 5] = ws;
  __syncthreads();
  MaxSum v{m, part[1][0]};
  for (int w = 1; w < nw; ++w) v.s += part[1][w];
  // Of the row.
  if (cs > 1) {
    cluster_wait();  // every CTA of the cluster runs
    if (tid < cs) {
      const uint32_t to = mapa_shared(smem_u32(&peers[rank]), tid);
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(v.m), "f"(v.s) : "memory");
    }
    cluster_sync_all();
    v = peers[0];
    for (int k = 1; k < cs; ++k) v = join(v, peers[k]);
  }
  if (tid == 0 && rank == 0) put_loss(a, r, j, v, xt);
  if (!g) return;
  const RowVecs<T> out(g, a.V);
  const float inv = j.w / v.s;
  const int target = static_cast<int>(j.target);
  if (out.ph == row.ph) {
#pragma unroll 2
    for (int i = tid; i < n; i += nt)
      put_vec<T, N>(g, out, v0 + i, grad_of<T, N>(slice[i], row.col(v0 + i), v.m, inv, j.w, target));
    return;
  }
  // dlogits lies otherwise to 16 bytes than logits: by way of shared memory, an
  // element a thread.
  for (int i = tid; i < n; i += nt)
    slice[i] = pack_raw<T, N>(grad_of<T, N>(slice[i], row.col(v0 + i), v.m, inv, j.w, target));
  __syncthreads();
  const T* const from = reinterpret_cast<const T*>(smem) - row.col(v0);
  const int c1 = min(a.V, row.col(v0 + n));
  for (int c = max(0, row.col(v0)) + tid; c < c1; c += nt) g[c] = from[c];
}

// -------------------------------------------------------------------- launching
template <typename T, int NV>
cudaError_t loss_warp(const LossArgs& a, int M, unsigned* status, cudaStream_t st) {
  k_loss_warp<T, NV><<<(M + 3) / 4, 128, 0, st>>>(a, M, status);
  return cudaGetLastError();
}

template <typename T>
cudaError_t loss_launch(const LossArgs& a, unsigned* status, int num_sms, cudaStream_t st) {
  constexpr int N = 16 / sizeof(T);
  const int M = static_cast<int>(a.rs.rows());
  const int nv = (a.V + 2 * N - 2) / N;  // vectors of a row, whatever its start
  if (nv <= 32) return loss_warp<T, 1>(a, M, status, st);
  if (nv <= 64) return loss_warp<T, 2>(a, M, status, st);
  if (nv <= 128) return loss_warp<T, 4>(a, M, status, st);
  if (nv <= 256) return loss_warp<T, 8>(a, M, status, st);
  int cs = 1;
  while (cs < kMaxCluster && (static_cast<long long>(nv) * 16 > 56 * 1024ll * cs)) cs *= 2;
  const int per = (nv + cs - 1) / cs, smem = per * 16;
  if (smem > 220 * 1024 || static_cast<long long>(M) * cs > 0x7FFFFFFFLL) {
    k_loss_rows<T><<<M, kThreads, 0, st>>>(a, status);
    return cudaGetLastError();
  }
  const int threads = std::min(kSliceThreads, std::max(64, (per / 6 + 31) / 32 * 32));
  if (smem > 40 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(k_loss<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(M) * cs);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cs;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cs > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k_loss<T>, a, per, cs, status);
}

}  // namespace

cudaError_t launch_cross_entropy(const LossArgs& a, bool bf16_, unsigned* status, int num_sms, cudaStream_t st) {
  return bf16_ ? loss_launch<bf16>(a, status, num_sms, st) : loss_launch<float>(a, status, num_sms, st);
}
