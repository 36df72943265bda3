// Token loss (cross entropy) and the gradient of its sum. Per row x of V logits:
//   lse = log sum_v exp(x_v),  loss = w (lse - x_target),
//   dx  = w (exp(x - lse) - e_target).
// HBM-bound: a row is read once and its gradient written once.
//
// The sum is formed in one pass with a running maximum, in powers of two: with
// c = m log2(e) for the maximum m so far, s = sum 2^(x log2(e) - c), one fused
// multiply-add and one exponential a logit; sums of different references are joined
// by 2^(c - c'). c is rounded to fp32 and x log2(e) is not, so 2^(x log2(e) - c) at
// x = m is not 1 but off by up to half a unit in c's last place in the exponent: by 8 up
// to kNearLogit, where it takes no digits that count, by 64 at 1e9, by more than a float
// holds beyond. Rows whose maximum is beyond kNearLogit, or infinite, take a plain path
// that forms x - m first (slow_row, one CTA: 1 GB of bf16 with gradient where every row
// does, 2.9 ms for 50,000 classes and 9.8 ms for 100,096, instead of 0.33 ms); logits
// below -kNearLogit are held against that bound's reference, so that those met before a
// row's larger ones add what they are worth, which is nothing, and no infinity.
//
// k_loss: a row lies in the shared memory of a CTA, or in slices in that of the CTAs
// of a cluster. A thread copies its vectors to its own places and reads them there
// for the sum and for the gradient, and the CTAs exchange their (maximum, sum) once
// by stores that a barrier in shared memory counts. Two to four CTAs share a
// multiprocessor: the copies of some run while others compute. Measured: 0.86 to
// 0.94 of the copy rate with the gradient, from 8192 to 131,072 classes (0.81 where rows
// of bf16 do not start on 16 bytes), 0.76 for 200,001.
// k_loss_warp: rows of up to 4 KB, one a warp, held in registers (1000 fp32 classes:
// at the copy rate).
// k_loss_rows: rows too long for a cluster's shared memory are read twice, and once more
// for the gradient, an element a load (1,000,003 classes: 0.29 of the copy rate for the
// loss alone, 0.21 with the gradient).
//
// Rows need not start on 16 bytes (an odd V): vectors are those of the aligned
// addresses, and the elements before the first and after the last are handled one
// by one.
#include <algorithm>

#include "rows_dev.cuh"

using namespace eogp;

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNearLogit = 134217728.f;  // 2^27: c's last place is 16 at most

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Maximum m and s = sum 2^(x log2(e) - ref(m)) of some logits; m = -inf: none yet.
struct __align__(8) MaxSum {
  float m, s;
};
// The reference c, rounded: sums are joined right only if every use has the same value,
// so the product is kept from being fused with what follows.
__device__ __forceinline__ float ref(float m) { return fmaxf(__fmul_rn(m, kLog2e), -kNearLogit * kLog2e); }
// Over a warp: the maximum first, then one rescaling a lane and a plain sum.
__device__ __forceinline__ MaxSum warp_join(MaxSum v) {
  float m = v.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  return MaxSum{m, warp_sum(v.s * exp2_fast(ref(v.m) - ref(m)))};
}
// Over n entries of shared memory, in order.
__device__ __forceinline__ MaxSum join_all(const MaxSum* p, int n) {
  float m = p[0].m;
  for (int i = 1; i < n; ++i) m = fmaxf(m, p[i].m);
  const float c = ref(m);
  float s = 0.f;
  for (int i = 0; i < n; ++i) s += p[i].s * exp2_fast(ref(p[i].m) - c);
  return MaxSum{m, s};
}
// A new maximum of the logits that follow.
__device__ __forceinline__ void raise(MaxSum& v, float m) {
  if (m > v.m) {
    v.s *= exp2_fast(ref(v.m) - ref(m));
    v.m = m;
  }
}
// Whether the reference of this maximum does for a row.
__device__ __forceinline__ bool near(float m) { return fabsf(m) <= kNearLogit; }

// Which row r is, whether it takes part, its target and weight.
struct RowJob {
  int b, t;
  long long target;
  float w;
  bool kept;
};
// Its loads do not wait for each other.
__device__ __forceinline__ RowJob row_job(const LossArgs& a, int r, unsigned* status, bool flag) {
  RowJob j;
  locate(a.rs, r, j.b, j.t);
  const int len = a.rs.lengths ? a.rs.lengths[j.b] : a.rs.T;
  j.target = token_at(a.targets, j.b, j.t);
  j.w = a.weights ? a.weights[r] : 1.f;
  j.kept = j.t < len && j.target != a.ignore && j.w != 0.f;
  if (j.kept && (j.target < 0 || j.target >= a.V)) {
    if (flag) flag_status(status, EOGP_ST_DEVICE);
    j.kept = false;
  }
  return j;
}

__device__ __forceinline__ void put_loss(const LossArgs& a, int r, float loss, float lse) {
  a.loss[r] = loss;
  if (a.lse) a.lse[r] = lse;
}
// From the row's maximum and sum and its target's logit: c - x_target log2(e) is
// formed by one fused multiply-add, so small losses keep their digits.
__device__ __forceinline__ void put_loss(const LossArgs& a, int r, const RowJob& j, MaxSum v, float xt) {
  const float l2 = log2f(v.s), c = ref(v.m);
  put_loss(a, r, j.w * (kLn2 * (fmaf(-xt, kLog2e, c) + l2)), kLn2 * (c + l2));
}

// ------------------------------------------------------------------ any row, slowly
// One block on row r: maximum, sum and gradient in a pass each, every difference
// formed before it is scaled. NaN and +inf logits, and rows of -inf, give NaN.
constexpr int kSlowThreads = 512;

template <typename T>
__device__ __noinline__ void slow_row(const LossArgs& a, int r, const RowJob& j) {
  __shared__ float part[2][kSlowThreads / 32], xt;
  const int tid = threadIdx.x, nt = blockDim.x, nw = nt >> 5;
  const T* const x = row_of<T>(a.logits, j.b, j.t);
  if (tid == 0) xt = to_f32(x[j.target]);  // read before the gradient may be written over it
  float m = -INFINITY;
  for (int c = tid; c < a.V; c += nt) m = fmaxf(m, to_f32(x[c]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if ((tid & 31) == 0) part[0][tid >> 5] = m;
  __syncthreads();
  m = part[0][0];
  for (int w = 1; w < nw; ++w) m = fmaxf(m, part[0][w]);
  float s = 0.f;
  for (int c = tid; c < a.V; c += nt) s += exp2_fast((to_f32(x[c]) - m) * kLog2e);
  s = warp_sum(s);
  if ((tid & 31) == 0) part[1][tid >> 5] = s;
  __syncthreads();
  s = 0.f;
  for (int w = 0; w < nw; ++w) s += part[1][w];
  if (tid == 0) {
    const float ls = logf(s);
    put_loss(a, r, j.w * ((m - xt) + ls), m + ls);
  }
  if (!a.dlogits.p) return;
  T* const g = row_out<T>(a.dlogits, j.b, j.t);
  const float inv = j.w / s;
  for (int c = tid; c < a.V; c += nt) {
    float p = exp2_fast((to_f32(x[c]) - m) * kLog2e) * inv;
    if (c == j.target) p -= j.w;
    g[c] = from_f32<T>(p);
  }
}

template <typename T>
__global__ void __launch_bounds__(kSlowThreads) k_loss_rows(const LossArgs a, unsigned* status) {
  const int r = blockIdx.x;
  const RowJob j = row_job(a, r, status, threadIdx.x == 0);
  if (j.kept) return slow_row<T>(a, r, j);
  if (threadIdx.x == 0) put_loss(a, r, 0.f, 0.f);
  if (!a.dlogits.p) return;
  T* const g = row_out<T>(a.dlogits, j.b, j.t);
  for (int c = threadIdx.x; c < a.V; c += kSlowThreads) g[c] = from_f32<T>(0.f);
}

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

// 2^(x log2(e) - c) of a vector.
template <typename T, int N>
__device__ __forceinline__ Vals<N> exp_of(const Raw<T, N>& r, float c) {
  Vals<N> v = unpack<T, N>(r);
#pragma unroll
  for (int i = 0; i < Vals<N>::P; ++i) {
    const float2 d = fma2(v.p[i], pair(kLog2e), pair(-c));
    v.p[i] = make_float2(exp2_fast(d.x), exp2_fast(d.y));
  }
  return v;
}

// Adds K vectors to a thread's sum.
template <typename T, int N, int K>
__device__ __forceinline__ void add_vecs(MaxSum& v, const Raw<T, N> (&r)[K]) {
  float m = max_of<T, N>(r[0]);
#pragma unroll
  for (int k = 1; k < K; ++k) m = fmaxf(m, max_of<T, N>(r[k]));
  raise(v, m);
  const float c = ref(v.m);
  float2 s = pair(0.f);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const Vals<N> e = exp_of<T, N>(r[k], c);
#pragma unroll
    for (int i = 0; i < Vals<N>::P; ++i) s = add2(s, e.p[i]);
  }
  v.s += s.x + s.y;
}
__device__ __forceinline__ void add_one(MaxSum& v, float x) {
  raise(v, x);
  v.s += exp2_fast(fmaf(x, kLog2e, -ref(v.m)));
}

// Gradient of a vector that the target is not in: w 2^(x log2(e) - c) / s, inv = w / s.
template <typename T, int N>
__device__ __forceinline__ Vals<N> grad_of(const Raw<T, N>& r, float c, float inv) {
  Vals<N> v = exp_of<T, N>(r, c);
#pragma unroll
  for (int i = 0; i < Vals<N>::P; ++i) v.p[i] = mul2(v.p[i], pair(inv));
  return v;
}
__device__ __forceinline__ float grad_one(float x, int col, float c, float inv, float w, int target) {
  return exp2_fast(fmaf(x, kLog2e, -c)) * inv - (col == target ? w : 0.f);
}

// Zeros in the row: vectors v0 + tid, + nt, .. below v1, and its edge elements.
template <typename T>
__device__ __forceinline__ void zero_vecs(T* g, const RowVecs<T>& row, int v0, int v1, int tid, int nt, bool edges) {
  constexpr int N = RowVecs<T>::N;
  for (int i = v0 + tid; i < v1; i += nt) st_vals<T, N>(g + row.col(i), fill<N>(0.f));
  if (edges && row.edge(tid) >= 0) g[row.edge(tid)] = from_f32<T>(0.f);
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
      zero_vecs<T>(g, out, out.f0, out.f1, lane, 32, true);
    }
    if (lane == 0) put_loss(a, r, 0.f, 0.f);
    return;
  }
  const T* const x = row_of<T>(a.logits, j.b, j.t);
  const RowVecs<T> row(x, a.V);
  const float xt = to_f32(x[j.target]);
  Raw<T, N> raw[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = row.f0 + k * 32 + lane;
    raw[k] = pack_raw<T, N>(fill<N>(-INFINITY));
    if (i < row.f1) raw[k] = ld_raw<T, N>(x + row.col(i));
  }
  const int ce = row.edge(lane);
  const float xe = ce >= 0 ? to_f32(x[ce]) : -INFINITY;
  float m = xe;
#pragma unroll
  for (int k = 0; k < NV; ++k) m = fmaxf(m, max_of<T, N>(raw[k]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const bool fast = near(m);
  const float c = ref(m);
  // Where the reference does not do: differences first (rows of -inf: NaN).
  auto exps = [&](const Raw<T, N>& v) {
    if (fast) return exp_of<T, N>(v, c);
    Vals<N> e = unpack<T, N>(v);
#pragma unroll
    for (int i = 0; i < Vals<N>::P; ++i)
      e.p[i] = make_float2(exp2_fast((e.p[i].x - m) * kLog2e), exp2_fast((e.p[i].y - m) * kLog2e));
    return e;
  };
  auto exp_one = [&](float v) { return exp2_fast(fast ? fmaf(v, kLog2e, -c) : (v - m) * kLog2e); };
  float2 s2 = pair(0.f);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (row.f0 + k * 32 + lane < row.f1) {
      const Vals<N> e = exps(raw[k]);
#pragma unroll
      for (int i = 0; i < Vals<N>::P; ++i) s2 = add2(s2, e.p[i]);
    }
  }
  const float s = warp_sum(s2.x + s2.y + (ce >= 0 ? exp_one(xe) : 0.f));
  if (lane == 0) {
    if (fast) {
      put_loss(a, r, j, MaxSum{m, s}, xt);
    } else {
      const float ls = logf(s);
      put_loss(a, r, j.w * ((m - xt) + ls), m + ls);
    }
  }
  if (!g) return;
  __syncwarp();  // lane 0 has read the target's logit, which another lane may now write the gradient over
  const RowVecs<T> out(g, a.V);
  const float inv = j.w / s;
  const int target = static_cast<int>(j.target);
  if (ce >= 0) g[ce] = from_f32<T>(exp_one(xe) * inv - (ce == target ? j.w : 0.f));
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = row.f0 + k * 32 + lane, col = row.col(i);
    if (i >= row.f1) continue;
    Vals<N> d = exps(raw[k]);
#pragma unroll
    for (int e = 0; e < Vals<N>::P; ++e) d.p[e] = mul2(d.p[e], pair(inv));
    if (static_cast<unsigned>(target - col) < static_cast<unsigned>(N)) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (col + e == target) (e & 1 ? d.p[e / 2].y : d.p[e / 2].x) -= j.w;
    }
    if (out.ph == row.ph) {
      st_vals<T, N>(g + col, d);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) g[col + e] = from_f32<T>(e & 1 ? d.p[e / 2].y : d.p[e / 2].x);
    }
  }
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

// A cluster works on `rows` consecutive rows. The next row's target and weight are
// asked for at the start of a row, and its vectors follow each vector's last use
// into the same places, which a thread shares with no other. The first warp waits for
// the other CTAs' sums and tells the rest of its CTA, so that all threads go the same
// way. Where a wait runs out, the CTA takes no further part, lets its copies arrive and
// stays until no CTA of the cluster may store to it any more; the others' waits for it
// run out in turn.
template <typename T, bool GRAD>
__global__ void __launch_bounds__(kSliceThreads, 4) k_loss(const LossArgs a, int M, int rows, int per, int cs,
                                                           unsigned* status) {
  constexpr int N = 16 / sizeof(T), K = 4;
  extern __shared__ __align__(128) uint8_t smem[];  // 16 bytes off 32 cost 8 % (8192 classes of bf16)
  __shared__ MaxSum part[kSliceThreads / 32], peers[2][kMaxCluster], all;
  __shared__ bool lost;
  __shared__ uint64_t bar[2];
  __shared__ float target_logit;
  const int tid = threadIdx.x, nt = blockDim.x, nw = nt >> 5;
  const int rank = cs > 1 ? static_cast<int>(blockIdx.x % cs) : 0;
  const int r0 = static_cast<int>(blockIdx.x / cs) * rows, r1 = min(M, r0 + rows);
  const bool first = tid == 0 && rank == 0;
  Raw<T, N>* const slice = reinterpret_cast<Raw<T, N>*>(smem);
  if (cs > 1) {
    if (tid == 0) {
      mbar_init(&bar[0], 1);
      mbar_init(&bar[1], 1);
      fence_barrier_init();
      mbar_arrive_expect_tx(&bar[0], cs * sizeof(MaxSum));
      mbar_arrive_expect_tx(&bar[1], cs * sizeof(MaxSum));
    }
    __syncwarp();
    cluster_arrive();  // waited for before the first store to another CTA
  }
  bool met = cs == 1;
  int turn = 0;  // kept rows so far: exchanges alternate between two sets of slots

  // A row's part of this CTA.
  struct Part {
    RowJob j;
    RowVecs<T> row;
    const T* x;
    int v0, n;  // first vector and number of vectors of the slice; n = 0 for a row left out
  };
  auto part_of = [&](const RowJob& j) {
    const T* const x = row_of<T>(a.logits, j.b, j.t);
    const RowVecs<T> row(x, a.V);
    const int v0 = row.f0 + rank * per;
    return Part{j, row, x, v0, j.kept ? max(0, min(row.f1 - v0, per)) : 0};
  };
  auto ask = [&](const Part& p, int k) { copy_async<T, N>(slice + k, p.x + p.row.col(p.v0 + k)); };
  auto edge_of = [&](const Part& p) { return p.j.kept && rank == 0 ? p.row.edge(tid) : -1; };

  Part p = part_of(row_job(a, r0, status, first));
  for (int k = tid; k < p.n; k += nt) ask(p, k);
  int ce = edge_of(p);
  float xe = ce >= 0 ? to_f32(p.x[ce]) : 0.f;
  float xt = first && p.j.kept ? to_f32(p.x[p.j.target]) : 0.f;
  for (int r = r0; r < r1; ++r) {
    RowJob jn = p.j;
    jn.kept = false;
    if (r + 1 < r1) jn = row_job(a, r + 1, status, first);
    T* const g = GRAD ? row_out<T>(a.dlogits, p.j.b, p.j.t) : nullptr;
    if (!p.j.kept) {  // in every CTA of the cluster
      if (GRAD) {
        const RowVecs<T> out(g, a.V);
        const int v0 = out.f0 + rank * per;
        zero_vecs<T>(g, out, v0, min(out.f1, v0 + per), tid, nt, rank == 0);
      }
      if (first) put_loss(a, r, 0.f, 0.f);
      p = part_of(jn);
      for (int k = tid; k < p.n; k += nt) ask(p, k);
    } else {
      commit_async();
      wait_async<0>();
      MaxSum v{-INFINITY, 0.f};
      int k = tid;
      for (; k + (K - 1) * nt < p.n; k += K * nt) {
        Raw<T, N> w[K];
#pragma unroll
        for (int u = 0; u < K; ++u) w[u] = slice[k + u * nt];
        add_vecs<T, N, K>(v, w);
      }
      for (; k < p.n; k += nt) {
        const Raw<T, N> w[1] = {slice[k]};
        add_vecs<T, N, 1>(v, w);
      }
      if (ce >= 0) add_one(v, xe);
      const Part next = part_of(jn);
      if (!GRAD)
        for (int i = tid; i < next.n; i += nt) ask(next, i);
      v = warp_join(v);
      if ((tid & 31) == 0) part[tid >> 5] = v;
      // Read before this barrier, after which the gradient may be written over it.
      if (first) target_logit = xt;
      __syncthreads();
      v = join_all(part, nw);
      if (cs > 1) {
        const int set = turn & 1;
        if (!met) cluster_wait();  // every CTA of the cluster runs, its mbarriers set
        met = true;
        if (tid < 32) {
          if (tid < cs) put_peer(&peers[set][rank], &bar[set], tid, v);
          const bool came = __all_sync(0xffffffffu, mbar_wait_cluster(&bar[set], (turn >> 1) & 1, status));
          if (tid == 0) {
            lost = !came;
            if (came) {
              mbar_arrive_expect_tx(&bar[set], cs * sizeof(MaxSum));  // for the turn after next
              all = join_all(peers[set], cs);
            }
          }
        }
        __syncthreads();
        if (lost) break;
        v = all;
        ++turn;
      }
      if (!near(v.m)) {  // in every CTA of the cluster
        if (rank == 0) slow_row<T>(a, r, p.j);
        if (GRAD)
          for (int i = tid; i < next.n; i += nt) ask(next, i);
      } else {
        if (first) put_loss(a, r, p.j, v, target_logit);
        if (GRAD) {
          const RowVecs<T> out(g, a.V);
          const float inv = p.j.w / v.s, c = ref(v.m);
          const int target = static_cast<int>(p.j.target), col0 = p.row.col(p.v0);
          if (ce >= 0) g[ce] = from_f32<T>(grad_one(xe, ce, c, inv, p.j.w, target));
          // The thread that has the target's vector writes its element once more.
          const int kt = (target - col0) / N;
          const bool mine = target >= col0 && kt < p.n && kt % nt == tid;
          const float gt = mine ? grad_one(to_f32(reinterpret_cast<const T*>(smem)[target - col0]), target, c, inv,
                                           p.j.w, target) : 0.f;
          if (out.ph == p.row.ph) {
            T* o = g + col0 + tid * N;
            const int both = min(p.n, next.n);
            int i = tid;
#pragma unroll 4
            for (; i < both; i += nt, o += nt * N) {
              st_vals<T, N>(o, grad_of<T, N>(slice[i], c, inv));
              ask(next, i);
            }
#pragma unroll 4
            for (; i < p.n; i += nt, o += nt * N) st_vals<T, N>(o, grad_of<T, N>(slice[i], c, inv));
            for (; i < next.n; i += nt) ask(next, i);
            if (mine) g[target] = from_f32<T>(gt);
          } else {
            // dlogits lies otherwise to 16 bytes than logits: by way of shared memory,
            // an element a thread.
            for (int i = tid; i < p.n; i += nt)
              slice[i] = pack_raw<T, N>(grad_of<T, N>(slice[i], c, inv));
            if (mine) reinterpret_cast<T*>(smem)[target - col0] = from_f32<T>(gt);
            __syncthreads();
            const T* const from = reinterpret_cast<const T*>(smem);
            for (int i = tid; i < p.n * N; i += nt) g[col0 + i] = from[i];
            __syncthreads();
            for (int i = tid; i < next.n; i += nt) ask(next, i);
          }
        }
      }
      p = next;
      __syncthreads();  // `part` and target_logit have been read
    }
    ce = edge_of(p);
    xe = ce >= 0 ? to_f32(p.x[ce]) : 0.f;
    xt = first && p.j.kept ? to_f32(p.x[p.j.target]) : 0.f;
  }
  if (!met) cluster_wait();
  if (cs > 1 && met && lost) {
    commit_async();
    wait_async<0>();
    cluster_arrive();
    cluster_wait();  // for the threads of the cluster that have not ended
  }
}

// -------------------------------------------------------------------- launching
template <typename T, int NV>
cudaError_t loss_warp(const LossArgs& a, int M, unsigned* status, cudaStream_t st) {
  k_loss_warp<T, NV><<<(M + 3) / 4, 128, 0, st>>>(a, M, status);
  return cudaGetLastError();
}

// Rows of a cluster: as many as leave every multiprocessor about four sets of
// clusters to take in turn, eight at most.
int loss_rows(int M, int cs, int threads, int num_sms) {
  const long long resident = std::max(1ll, static_cast<long long>(num_sms) * (1024 / threads) / cs);
  return static_cast<int>(std::max(1ll, std::min(8ll, M / (4 * resident))));
}

template <typename T>
cudaError_t loss_launch(LossArgs a, unsigned* status, int num_sms, cudaStream_t st) {
  constexpr int N = 16 / sizeof(T);
  if (!a.rs.lengths && flat(a.logits, a.rs) && (!a.dlogits.p || flat(a.dlogits, a.rs)) && a.targets.bs == a.rs.T)
    a.rs = RowSet{1, static_cast<int>(a.rs.rows()), nullptr};
  const int M = static_cast<int>(a.rs.rows());
  const int nv = a.V / N;  // whole vectors of a row at most
  if (nv <= 32) return loss_warp<T, 1>(a, M, status, st);
  if (nv <= 64) return loss_warp<T, 2>(a, M, status, st);
  if (nv <= 128) return loss_warp<T, 4>(a, M, status, st);
  if (nv <= 256) return loss_warp<T, 8>(a, M, status, st);
  // Rows of up to 108 KB stay in one CTA, two of which share a multiprocessor; longer
  // ones are cut into slices of up to 56 KB (four CTAs). Measured, 1 GB of bf16
  // logits with gradient: 50,000 classes 328 us uncut and 338 us in two slices,
  // 131,072 classes 340 us in slices of up to 100 KB and 324 us in 56 KB.
  const long long bytes = nv * 16ll;
  int cs = 1;
  if (bytes > 108 * 1024)
    while (cs < kMaxCluster && bytes > 56 * 1024ll * cs) cs *= 2;
  // Few rows: spread over the multiprocessors.
  while (cs < kMaxCluster && static_cast<long long>(M) * cs * 2 <= num_sms && nv / cs >= 512) cs *= 2;
  const int per = (nv + cs - 1) / cs;
  const bool grad = a.dlogits.p != nullptr;
  const long long smem = per * 16ll;
  if (smem > 220 * 1024 || static_cast<long long>(M) * cs > 0x7FFFFFFFLL) {
    k_loss_rows<T><<<M, kSlowThreads, 0, st>>>(a, status);
    return cudaGetLastError();
  }
  // About 28 vectors a thread: what a thread does once a row weighs little beside
  // them (56 KB slices by 256 threads instead of 128: 412 us against 387 us for
  // 4 x 2048 rows of 100,096). Few rows: more threads, for their latency.
  const int each = static_cast<long long>(M) * cs < 2 * num_sms ? 12 : 28;
  const int threads = std::min(kSliceThreads, std::max(64, (per / each + 31) / 32 * 32));
  const int rows = loss_rows(M, cs, threads, num_sms);
  auto k = grad ? k_loss<T, true> : k_loss<T, false>;
  if (cudaError_t e = allow_smem(k, smem); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>((M + rows - 1) / rows) * cs);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cs;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cs > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k, a, M, rows, per, cs, status);
}

}  // namespace

cudaError_t launch_cross_entropy(const LossArgs& a, bool bf16_, unsigned* status, int num_sms, cudaStream_t st) {
  return bf16_ ? loss_launch<bf16>(a, status, num_sms, st) : loss_launch<float>(a, status, num_sms, st);
}
