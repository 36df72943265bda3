// Distillation from a teacher's top logits and the gradient of the losses' sum. Per row
// x of V logits and list of classes j_k with the teacher's logits y_k, h the temperature:
//   p = softmax(x / h), q_k = exp(y_k / h - whole), whole the teacher's log-sum (given, or
//   the list's own),
//   loss = w sum q_k (log q_k - log p_jk),  dx = (w / h) (p - sum_k q_k e_jk);
// with a given log-sum the classes not listed are one more class on both sides,
//   q_r = max(0, 1 - sum q_k), p_r = sum of their p: loss += w q_r (log q_r - log p_r), and
//   dx = (w / h) p (1 - q_r / p_r) for them.
//
// Both parts of the classes have their own maximum, and so has the remainder's log p_r; with
// e = exp((x - m_r) / h) and s_r = sum e over the classes not listed, dx = (w / h) (p_r - q_r) e / s_r
// there, whatever the sizes: p_r is no difference, and may be too small for a float.
//
// k_distill_rows: one block on a row, in passes over global memory, every difference
// x - max formed before it is scaled.
#include <algorithm>

#include "rows_dev.cuh"

using namespace eogp;

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kListMax = EOGP_DISTILL_MAX;
constexpr int kThreads = 512;
constexpr int kSeen = 8192;
constexpr float kLowest = -3.402823466e38f;

// A row's list in shared memory.
struct List {
  int cls[kListMax];  // -1: no entry
  float q[kListMax];  // the teacher's probability
  float y[kListMax];  // its logarithm
  float x[kListMax];  // the student's logit
  bool first[kListMax];  // the first entry of its class
  unsigned seen[kSeen / 32];  // bit c % kSeen: a class like c is listed
  float sum;   // of q
  bool whole;  // all V classes are listed
};

struct Job {
  int b, t;
  float w;
  bool kept;
};
__device__ __forceinline__ Job job_of(const DistillArgs& a, int r) {
  Job j;
  locate(a.rs, r, j.b, j.t);
  j.w = a.weights ? a.weights[r] : 1.f;
  j.kept = row_kept(a.rs, j.b, j.t) && j.w != 0.f;
  return j;
}

__device__ __forceinline__ float log_term(float q, float log_q, float log_p) {
  return q > 0.f || q != q ? q * (log_q - log_p) : 0.f;
}

// One warp reads a row's list; false where there is nothing to learn from, or a class is out
// of range.
__device__ __forceinline__ bool read_list(const DistillArgs& a, const Job& j, int r, List& l, unsigned* status) {
  const int lane = threadIdx.x & 31;
  const long long c0 = j.b * a.classes.bs + j.t * a.classes.ld, y0 = j.b * a.teacher.bs + j.t * a.teacher.ld;
  const float inv_t = 1.f / a.temperature;
  float m = -INFINITY;
  bool bad = false, nan = false;
  for (int k = lane; k < a.K; k += 32) {
    const long long c = a.classes_i64 ? static_cast<const long long*>(a.classes.p)[c0 + k]
                                      : static_cast<const int*>(a.classes.p)[c0 + k];
    const float y = a.teacher_bf16 ? to_f32(static_cast<const bf16*>(a.teacher.p)[y0 + k])
                                   : static_cast<const float*>(a.teacher.p)[y0 + k];
    const bool there = c >= 0;
    bad |= there && c >= a.V;
    nan |= there && y != y;
    l.cls[k] = there && c < a.V ? static_cast<int>(c) : -1;
    l.y[k] = there ? y : -INFINITY;
    if (there) m = fmaxf(m, y);
  }
  if (__any_sync(0xffffffffu, bad)) {
    if (lane == 0) flag_status(status, EOGP_ST_DEVICE);
    return false;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  nan = __any_sync(0xffffffffu, nan);
  if (!a.teacher_lse && m == -INFINITY && !nan) return false;
  float log_s = 0.f;
  if (!a.teacher_lse) {
    float s = 0.f;
    for (int k = lane; k < a.K; k += 32) s += expf((l.y[k] - m) * inv_t);
    log_s = logf(warp_sum(s));
  }
  for (int k = lane; k < kSeen / 32; k += 32) l.seen[k] = 0u;
  __syncwarp();
  float sum = 0.f;
  int classes = 0;
  for (int k = lane; k < a.K; k += 32) {
    const int c = l.cls[k];
    const float log_q = a.teacher_lse ? l.y[k] * inv_t - a.teacher_lse[r] : (l.y[k] - m) * inv_t - log_s;
    const float q = c < 0 ? 0.f : expf(log_q);
    bool first = c >= 0;
    for (int i = 0; first && i < k; ++i) first = l.cls[i] != c;
    l.first[k] = first;
    classes += first;
    if (c >= 0) atomicOr(&l.seen[c % kSeen / 32], 1u << c % 32);
    l.y[k] = log_q;
    l.q[k] = q;
    sum += q;
  }
  sum = warp_sum(sum);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) classes += __shfl_xor_sync(0xffffffffu, classes, o);
  if (lane == 0) {
    l.sum = sum;
    l.whole = classes == a.V;
  }
  __syncwarp();
  return true;
}

// Whether a class is listed.
__device__ __forceinline__ bool listed(const List& l, int K, int c) {
  if (!(l.seen[c % kSeen / 32] >> c % 32 & 1u)) return false;
  for (int k = 0; k < K; ++k)
    if (l.cls[k] == c) return true;
  return false;
}

template <typename T>
__device__ __forceinline__ void no_row(const DistillArgs& a, const Job& j, int r, int tid, int nt) {
  if (tid == 0) {
    a.loss[r] = 0.f;
    if (a.lse) a.lse[r] = 0.f;
  }
  if (!a.dlogits.p) return;
  T* const g = row_out<T>(a.dlogits, j.b, j.t);
  for (int c = tid; c < a.V; c += nt) g[c] = from_f32<T>(0.f);
}

__device__ __forceinline__ float block_max(float m, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
  m = part[0];
  for (int w = 1; w < kThreads / 32; ++w) m = fmaxf(m, part[w]);
  return m;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_distill_rows(const DistillArgs a, unsigned* status) {
  __shared__ List l;
  __shared__ float part[2][kThreads / 32];
  __shared__ bool some;
  const int r = blockIdx.x, tid = threadIdx.x;
  const Job j = job_of(a, r);
  if (!j.kept) return no_row<T>(a, j, r, tid, kThreads);
  if (tid < 32) {
    const bool ok = read_list(a, j, r, l, status);
    if (tid == 0) some = ok;
  }
  __syncthreads();
  if (!some) return no_row<T>(a, j, r, tid, kThreads);
  const T* const x = row_of<T>(a.logits, j.b, j.t);
  const float inv_t = 1.f / a.temperature, f = kLog2e * inv_t;
  for (int k = tid; k < a.K; k += kThreads) l.x[k] = l.cls[k] < 0 ? 0.f : to_f32(x[l.cls[k]]);
  float m = kLowest;
  for (int c = tid; c < a.V; c += kThreads) {
    const float v = to_f32(x[c]);
    if (v > m && !listed(l, a.K, c)) m = v;
  }
  const float m_r = block_max(m, part[0]);
  float s = 0.f;
  for (int c = tid; c < a.V; c += kThreads)
    if (!listed(l, a.K, c)) s += exp2f((to_f32(x[c]) - m_r) * f);
  const float s_r = block_sum<kThreads / 32>(s, part[1]);
  m = kLowest;
  for (int k = tid; k < a.K; k += kThreads)
    if (l.cls[k] >= 0) m = fmaxf(m, l.x[k]);
  __syncthreads();
  m = fmaxf(block_max(m, part[0]), m_r);
  s = 0.f;
  for (int k = tid; k < a.K; k += kThreads)
    if (l.first[k]) s += exp2f((l.x[k] - m) * f);
  s = block_sum<kThreads / 32>(s, part[1]) + s_r * exp2f((m_r - m) * f);
  const float ls = s > 0.f ? logf(s) : NAN;
  const float log_pr = (m_r - m) * inv_t + (logf(s_r) - ls);
  const float q_r = a.teacher_lse && !l.whole ? fmaxf(0.f, 1.f - l.sum) : 0.f;
  float v = 0.f;
  for (int k = tid; k < a.K; k += kThreads)
    if (l.cls[k] >= 0) v += log_term(l.q[k], l.y[k], (l.x[k] - m) * inv_t - ls);
  __syncthreads();
  v = block_sum<kThreads / 32>(v, part[1]);
  if (tid == 0) {
    a.loss[r] = j.w * (v + log_term(q_r, logf(q_r), log_pr));
    if (a.lse) a.lse[r] = m * inv_t + ls;
  }
  if (!a.dlogits.p) return;
  T* const g = row_out<T>(a.dlogits, j.b, j.t);
  const float wt = j.w * inv_t;
  const float out = s_r > 0.f ? wt * (expf(log_pr) - q_r) / s_r : ls * 0.f;
  for (int c = tid; c < a.V; c += kThreads) {
    const float xc = to_f32(x[c]);
    float d;
    if (listed(l, a.K, c)) {
      float q = 0.f;
      for (int k = 0; k < a.K; ++k)
        if (l.cls[k] == c) q += l.q[k];
      d = wt * (expf((xc - m) * inv_t - ls) - q);
    } else {
      d = exp2f((xc - m_r) * f) * out;
    }
    g[c] = from_f32<T>(d);
  }
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, bool bf16_, unsigned* status, int num_sms, cudaStream_t st) {
  const unsigned M = static_cast<unsigned>(a.rs.rows());
  if (bf16_)
    k_distill_rows<bf16><<<M, kThreads, 0, st>>>(a, status);
  else
    k_distill_rows<float><<<M, kThreads, 0, st>>>(a, status);
  return cudaGetLastError();
}
