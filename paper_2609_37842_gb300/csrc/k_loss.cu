// Token loss (cross entropy) and the gradient of its sum. Per row x of V logits:
//   lse = log sum_v exp(x_v),  loss = w (lse - x_target),
//   dx  = w (exp(x - lse) - e_target).
// The sum is formed relative to a running maximum (exp never overflows), so the
// statistics take one pass; the gradient takes a second one.
#include "rows_dev.cuh"

using namespace eogp;

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;

// exp(x - m). The difference is formed before it is scaled: logits at the type's
// lowest value would overflow if they were scaled first.
__device__ __forceinline__ float exp_diff(float x, float m) { return exp2f((x - m) * kLog2e); }

// Maximum m and s = sum exp(x - m). A maximum of -inf stands for "nothing above
// -inf yet"; NaN and +inf stay in s.
struct MaxSum {
  float m, s;
};
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return MaxSum{m, a.s + b.s};
  return MaxSum{m, a.s * exp_diff(a.m, m) + b.s * exp_diff(b.m, m)};
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_loss_rows(LossArgs a, unsigned* status) {
  __shared__ MaxSum part[kWarps];
  const int r = blockIdx.x, b = r / a.rs.T, t = r - b * a.rs.T;
  T* gr = a.dlogits.p ? row_out<T>(a.dlogits, b, t) : nullptr;
  bool kept = row_kept(a.rs, b, t);
  long long tgt = -1;
  float w = 1.f;
  if (kept) {
    tgt = token_at(a.targets, b, t);
    if (a.weights) w = a.weights[r];
    kept = tgt != a.ignore && w != 0.f;
    if (kept && (tgt < 0 || tgt >= a.V)) {
      if (threadIdx.x == 0) flag_status(status, EOGP_ST_DEVICE);
      kept = false;
    }
  }
  if (!kept) {
    if (gr)
      for (int c = threadIdx.x; c < a.V; c += kThreads) gr[c] = from_f32<T>(0.f);
    if (threadIdx.x == 0) {
      a.loss[r] = 0.f;
      if (a.lse) a.lse[r] = 0.f;
    }
    return;
  }
  const T* xr = row_of<T>(a.logits, b, t);
  const float xt = to_f32(xr[tgt]);
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
  if (threadIdx.x == 0) {
    // A row of -inf has no softmax: NaN, as its terms exp(x - lse) are.
    const float ls = v.m == -INFINITY ? NAN : logf(v.s);
    a.loss[r] = w * ((v.m - xt) + ls);  // m - x_target first: exact where the target is the maximum
    if (a.lse) a.lse[r] = v.m + ls;
  }
  if (!gr) return;
  const float inv = w / v.s;
  for (int c = threadIdx.x; c < a.V; c += kThreads) {
    float p = exp_diff(to_f32(xr[c]), v.m) * inv;
    if (c == tgt) p -= w;
    gr[c] = from_f32<T>(p);
  }
}

}  // namespace

cudaError_t launch_cross_entropy(const LossArgs& a, bool bf16_, unsigned* status, int num_sms, cudaStream_t st) {
  const int M = static_cast<int>(a.rs.rows());
  if (bf16_)
    k_loss_rows<bf16><<<M, kThreads, 0, st>>>(a, status);
  else
    k_loss_rows<float><<<M, kThreads, 0, st>>>(a, status);
  return cudaGetLastError();
}
