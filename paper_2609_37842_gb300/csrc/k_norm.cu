// Normalisation over the channels of each row (layer norm and RMS norm) and its
// gradient. With mu = mean(x) (0 for RMS), r = (mean((x - mu)^2) + eps)^(-1/2),
// xh = (x - mu) r:
//   y  = xh w + b,
//   dx = r (g - mean(g) - xh mean(g xh)),  g = dy w  (RMS: no mean(g)),
//   dw = sum over tokens of dy xh,  db = sum over tokens of dy.
// Statistics and sums are fp32; the variance is the mean of squared differences
// from the mean, not a difference of moments. HBM-bound: a few flop per byte.
#include "rows_dev.cuh"

using namespace eogp;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// One block per row, three passes over the row (the later ones from cache).
template <typename T, bool RMS>
__global__ void __launch_bounds__(kThreads) k_norm_rows(RowSet rs, RowView x, const void* w, const void* bias,
                                                        bool pbf, float eps, int d, RowView y, float* mean,
                                                        float* rstd) {
  __shared__ float part[2][kWarps];
  const int r = blockIdx.x, b = r / rs.T, t = r - b * rs.T;
  T* yr = row_out<T>(y, b, t);
  if (!row_kept(rs, b, t)) {
    for (int c = threadIdx.x; c < d; c += kThreads) yr[c] = from_f32<T>(0.f);
    if (threadIdx.x == 0) {
      if (mean) mean[r] = 0.f;
      if (rstd) rstd[r] = 0.f;
    }
    return;
  }
  const T* xr = row_of<T>(x, b, t);
  float mu = 0.f;
  if (!RMS) {
    float s = 0.f;
    for (int c = threadIdx.x; c < d; c += kThreads) s += to_f32(xr[c]);
    mu = block_sum<kWarps>(s, part[0]) / d;
  }
  float q = 0.f;
  for (int c = threadIdx.x; c < d; c += kThreads) {
    const float v = to_f32(xr[c]) - mu;
    q = fmaf(v, v, q);
  }
  const float rs_ = 1.0f / sqrtf(block_sum<kWarps>(q, part[1]) / d + eps);
  for (int c = threadIdx.x; c < d; c += kThreads) {
    const float v = (to_f32(xr[c]) - mu) * rs_;
    yr[c] = from_f32<T>(fmaf(v, param_at(w, pbf, c, 1.f), param_at(bias, pbf, c, 0.f)));
  }
  if (threadIdx.x == 0) {
    if (mean) mean[r] = mu;
    if (rstd) rstd[r] = rs_;
  }
}

// dx: one block per row, two passes over the row.
template <typename T, bool RMS>
__global__ void __launch_bounds__(kThreads) k_norm_dx_rows(NormGrad g) {
  __shared__ float part[2][kWarps];
  const int r = blockIdx.x, b = r / g.rs.T, t = r - b * g.rs.T;
  T* dxr = row_out<T>(g.dx, b, t);
  if (!row_kept(g.rs, b, t)) {
    for (int c = threadIdx.x; c < g.d; c += kThreads) dxr[c] = from_f32<T>(0.f);
    return;
  }
  const T* xr = row_of<T>(g.x, b, t);
  const T* dyr = row_of<T>(g.dy, b, t);
  const float mu = RMS ? 0.f : g.mean[r], rstd = g.rstd[r];
  float s1 = 0.f, s2 = 0.f;
  for (int c = threadIdx.x; c < g.d; c += kThreads) {
    const float gv = to_f32(dyr[c]) * param_at(g.weight, g.param_bf16, c, 1.f);
    s1 += gv;
    s2 = fmaf(gv, (to_f32(xr[c]) - mu) * rstd, s2);
  }
  const float m1 = RMS ? 0.f : block_sum<kWarps>(s1, part[0]) / g.d;
  const float m2 = block_sum<kWarps>(s2, part[1]) / g.d;
  for (int c = threadIdx.x; c < g.d; c += kThreads) {
    const float gv = to_f32(dyr[c]) * param_at(g.weight, g.param_bf16, c, 1.f);
    const float xh = (to_f32(xr[c]) - mu) * rstd;
    dxr[c] = from_f32<T>(rstd * (gv - m1 - xh * m2));
  }
}

// dw, db: one thread per channel sums a run of rows; partial sums of run p of
// group e go to part[(e * n_parts + p) * 2 + {0, 1}][d].
template <typename T, bool RMS>
__global__ void __launch_bounds__(kThreads) k_norm_dparam_rows(NormGrad g, int rows_per_group, int rows_per_part,
                                                               int n_parts, float* part) {
  const int c = blockIdx.x * kThreads + threadIdx.x, p = blockIdx.y;
  if (c >= g.d) return;
  const int groups = g.per_example ? g.rs.B : 1;
  for (int e = blockIdx.z; e < groups; e += gridDim.z) {
    const int end = min(rows_per_group, (p + 1) * rows_per_part);
    float sw = 0.f, sb = 0.f;
    for (int i = p * rows_per_part; i < end; ++i) {
      const int r = e * rows_per_group + i, b = r / g.rs.T, t = r - b * g.rs.T;
      if (!row_kept(g.rs, b, t)) continue;
      const float dy = to_f32(row_of<T>(g.dy, b, t)[c]);
      const float xh = (to_f32(row_of<T>(g.x, b, t)[c]) - (RMS ? 0.f : g.mean[r])) * g.rstd[r];
      sw = fmaf(dy, xh, sw);
      sb += dy;
    }
    float* o = part + (static_cast<size_t>(e) * n_parts + p) * 2 * g.d;
    o[c] = sw;
    o[g.d + c] = sb;
  }
}

// Adds a group's n_parts partial sums in order.
__global__ void __launch_bounds__(kThreads) k_norm_dparam_join(NormGrad g, int n_parts, const float* part) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= g.d) return;
  const int groups = g.per_example ? g.rs.B : 1;
  for (int e = blockIdx.y; e < groups; e += gridDim.y) {
    float sw = 0.f, sb = 0.f;
    const float* o = part + static_cast<size_t>(e) * n_parts * 2 * g.d;
    for (int p = 0; p < n_parts; ++p, o += 2 * g.d) {
      sw += o[c];
      sb += o[g.d + c];
    }
    const size_t at = static_cast<size_t>(e) * g.ld_dparam + c;
    if (g.dweight) g.dweight[at] = g.accumulate ? g.dweight[at] + sw : sw;
    if (g.dbias) g.dbias[at] = g.accumulate ? g.dbias[at] + sb : sb;
  }
}

// Runs of rows whose weight-gradient sums are formed apart.
int grad_parts(int rows_per_group, int groups, int num_sms) {
  const int want = std::max(1, 4 * num_sms / std::max(1, groups));
  return std::max(1, std::min(want, (rows_per_group + 63) / 64));
}

}  // namespace

cudaError_t launch_norm(bool rms, RowSet rs, RowView x, bool bf16_, const void* weight, const void* bias,
                        bool param_bf16, float eps, int d, RowView y, float* mean, float* rstd, int num_sms,
                        cudaStream_t st) {
  const int M = static_cast<int>(rs.rows());
  auto k = bf16_ ? (rms ? k_norm_rows<bf16, true> : k_norm_rows<bf16, false>)
                 : (rms ? k_norm_rows<float, true> : k_norm_rows<float, false>);
  k<<<M, kThreads, 0, st>>>(rs, x, weight, bias, param_bf16, eps, d, y, mean, rstd);
  return cudaGetLastError();
}

size_t norm_grad_ws_bytes(int B, int T, int d, bool per_example, int num_sms) {
  const int groups = per_example ? B : 1, rows = per_example ? T : B * T;
  return static_cast<size_t>(groups) * grad_parts(rows, groups, num_sms) * 2 * d * 4;
}

cudaError_t launch_norm_grad(const NormGrad& g, void* ws, int num_sms, cudaStream_t st) {
  const int M = static_cast<int>(g.rs.rows());
  if (g.dweight || g.dbias) {
    const int groups = g.per_example ? g.rs.B : 1, rows = g.per_example ? g.rs.T : M;
    if (groups > 0) {
      const int parts = grad_parts(rows, groups, num_sms);
      const int cols = (g.d + kThreads - 1) / kThreads;
      auto k = g.bf16 ? (g.rms ? k_norm_dparam_rows<bf16, true> : k_norm_dparam_rows<bf16, false>)
                      : (g.rms ? k_norm_dparam_rows<float, true> : k_norm_dparam_rows<float, false>);
      k<<<dim3(cols, parts, std::min(groups, 65535)), kThreads, 0, st>>>(g, rows, (rows + parts - 1) / parts, parts,
                                                                        static_cast<float*>(ws));
      k_norm_dparam_join<<<dim3(cols, std::min(groups, 65535)), kThreads, 0, st>>>(g, parts,
                                                                                  static_cast<const float*>(ws));
    }
  }
  if (g.dx.p && M > 0) {
    auto k = g.bf16 ? (g.rms ? k_norm_dx_rows<bf16, true> : k_norm_dx_rows<bf16, false>)
                    : (g.rms ? k_norm_dx_rows<float, true> : k_norm_dx_rows<float, false>);
    k<<<M, kThreads, 0, st>>>(g);
  }
  return cudaGetLastError();
}
