// Token embedding and its gradient.
//   out[t] = scale E[tok_t] (+ P[t]);   dE[v] = scale sum over {t: tok_t = v} of dout[t].
// The gradient's positions are sorted by token (a stable radix sort, so each
// token's positions stay in ascending order) and each token's run is summed in
// that order: bitwise reproducible without floating-point atomics.
#include <algorithm>

#include "rows_dev.cuh"

using namespace eogp;

namespace {

constexpr int kThreads = 256;

// One block per row.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_embed_rows(RowSet rs, TokenView tok, const T* __restrict__ table, int V,
                                                         int d, long long ld_table, float scale,
                                                         const T* __restrict__ pos, long long ld_pos, RowView out,
                                                         unsigned* status) {
  const int r = blockIdx.x, b = r / rs.T, t = r - b * rs.T;
  T* o = row_out<T>(out, b, t);
  bool kept = row_kept(rs, b, t);
  long long v = 0;
  if (kept) {
    v = token_at(tok, b, t);
    if (v < 0 || v >= V) {
      if (threadIdx.x == 0) flag_status(status, EOGP_ST_DEVICE);
      kept = false;
    }
  }
  const T* e = table + v * ld_table;
  for (int c = threadIdx.x; c < d; c += kThreads) {
    float x = 0.f;
    if (kept) {
      x = scale * to_f32(e[c]);
      if (pos) x += to_f32(pos[t * ld_pos + c]);
    }
    o[c] = from_f32<T>(x);
  }
}

// ---------------------------------------------------------------- radix sort
// Stable sort of the positions r = 0..M-1 by key, the key being the token, or V
// for positions that take no part. One pass per digit of `bits` bits: each block
// counts the digits of its contiguous range of elements, then places them; the
// elements of one warp's step are ranked with a warp match, the warps and steps
// in order by counters in shared memory.
constexpr int kMaxBins = 512;
constexpr int kSortThreads = 256;
constexpr int kSortWarps = kSortThreads / 32;

struct SortPlan {
  int passes, bits, bins, blocks, per_block;  // per_block: elements of a block's range
};

SortPlan sort_plan(int V, long long M) {
  SortPlan p;
  int key_bits = 1;
  while ((1ll << key_bits) <= V) ++key_bits;  // keys 0..V
  p.passes = (key_bits + 8) / 9;
  p.bits = (key_bits + p.passes - 1) / p.passes;
  p.bins = 1 << p.bits;
  const long long step = kSortThreads;
  long long per = (M + 127) / 128;
  per = std::max(step * 4, (per + step - 1) / step * step);
  p.per_block = static_cast<int>(per);
  p.blocks = static_cast<int>((M + per - 1) / per);
  return p;
}

__global__ void __launch_bounds__(kSortThreads) k_token_keys(RowSet rs, TokenView tok, int V, int M, int* key, int* idx,
                                                             unsigned* status) {
  const int r = blockIdx.x * kSortThreads + threadIdx.x;
  if (r >= M) return;
  const int b = r / rs.T, t = r - b * rs.T;
  int k = V;
  if (row_kept(rs, b, t)) {
    const long long v = token_at(tok, b, t);
    if (v >= 0 && v < V)
      k = static_cast<int>(v);
    else
      flag_status(status, EOGP_ST_DEVICE);
  }
  key[r] = k;
  idx[r] = r;
}

// hist[block][digit] = elements of the block's range with that digit.
__global__ void __launch_bounds__(kSortThreads) k_sort_count(const int* __restrict__ key, int M, int shift, int bins,
                                                             int per_block, int* __restrict__ hist) {
  __shared__ int cnt[kMaxBins];
  for (int d = threadIdx.x; d < bins; d += kSortThreads) cnt[d] = 0;
  __syncthreads();
  const long long lo = static_cast<long long>(blockIdx.x) * per_block;
  const int hi = static_cast<int>(min(static_cast<long long>(M), lo + per_block));
  for (int i = static_cast<int>(lo) + threadIdx.x; i < hi; i += kSortThreads)
    atomicAdd(&cnt[(key[i] >> shift) & (bins - 1)], 1);
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += kSortThreads) hist[blockIdx.x * bins + d] = cnt[d];
}

// Places the block's elements: element -> (elements with a smaller digit) +
// (elements of earlier blocks with the same digit) + (its rank in the block).
__global__ void __launch_bounds__(kSortThreads) k_sort_place(const int* __restrict__ key, const int* __restrict__ idx,
                                                             int M, int shift, int bins, int per_block, int blocks,
                                                             const int* __restrict__ hist, int* __restrict__ key_out,
                                                             int* __restrict__ idx_out) {
  __shared__ int base[kMaxBins];
  __shared__ int total[kMaxBins];
  __shared__ int wcnt[kSortWarps][kMaxBins];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int d = tid; d < bins; d += kSortThreads) {
    int before = 0, all = 0;
    for (int k = 0; k < blocks; ++k) {
      const int h = hist[k * bins + d];
      if (k < static_cast<int>(blockIdx.x)) before += h;
      all += h;
    }
    base[d] = before;
    total[d] = all;
  }
  __syncthreads();
  if (warp == 0) {  // exclusive sum of the totals, 32 digits at a time
    int carry = 0;
    for (int d0 = 0; d0 < bins; d0 += 32) {
      const int d = d0 + lane, v = d < bins ? total[d] : 0;
      int s = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
      }
      if (d < bins) base[d] += carry + s - v;
      carry += __shfl_sync(0xffffffffu, s, 31);
    }
  }
  const long long lo = static_cast<long long>(blockIdx.x) * per_block;
  const int hi = static_cast<int>(min(static_cast<long long>(M), lo + per_block));
  for (int i0 = static_cast<int>(lo); i0 < hi; i0 += kSortThreads) {
    for (int d = lane; d < bins; d += 32) wcnt[warp][d] = 0;
    __syncwarp();
    const int i = i0 + tid;
    const bool on = i < hi;
    const int k = on ? key[i] : 0, p = on ? idx[i] : 0;
    const int dg = on ? (k >> shift) & (bins - 1) : -1;
    const unsigned same = __match_any_sync(0xffffffffu, dg);
    const int rank = __popc(same & ((1u << lane) - 1u));
    if (on && rank == 0) wcnt[warp][dg] = __popc(same);
    __syncthreads();
    if (on) {
      int at = base[dg] + rank;
      for (int w = 0; w < warp; ++w) at += wcnt[w][dg];
      key_out[at] = k;
      idx_out[at] = p;
    }
    __syncthreads();
    for (int d = tid; d < bins; d += kSortThreads) {
      int s = 0;
      for (int w = 0; w < kSortWarps; ++w) s += wcnt[w][d];
      base[d] += s;
    }
    __syncthreads();
  }
}

__device__ __forceinline__ int lower_bound(const int* __restrict__ key, int n, int v) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (key[mid] < v)
      lo = mid + 1;
    else
      hi = mid;
  }
  return lo;
}

// One block per table row: its run of the sorted positions, summed in order.
template <typename T, typename G>
__global__ void __launch_bounds__(kThreads) k_embed_sum_rows(RowSet rs, RowView dout, const int* __restrict__ key,
                                                             const int* __restrict__ idx, int M, int V, int d,
                                                             float scale, G* __restrict__ dtable, long long ld,
                                                             bool accumulate) {
  const int v = blockIdx.x;
  const int lo = lower_bound(key, M, v), hi = lower_bound(key, M, v + 1);
  if (accumulate && lo == hi) return;
  G* o = dtable + v * ld;
  for (int c = threadIdx.x; c < d; c += kThreads) {
    float s = 0.f;
    for (int i = lo; i < hi; ++i) {
      const int r = idx[i], b = r / rs.T, t = r - b * rs.T;
      s += to_f32(row_of<T>(dout, b, t)[c]);
    }
    s *= scale;
    o[c] = from_f32<G>(accumulate ? to_f32(o[c]) + s : s);
  }
}

size_t al256(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace

cudaError_t launch_embed(RowSet rs, TokenView tok, const void* table, bool bf16_, int V, int d, long long ld_table,
                         float scale, const void* pos, long long ld_pos, RowView out, unsigned* status,
                         cudaStream_t st) {
  const int M = static_cast<int>(rs.rows());
  if (bf16_)
    k_embed_rows<bf16><<<M, kThreads, 0, st>>>(rs, tok, static_cast<const bf16*>(table), V, d, ld_table, scale,
                                              static_cast<const bf16*>(pos), ld_pos, out, status);
  else
    k_embed_rows<float><<<M, kThreads, 0, st>>>(rs, tok, static_cast<const float*>(table), V, d, ld_table, scale,
                                               static_cast<const float*>(pos), ld_pos, out, status);
  return cudaGetLastError();
}

size_t embed_grad_ws_bytes(int V, int d, long long M) {
  if (M == 0) return 0;
  const SortPlan p = sort_plan(V, M);
  return 4 * al256(M * 4) + al256(static_cast<size_t>(p.blocks) * p.bins * 4);
}

cudaError_t launch_embed_grad(RowSet rs, TokenView tok, RowView dout, bool bf16_, int V, int d, float scale,
                              void* dtable, bool grad_bf16, long long ld_dtable, bool accumulate, void* ws,
                              unsigned* status, int num_sms, cudaStream_t st) {
  const int M = static_cast<int>(rs.rows());
  int *key = nullptr, *idx = nullptr;
  if (M > 0) {
    const SortPlan p = sort_plan(V, M);
    uint8_t* w = static_cast<uint8_t*>(ws);
    const size_t a = al256(static_cast<size_t>(M) * 4);
    key = reinterpret_cast<int*>(w);
    idx = reinterpret_cast<int*>(w + a);
    int* key2 = reinterpret_cast<int*>(w + 2 * a);
    int* idx2 = reinterpret_cast<int*>(w + 3 * a);
    int* hist = reinterpret_cast<int*>(w + 4 * a);
    k_token_keys<<<(M + kSortThreads - 1) / kSortThreads, kSortThreads, 0, st>>>(rs, tok, V, M, key, idx, status);
    for (int s = 0; s < p.passes; ++s) {
      k_sort_count<<<p.blocks, kSortThreads, 0, st>>>(key, M, s * p.bits, p.bins, p.per_block, hist);
      k_sort_place<<<p.blocks, kSortThreads, 0, st>>>(key, idx, M, s * p.bits, p.bins, p.per_block, p.blocks, hist,
                                                      key2, idx2);
      std::swap(key, key2);
      std::swap(idx, idx2);
    }
  }
  if (bf16_ && grad_bf16)
    k_embed_sum_rows<bf16, bf16><<<V, kThreads, 0, st>>>(rs, dout, key, idx, M, V, d, scale, static_cast<bf16*>(dtable),
                                                        ld_dtable, accumulate);
  else if (bf16_)
    k_embed_sum_rows<bf16, float><<<V, kThreads, 0, st>>>(rs, dout, key, idx, M, V, d, scale,
                                                         static_cast<float*>(dtable), ld_dtable, accumulate);
  else if (grad_bf16)
    k_embed_sum_rows<float, bf16><<<V, kThreads, 0, st>>>(rs, dout, key, idx, M, V, d, scale,
                                                         static_cast<bf16*>(dtable), ld_dtable, accumulate);
  else
    k_embed_sum_rows<float, float><<<V, kThreads, 0, st>>>(rs, dout, key, idx, M, V, d, scale,
                                                          static_cast<float*>(dtable), ld_dtable, accumulate);
  return cudaGetLastError();
}
