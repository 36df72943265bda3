// Device code that the kernels of the token loss through the output matrix share
// (k_head.cu, k_head_tc.cu).
#pragma once

#include <algorithm>

#include "rows_dev.cuh"

namespace eogp {

constexpr int kMostSplits = 32;

// The kernels of a call follow each other by programmatic launch: each is let in as soon as the one before has
// begun everywhere, sets itself up, and waits here for that one's end. (511 tokens with gradient: nine launches.)
__device__ __forceinline__ void after_previous() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// How many slabs the sums of `tiles` tiles of 256 rows are split into, `steps` 64-deep steps each, so that
// the pairs of multiprocessors take about the same share, by a whole warp. Tiles are taken in rounds;
// a round costs its steps and about 8 more (filling the ring, ending a tile), and a split the
// writing and reading of its slabs and the launch that joins them, in steps of 0.38 us (3,977 rows
// of 4096 columns, 1,563 steps: 2.40 ms unsplit in four rounds of 76, the last a third full).
// More than 16 rounds are not split: what the last one leaves idle is no more than that.
__host__ __device__ __forceinline__ bool head_split_at_all(long long tiles, int clusters) { return tiles <= 16ll * clusters; }
__device__ __forceinline__ int head_splits(const HeadTc& h, long long tiles, int steps, int rows) {
  if (!head_split_at_all(tiles, h.clusters)) return 1;
  const int s = static_cast<int>(threadIdx.x & 31) + 1;
  const unsigned long long slab = static_cast<unsigned long long>(rows) * h.ld_slab;
  long long cost = (tiles * s + h.clusters - 1) / h.clusters * ((steps + s - 1) / s * (h.used_a == 2 ? 2 : 1) + 8);
  if (s > 1) cost += 8 + static_cast<long long>(s * slab / 323000);
  if (s > 1 && (s > steps || s * slab * 4 > h.slab_bytes)) cost = 0x7fffffffffffffffll;
  unsigned long long best = static_cast<unsigned long long>(cost);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
  return __ffs(__ballot_sync(0xffffffffu, static_cast<unsigned long long>(cost) == best));
}

// Most floats of slabs that head_splits may choose for such a sum, of `weight` (2: D in two parts) times the steps and
// slabs of `slab` floats. From cost(s) < cost(1), with rounds(s) >= tiles s / clusters and steps of a split >= steps / s:
//   s (slab / 323000 + 8 tiles / clusters) < (rounds(1) - tiles / clusters) weight steps + 8 rounds(1) - 7.
// It grows with the steps.
inline size_t head_slab_floats(long long tiles, long long steps, int weight, size_t slab, int clusters) {
  if (!head_split_at_all(tiles, clusters)) return 0;
  const double each = static_cast<double>(tiles) / clusters, rounds = static_cast<double>((tiles + clusters - 1) / clusters);
  const double s = ((rounds - each) * weight * steps + 8 * rounds - 7) / (slab / 323000.0 + 8 * each) + 1e-6;
  const long long most = std::min<long long>(steps, s < 2 ? 1 : s < kMostSplits ? static_cast<long long>(s) : kMostSplits);
  return most < 2 ? 0 : most * slab;
}

}  // namespace eogp

// Launches k after what was launched before on the stream, as after_previous() has it; `next` false: plainly.
template <typename... P, typename... A>
cudaError_t head_launch(void (*k)(P...), bool next, unsigned grid, unsigned block, size_t smem, cudaStream_t st,
                        A... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = next ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k, static_cast<P>(args)...);
}
