// Token embedding and its gradient.
//   out[t] = scale E[tok_t] (+ P[t]);   dE[v] = scale sum over {t: tok_t = v} of dout[t].
// The gradient's positions are sorted by token (a stable radix sort, so each
// token's positions stay in ascending order) and each token's run is summed, its chunks
// in that order and then the chunks' sums in a fixed one: bitwise reproducible without
// floating-point atomics.
#include <algorithm>

#include "rows_dev.cuh"
#include "sort_plan.h"

using namespace eogp;

namespace {

constexpr int kThreads = 256;

// A team of TL threads copies NV vectors of N elements a thread of each of R rows
// (wider rows are cut into slices of TL * NV vectors): the R token numbers are
// waited for together, then R * NV table reads a thread are in flight. HBM-bound:
// 32 x 2048 rows of 4096 bf16 with lengths in 100 us, 0.95 of the copy rate; one row
// of 768 in 1.6 us.
template <typename T, int N, int TL, int NV, int R>
__global__ void __launch_bounds__(kThreads) k_embed(RowSet rs, TokenView tok, const T* __restrict__ table, int V, int d,
                                                    long long ld_table, float scale, const T* __restrict__ pos,
                                                    long long ld_pos, RowView out, int M, int slices,
                                                    unsigned* status) {
  constexpr int teams = kThreads / TL;
  const long long team = static_cast<long long>(blockIdx.x) * teams + threadIdx.x / TL;
  const long long rows = slices == 1 ? team : team / slices;
  const int lane = threadIdx.x & (TL - 1), c0 = (static_cast<int>(team - rows * slices) * TL * NV + lane) * N;
  int b[R], t[R];
  int v[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const long long r = rows * R + k;
    b[k] = -1;
    v[k] = -1;
    if (r < M) {
      locate(rs, static_cast<int>(r), b[k], t[k]);
      if (row_kept(rs, b[k], t[k])) {
        const long long id = token_at(tok, b[k], t[k]);
        if (id >= 0 && id < V)
          v[k] = static_cast<int>(id);
        else if (c0 == 0)
          flag_status(status, EOGP_ST_DEVICE);
      }
    }
  }
  Raw<T, N> e[R][NV];
#pragma unroll
  for (int k = 0; k < R; ++k)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + j * TL * N;
      e[k][j] = Raw<T, N>{};
      if (v[k] >= 0 && c < d) e[k][j] = ld_keep<T, N>(table + v[k] * ld_table + c);
    }
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (b[k] < 0) continue;
    T* o = row_out<T>(out, b[k], t[k]);
    const T* q = pos && v[k] >= 0 ? pos + t[k] * ld_pos : nullptr;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + j * TL * N;
      if (c >= d) continue;
      Vals<N> x = unpack<T, N>(e[k][j]), y = fill<N>(0.f);
      if (q) y = unpack<T, N>(ld_keep<T, N>(q + c));
#pragma unroll
      for (int i = 0; i < Vals<N>::P; ++i) x.p[i] = fma2(x.p[i], Vals<N>::all(scale), y.p[i]);
      st_vals<T, N>(o + c, x);
    }
  }
}

// ---------------------------------------------------------------- radix sort
// Stable sort of the positions r = 0..M-1 by key, the key being the token, or V
// for positions that take no part. A pass places the positions by one digit of
// the key: each block counts the digits of its contiguous range, then (next
// launch) places its range tile by tile. Within a tile a warp owns 256 consecutive
// positions; 32 at a time they are ranked among equal digits by a warp match and
// the warp's own counters in shared memory, and the warps' counters are added up
// once a tile. Up to one tile of positions is sorted by one block, up to eight by a
// cluster of blocks, in one launch.
constexpr int kMaxBins = 1 << kMaxSortBits;
constexpr int kItems = kSortItems;
constexpr int kTile = kSortTile;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMarked = 1024;

// A token's mark. Neighbours lie apart: the frequent tokens of many vocabularies are
// neighbours, and stores to one sector wait for each other (keys and marks of 262,144
// positions: 17 us with neighbours together, 10 us so).
__host__ __device__ __forceinline__ int mark_stride(int V) { return (V + 31) / 32; }
__device__ __forceinline__ int mark_of(int v, int V) { return (v & 31) * mark_stride(V) + (v >> 5); }

// Zeroing of dtable's rows of absent tokens, by blocks of their own beside those of
// another job in the same launch: the stores fill the time that the sort waits.
struct ZeroArgs {
  uint8_t* table;
  size_t stride, row_bytes;
  int unit;                 // bytes of a store: 16, or an element's
  const uint8_t* present;   // tokens that occur, or NULL: every row is zeroed
  int V, v0, v1, rows, blocks;  // rows [v0, v1), `rows` of them a block
};

__device__ void zero_rows(const ZeroArgs& z, int block) {
  const int lane = threadIdx.x & 31;
  for (int i = threadIdx.x >> 5; i < z.rows; i += kSortWarps) {
    const long long v = z.v0 + static_cast<long long>(block) * z.rows + i;
    if (v >= z.v1 || (z.present && z.present[mark_of(static_cast<int>(v), z.V)])) continue;
    uint8_t* o = z.table + v * z.stride;
    if (z.unit == 16) {
      for (size_t k = lane * 16; k < z.row_bytes; k += 512)
        __stcs(reinterpret_cast<uint4*>(o + k), make_uint4(0, 0, 0, 0));
    } else if (z.unit == 4) {
      for (size_t k = lane * 4; k < z.row_bytes; k += 128) *reinterpret_cast<uint32_t*>(o + k) = 0;
    } else {
      for (size_t k = lane * 2; k < z.row_bytes; k += 64) *reinterpret_cast<uint16_t*>(o + k) = 0;
    }
  }
}

// Keys of positions at0 + s * step (those below hi, else -1), all their
// loads in flight at once.
template <bool I64, int K>
__device__ __forceinline__ void token_keys(const RowSet& rs, const TokenView& tok, int V, int at0, int step, int hi,
                                           int (&k)[K], unsigned* status) {
  long long id[K];
#pragma unroll
  for (int s = 0; s < K; ++s) {
    const int i = at0 + s * step;
    int b, t;
    locate(rs, i < hi ? i : 0, b, t);
    id[s] = V;
    if (i < hi && row_kept(rs, b, t)) {
      if constexpr (I64)
        id[s] = static_cast<const long long*>(tok.p)[b * tok.bs + t];
      else
        id[s] = static_cast<const int*>(tok.p)[b * tok.bs + t];
      if (id[s] == V) id[s] = -1;  // V itself is no token
    }
  }
  bool bad = false;
#pragma unroll
  for (int s = 0; s < K; ++s) {
    const bool out = id[s] < 0 || id[s] > V;
    bad |= out;
    k[s] = at0 + s * step < hi ? (out ? V : static_cast<int>(id[s])) : -1;
  }
  if (bad) flag_status(status, EOGP_ST_DEVICE);
}

// Counting takes kCount positions a block, several blocks adding to the counts of
// one range (whole numbers: the order does not matter).
constexpr int kCount = kThreads * kItems / 2;

// Keys, the tokens that occur, and hist[range][digit] of the lowest digit. present
// and hist start at 0.
template <bool I64>
__global__ void __launch_bounds__(kThreads) k_sort_keys(RowSet rs, TokenView tok, int V, int M, int bins, int per_block,
                                                        int* __restrict__ key, uint8_t* __restrict__ present,
                                                        int* __restrict__ hist, unsigned* status) {
  __shared__ int cnt[kMaxBins];
  // Tokens that this block has marked lately: a frequent token's mark would
  // otherwise be stored at one address by every position that holds it.
  __shared__ int marked[kMarked];
  for (int d = threadIdx.x; d < bins; d += kThreads) cnt[d] = 0;
  for (int d = threadIdx.x; d < kMarked; d += kThreads) marked[d] = -1;
  __syncthreads();
  const int lo = blockIdx.x * kCount;
  int k[kCount / kThreads];
  token_keys<I64>(rs, tok, V, lo + threadIdx.x, kThreads, M, k, status);
#pragma unroll
  for (int s = 0; s < kCount / kThreads; ++s) {
    if (k[s] < 0) continue;
    key[lo + threadIdx.x + s * kThreads] = k[s];
    volatile int* const seen = &marked[k[s] & (kMarked - 1)];
    if (k[s] < V && *seen != k[s]) {
      *seen = k[s];
      present[mark_of(k[s], V)] = 1;
    }
    atomicAdd(&cnt[k[s] & (bins - 1)], 1);
  }
  __syncthreads();
  int* const to = hist + lo / per_block * bins;
  for (int d = threadIdx.x; d < bins; d += kThreads)
    if (cnt[d]) atomicAdd(&to[d], cnt[d]);
}

// hist[range][digit] of another digit.
__global__ void __launch_bounds__(kSortThreads) k_sort_count(const int* __restrict__ key, int M, int shift, int bins,
                                                             int per_block, int blocks, int* __restrict__ hist,
                                                             const ZeroArgs z) {
  if (blockIdx.x >= blocks) return zero_rows(z, blockIdx.x - blocks);
  __shared__ int cnt[kMaxBins];
  for (int d = threadIdx.x; d < bins; d += kSortThreads) cnt[d] = 0;
  __syncthreads();
  const int lo = blockIdx.x * kCount;
  int k[kCount / kSortThreads];
#pragma unroll
  for (int s = 0; s < kCount / kSortThreads; ++s) {
    const int i = lo + threadIdx.x + s * kSortThreads;
    k[s] = i < M ? key[i] : -1;
  }
#pragma unroll
  for (int s = 0; s < kCount / kSortThreads; ++s)
    if (k[s] >= 0) atomicAdd(&cnt[(k[s] >> shift) & (bins - 1)], 1);
  __syncthreads();
  int* const to = hist + lo / per_block * bins;
  for (int d = threadIdx.x; d < bins; d += kSortThreads)
    if (cnt[d]) atomicAdd(&to[d], cnt[d]);
}

// Exclusive sum of total[0..bins) added into base, by the first warp.
__device__ __forceinline__ void scan_bins(const int* total, int* base, int bins) {
  const int lane = threadIdx.x;
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

// Ranks of a tile: on return position dst of item s of this thread is
// base[digit] + wcnt[warp][digit] + off[s]. dg < 0: no item. Uses two barriers.
__device__ __forceinline__ void rank_tile(const int (&dg)[kItems], int (&off)[kItems], unsigned short (*wcnt)[kMaxBins],
                                          int* tile_total, int bins) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int d = lane; d < bins; d += 32) wcnt[warp][d] = 0;
  __syncwarp();
#pragma unroll
  for (int s = 0; s < kItems; ++s) {
    const unsigned same = __match_any_sync(0xffffffffu, dg[s]);
    const int rank = __popc(same & ((1u << lane) - 1u));
    off[s] = dg[s] >= 0 ? wcnt[warp][dg[s]] + rank : 0;
    __syncwarp();
    if (dg[s] >= 0 && rank == 0) wcnt[warp][dg[s]] = static_cast<unsigned short>(off[s] + __popc(same));
    __syncwarp();
  }
  __syncthreads();
  for (int d = tid; d < bins; d += kSortThreads) {
    int run = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      const int n = wcnt[w][d];
      wcnt[w][d] = static_cast<unsigned short>(run);
      run += n;
    }
    tile_total[d] = run;
  }
  __syncthreads();
}

// Places the block's range: position -> (positions with a smaller digit) + (earlier
// blocks' with the same) + (its rank in the block). idx NULL: the positions themselves.
__global__ void __launch_bounds__(kSortThreads) k_sort_place(const int* __restrict__ key, const int* __restrict__ idx,
                                                         int M, int shift, int bins, int per_block, int blocks,
                                                         const int* __restrict__ hist, int* __restrict__ key_out,
                                                         int* __restrict__ idx_out, const ZeroArgs z) {
  if (blockIdx.x >= blocks) return zero_rows(z, blockIdx.x - blocks);
  __shared__ int base[kMaxBins], total[kMaxBins];
  __shared__ unsigned short wcnt[kSortWarps][kMaxBins];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int lo = blockIdx.x * per_block, hi = min(M, lo + per_block);
  int k[kItems], p[kItems];
  auto load = [&](int t0) {
#pragma unroll
    for (int s = 0; s < kItems; ++s) {
      const int i = t0 + warp * (32 * kItems) + s * 32 + lane;
      k[s] = i < hi ? key[i] : 0;
      p[s] = i < hi ? (idx ? idx[i] : i) : 0;
    }
  };
  load(lo);  // on their way beside the counts
  for (int d = tid; d < bins; d += kSortThreads) {
    int before = 0, all = 0;
#pragma unroll 32
    for (int k = 0; k < blocks; ++k) {
      const int h = hist[k * bins + d];
      if (k < static_cast<int>(blockIdx.x)) before += h;
      all += h;
    }
    base[d] = before;
    total[d] = all;
  }
  __syncthreads();
  if (warp == 0) scan_bins(total, base, bins);
  for (int t0 = lo; t0 < hi; t0 += kTile) {
    int dg[kItems], off[kItems];
#pragma unroll
    for (int s = 0; s < kItems; ++s)
      dg[s] = t0 + warp * (32 * kItems) + s * 32 + lane < hi ? (k[s] >> shift) & (bins - 1) : -1;
    rank_tile(dg, off, wcnt, total, bins);
#pragma unroll
    for (int s = 0; s < kItems; ++s) {
      if (dg[s] < 0) continue;
      const int at = base[dg[s]] + wcnt[warp][dg[s]] + off[s];
      key_out[at] = k[s];
      idx_out[at] = p[s];
    }
    load(min(t0 + kTile, hi));
    __syncthreads();
    for (int d = tid; d < bins; d += kSortThreads) base[d] += total[d];
    __syncthreads();
  }
}

// M <= kTile: keys and every pass in block 0; the other blocks zero dtable.
template <bool I64>
__global__ void __launch_bounds__(kSortThreads) k_sort_one(RowSet rs, TokenView tok, int V, int M, int passes, int bits,
                                                       int* __restrict__ key_out, int* __restrict__ idx_out,
                                                       const ZeroArgs z, unsigned* status) {
  if (blockIdx.x > 0) return zero_rows(z, blockIdx.x - 1);
  __shared__ int base[kMaxBins], total[kMaxBins];
  __shared__ unsigned short wcnt[kSortWarps][kMaxBins];
  __shared__ int skey[kTile];
  __shared__ unsigned short sidx[kTile];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, bins = 1 << bits;
  int k[kItems], p[kItems], dg[kItems], off[kItems];
  token_keys<I64, kItems>(rs, tok, V, warp * (32 * kItems) + lane, 32, M, k, status);
#pragma unroll
  for (int s = 0; s < kItems; ++s) p[s] = warp * (32 * kItems) + s * 32 + lane;
  for (int pass = 0; pass < passes; ++pass) {
#pragma unroll
    for (int s = 0; s < kItems; ++s) {
      const int i = warp * (32 * kItems) + s * 32 + lane;
      if (pass > 0 && i < M) {
        k[s] = skey[i];
        p[s] = sidx[i];
      }
      dg[s] = i < M ? (k[s] >> (pass * bits)) & (bins - 1) : -1;
    }
    for (int d = tid; d < bins; d += kSortThreads) base[d] = 0;
    rank_tile(dg, off, wcnt, total, bins);
    if (warp == 0) scan_bins(total, base, bins);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kItems; ++s) {
      if (dg[s] < 0) continue;
      const int at = base[dg[s]] + wcnt[warp][dg[s]] + off[s];
      if (pass == passes - 1) {
        key_out[at] = k[s];
        idx_out[at] = p[s];
      } else {
        skey[at] = k[s];
        sidx[at] = static_cast<unsigned short>(p[s]);
      }
    }
    __syncthreads();
  }
}

// kTile < M <= kClusterRows: keys and every pass in the first cluster, a tile a block,
// whose blocks wait for each other between the steps; the other clusters zero dtable.
// A pass reads one pair of keys and positions and writes the other, as hist
// [passes][blocks][bins], in device memory, where data of other blocks is read past
// the first-level cache. Launches of their own for the steps: 34.9 us instead of 21.1
// for all of 8192 positions of 768 bf16, 51 us instead of 42 for 32,768. Two tiles a
// block do not pay (49,152 positions: 74.5 us, launches 71.0 us).
constexpr int kSortCluster = 8;
constexpr int kClusterRows = kSortCluster * kTile;

struct ClusterSort {
  RowSet rs;
  TokenView tok;
  int V, M, passes, bits, per_block;
  int *key[2], *idx[2];  // sorted: [passes & 1]
  int* hist;
  ZeroArgs z;
  unsigned* status;
};

template <bool I64>
__global__ void __launch_bounds__(kSortThreads, 2) k_sort_cluster(const ClusterSort a) {
  if (blockIdx.x >= kSortCluster) return zero_rows(a.z, blockIdx.x - kSortCluster);
  __shared__ int base[kMaxBins], total[kMaxBins];
  __shared__ unsigned short wcnt[kSortWarps][kMaxBins];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, bins = 1 << a.bits;
  const int lo = min(a.M, static_cast<int>(blockIdx.x) * a.per_block), hi = min(a.M, lo + a.per_block);
  const int in_tile = warp * (32 * kItems) + lane;
  int k[kItems], p[kItems];
  for (int pass = 0; pass < a.passes; ++pass) {
    const int* const key = a.key[pass & 1];
    const int* const idx = a.idx[pass & 1];
    int* const key_out = a.key[~pass & 1];
    int* const idx_out = a.idx[~pass & 1];
    int* const hist = a.hist + pass * kSortCluster * bins;
    const int shift = pass * a.bits;
    for (int d = tid; d < bins; d += kSortThreads) total[d] = 0;
    __syncthreads();
    // A range is one tile, which stays in registers from the counting to the placing.
    // Both are written as loops over tiles all the same: as straight code they came out
    // slower (8192 positions into 50,000 rows 39.6 us instead of 35.1).
    for (int t0 = lo; t0 < hi; t0 += kTile) {
      if (pass == 0) {
        token_keys<I64, kItems>(a.rs, a.tok, a.V, t0 + in_tile, 32, hi, k, a.status);
#pragma unroll
        for (int s = 0; s < kItems; ++s) p[s] = t0 + in_tile + s * 32;
      } else {
#pragma unroll
        for (int s = 0; s < kItems; ++s) {
          const int i = t0 + in_tile + s * 32;
          k[s] = i < hi ? __ldcg(key + i) : -1;
          p[s] = i < hi ? __ldcg(idx + i) : 0;
        }
      }
#pragma unroll
      for (int s = 0; s < kItems; ++s)
        if (k[s] >= 0) atomicAdd(&total[(k[s] >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
    for (int d = tid; d < bins; d += kSortThreads) hist[blockIdx.x * bins + d] = total[d];
    cluster_arrive();
    cluster_wait();
    for (int d = tid; d < bins; d += kSortThreads) {
      int h[kSortCluster], before = 0, all = 0;
#pragma unroll
      for (int c = 0; c < kSortCluster; ++c) h[c] = __ldcg(hist + c * bins + d);
#pragma unroll
      for (int c = 0; c < kSortCluster; ++c) {
        if (c < static_cast<int>(blockIdx.x)) before += h[c];
        all += h[c];
      }
      base[d] = before;
      total[d] = all;
    }
    __syncthreads();
    if (warp == 0) scan_bins(total, base, bins);
    for (int t0 = lo; t0 < hi; t0 += kTile) {
      int dg[kItems], off[kItems];
#pragma unroll
      for (int s = 0; s < kItems; ++s) dg[s] = k[s] >= 0 ? (k[s] >> shift) & (bins - 1) : -1;
      rank_tile(dg, off, wcnt, total, bins);
#pragma unroll
      for (int s = 0; s < kItems; ++s) {
        if (dg[s] < 0) continue;
        const int at = base[dg[s]] + wcnt[warp][dg[s]] + off[s];
        key_out[at] = k[s];
        idx_out[at] = p[s];
      }
      __syncthreads();
      for (int d = tid; d < bins; d += kSortThreads) base[d] += total[d];
      __syncthreads();
    }
    if (pass + 1 < a.passes) {
      cluster_arrive();
      cluster_wait();
    }
  }
}

// -------------------------------------------------------------- sums of runs
// The sorted positions are cut into chunks of `chunk`, `teams` chunks a block. A
// thread sums one vector of N channels over one chunk, run after run. A run inside
// a chunk is a finished row of dtable; the pieces of one that several chunks share
// are added in order, those of a block in shared memory, those of several blocks by
// k_embed_join from the blocks' slots: 0 for a run that began in an earlier block,
// 1 for one that goes on in the next, d floats each. HBM-bound, with rows read in
// pieces of 512 bytes in token order: 512 x 512 positions of 768 bf16 with lengths
// (253 MB in, 77 MB out) in 66 us of the call's 118. Without lengths, 50,000 rows of
// table: fp32 149 us and 160 accumulated into, bf16 133 and 151.
struct SumArgs {
  RowSet rs;  // B = 1 where dout's rows follow each other
  RowView dout;
  const int *key, *idx;
  int M, V, d, nv, chunk, ct, teams, tiles, groups;  // ct vectors a column tile; tiles x groups blocks
  float scale;
  void* dtable;
  long long ld;
  bool accumulate;
  float* slots;
};

template <typename G, int N>
__device__ __forceinline__ void st_run(G* o, Vals<N> s, float scale, bool accumulate) {
#pragma unroll
  for (int i = 0; i < Vals<N>::P; ++i) s.p[i] = mul2(s.p[i], Vals<N>::all(scale));
  if (accumulate) {
    const Vals<N> old = ld_wide<G, N>(o);
#pragma unroll
    for (int i = 0; i < Vals<N>::P; ++i) s.p[i] = add2(old.p[i], s.p[i]);
  }
  st_wide<G, N>(o, s);
}

constexpr int kAhead = 8;                            // rows a thread has asked for and not added yet
constexpr int kChunk = 32;                           // most positions of a chunk

// Shared memory of a block: the rows in flight (later the pieces), then the rows'
// offsets and keys.
template <typename T, int N>
constexpr int kFlightBytes = kThreads * (kAhead * N * int(sizeof(T)) > 8 * N ? kAhead * N * int(sizeof(T)) : 8 * N);

template <typename T, typename G, int N>
__global__ void __launch_bounds__(kThreads, 4) k_embed_sum(const SumArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, grp = blockIdx.x / a.tiles, tile = blockIdx.x - grp * a.tiles;
  const int per_block = a.teams * a.chunk;
  // row[i]: the row of the block's position i; skey[1 + i]: its key, skey[0] the
  // one before.
  const T** const row = reinterpret_cast<const T**>(smem + kFlightBytes<T, N>);
  int* const skey = reinterpret_cast<int*>(row + per_block);
  __shared__ int snext, sn;  // key after the block's last position, -1 at the end; positions that are tokens
  const int g0 = grp * per_block, n0 = min(a.M - g0, per_block);
  if (a.key[g0] == a.V) return;  // sorted: none from here on
  if (tid == 0) {
    skey[0] = g0 > 0 ? a.key[g0 - 1] : -1;
    snext = g0 + n0 < a.M ? a.key[g0 + n0] : -1;
    sn = n0;
  }
  __syncthreads();
  for (int i = tid; i < n0; i += kThreads) {
    const int k = a.key[g0 + i], r = a.idx[g0 + i];
    skey[1 + i] = k;
    if (k == a.V) atomicMin(&sn, i);
    int b, t;
    locate(a.rs, r, b, t);
    row[i] = row_of<T>(a.dout, b, t);
  }
  __syncthreads();
  const int n = sn;
  const int team = tid / a.ct, j = tile * a.ct + (tid - team * a.ct);
  const bool on = j < a.nv;
  G* const table = static_cast<G*>(a.dtable) + j * N;
  // Key of position i of the block, i <= n.
  auto key_at = [&](int i) { return i < n0 ? skey[1 + i] : snext; };
  const int lo = team * a.chunk, hi = min(n, lo + a.chunk);
  Vals<N> s = fill<N>(0.f), head = fill<N>(0.f);  // of the run in hand; of one begun earlier that ended here
  bool begins = true;
  if (on && lo < hi) {
    int run = skey[1 + lo];
    begins = run != skey[lo];
    // Rows arrive in this thread's own places of shared memory, kAhead - 1 of them
    // on their way, so nothing but the thread waits for them.
    Raw<T, N>* const flight = reinterpret_cast<Raw<T, N>*>(smem) + tid;
#pragma unroll
    for (int u = 0; u < kAhead - 1; ++u) {
      if (lo + u < hi) copy_async<T, N>(flight + u * kThreads, row[lo + u] + j * N);
      commit_async();
    }
    for (int i0 = lo; i0 < hi; i0 += kAhead) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = i0 + u, next = i + kAhead - 1;
        if (next < hi) copy_async<T, N>(flight + (u + kAhead - 1) % kAhead * kThreads, row[next] + j * N);
        commit_async();
        if (i < hi) {
          wait_async<kAhead - 1>();
          const Vals<N> v = unpack<T, N>(flight[u * kThreads]);
          const int k = skey[1 + i];
          if (k != run) {  // `run` ends inside the chunk
            if (begins)
              st_run<G, N>(table + run * a.ld, s, a.scale, a.accumulate);
            else
              head = s;
            run = k;
            begins = true;
            s = fill<N>(0.f);
          }
#pragma unroll
          for (int p = 0; p < Vals<N>::P; ++p) s.p[p] = add2(s.p[p], v.p[p]);
        }
      }
    }
    if (begins && key_at(hi) != run) st_run<G, N>(table + run * a.ld, s, a.scale, a.accumulate);
  }
  // The pieces of shared runs go where the positions were: [0] of a run begun
  // earlier, [1] of one that goes on. The first team's threads add them in order.
  __syncthreads();
  float* const piece = reinterpret_cast<float*>(smem);
  if (on && lo < hi) {
    const bool whole = skey[1 + lo] == skey[hi];  // one run
    if (skey[1 + lo] == skey[lo]) st_floats<N>(piece + tid * 2 * N, whole ? s : head);
    if (begins) st_floats<N>(piece + tid * 2 * N + N, s);
  }
  __syncthreads();
  if (team > 0 || !on) return;
  s = fill<N>(0.f);
  bool inside = false;  // the run being added began in this block
  for (int k = 0; k * a.chunk < n; ++k) {
    const int l = k * a.chunk, h = min(n, l + a.chunk);
    const float* pk = piece + (k * a.ct + tid) * 2 * N;
    const int first = skey[1 + l], last = skey[h];
    if (first == skey[l]) {
      const Vals<N> v = ld_floats<N>(pk);
#pragma unroll
      for (int i = 0; i < Vals<N>::P; ++i) s.p[i] = add2(s.p[i], v.p[i]);
      if (first != last || key_at(h) != first) {  // it ends in this chunk
        if (inside)
          st_run<G, N>(table + first * a.ld, s, a.scale, a.accumulate);
        else
          st_floats<N>(a.slots + (static_cast<size_t>(grp) * 2 * a.nv + j) * N, s);
        s = fill<N>(0.f);
      }
      if (first == last) continue;
    }
    if (key_at(h) == last) {  // it begins in this chunk and goes on
      s = ld_floats<N>(pk + N);
      inside = true;
    }
  }
  if (key_at(n) == skey[n])
    st_floats<N>(a.slots + ((static_cast<size_t>(grp) * 2 + (inside ? 1 : 0)) * a.nv + j) * N, s);
}

// Runs over several blocks, each added by a warp for 4 vectors: lane = slice * 4 +
// vector, slice s of 8 taking every eighth of the run's blocks in order, the slices
// then joined in a tree.
template <typename G, int N>
__global__ void __launch_bounds__(kThreads) k_embed_join(const SumArgs a) {
  const int lane = threadIdx.x & 31, slice = lane >> 2, quads = (a.nv + 3) / 4;
  const long long warp = static_cast<long long>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  const int c = static_cast<int>(warp / quads), j = static_cast<int>(warp - static_cast<long long>(c) * quads) * 4 + (lane & 3);
  const int per_block = a.teams * a.chunk;
  if (c >= a.groups - 1) return;
  const int lo = c * per_block, hi = lo + per_block;
  const int run = a.key[hi - 1];
  if (run == a.V || a.key[hi] != run || (lo > 0 && a.key[lo - 1] == run)) return;
  const size_t stride = static_cast<size_t>(a.nv) * N;
  const float* slot = a.slots + static_cast<size_t>(min(j, a.nv - 1)) * N;
  Vals<N> s = fill<N>(0.f);
  if (slice == 0) s = ld_floats<N>(slot + (static_cast<size_t>(c) * 2 + 1) * stride);
  // Block k has a piece if the run goes on at its first position.
  constexpr int kAhead = 4;
  bool more = true;
  for (int k0 = c + 1 + slice; more; k0 += 8 * kAhead) {
    Vals<N> v[kAhead];
    bool has[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int k = min(k0 + 8 * u, a.groups - 1);
      has[u] = k0 + 8 * u < a.groups && a.key[k * per_block] == run;
      v[u] = ld_floats<N>(slot + static_cast<size_t>(k) * 2 * stride);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      more = more && has[u];
      if (more) {
#pragma unroll
        for (int i = 0; i < Vals<N>::P; ++i) s.p[i] = add2(s.p[i], v[u].p[i]);
      }
    }
  }
  __syncwarp();
#pragma unroll
  for (int o = 16; o >= 4; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) s.set(i, s.get(i) + __shfl_xor_sync(0xffffffffu, s.get(i), o));
  if (slice == 0 && j < a.nv)
    st_run<G, N>(static_cast<G*>(a.dtable) + run * a.ld + j * N, s, a.scale, a.accumulate);
}

size_t al256(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace

namespace {

struct EmbedArgs {
  RowSet rs;
  TokenView tok;
  const void* table;
  int V, d;
  long long ld_table;
  float scale;
  const void* pos;
  long long ld_pos;
  RowView out;
  unsigned* status;
};

template <typename T, int N, int TL, int NV, int R>
cudaError_t embed_team(const EmbedArgs& a, cudaStream_t st) {
  const long long M = a.rs.rows(), nv = a.d / N, slices = (nv + TL * NV - 1) / (TL * NV);
  const long long teams = (M + R - 1) / R * slices, blocks = (teams + kThreads / TL - 1) / (kThreads / TL);
  if (blocks > 0x7FFFFFFFLL) return cudaErrorInvalidConfiguration;  // more than any memory holds
  k_embed<T, N, TL, NV, R><<<static_cast<unsigned>(blocks), kThreads, 0, st>>>(
      a.rs, a.tok, static_cast<const T*>(a.table), a.V, a.d, a.ld_table, a.scale, static_cast<const T*>(a.pos), a.ld_pos,
      a.out, static_cast<int>(M), static_cast<int>(slices), a.status);
  return cudaGetLastError();
}

template <typename T>
cudaError_t embed_any(const EmbedArgs& a, cudaStream_t st) {
  constexpr int F = 16 / sizeof(T);
  const int es = sizeof(T);
  int vec = std::min(row_vec(a.out, a.rs, a.d, es), row_vec(a.table, 0, a.ld_table, RowSet{1, a.V, nullptr}, a.d, es));
  if (a.pos) vec = std::min(vec, row_vec(a.pos, 0, a.ld_pos, RowSet{1, a.rs.T, nullptr}, a.d, es));
  const int nv = a.d / vec;
  if (vec == F) {
    if (nv <= 8) return embed_team<T, F, 8, 1, 4>(a, st);
    if (nv <= 16) return embed_team<T, F, 8, 2, 4>(a, st);
    if (nv <= 32) return embed_team<T, F, 32, 1, 4>(a, st);
    if (nv <= 64) return embed_team<T, F, 32, 2, 2>(a, st);
    if (nv <= 96) return embed_team<T, F, 32, 3, 2>(a, st);
    return embed_team<T, F, 32, 4, 1>(a, st);
  }
  if (vec == 2) return embed_team<T, 2, 32, 8, 1>(a, st);
  return embed_team<T, 1, 32, 8, 1>(a, st);
}

}  // namespace

cudaError_t launch_embed(RowSet rs, TokenView tok, const void* table, bool bf16_, int V, int d, long long ld_table,
                         float scale, const void* pos, long long ld_pos, RowView out, unsigned* status,
                         cudaStream_t st) {
  const EmbedArgs a{rs, tok, table, V, d, ld_table, scale, pos, ld_pos, out, status};
  return bf16_ ? embed_any<bf16>(a, st) : embed_any<float>(a, st);
}

namespace {

// Positions of a chunk: 32, fewer where that leaves less than 131,072 threads.
int chunk_of(long long M, int nv) {
  int c = kChunk;
  while (c > 8 && M * nv / c < 131072) c >>= 1;
  return c;
}
// Vectors of a column tile.
int tile_of(int nv) { return nv <= 8 ? 8 : nv <= 16 ? 16 : 32; }

template <typename T, typename G, int N>
cudaError_t embed_sum(SumArgs a, cudaStream_t st) {
  a.nv = a.d / N;
  a.chunk = chunk_of(a.M, a.nv);
  a.ct = tile_of(a.nv);
  a.teams = kThreads / a.ct;
  a.tiles = (a.nv + a.ct - 1) / a.ct;
  a.groups = (a.M + a.teams * a.chunk - 1) / (a.teams * a.chunk);
  const long long blocks = static_cast<long long>(a.tiles) * a.groups;
  if (blocks > 0x7FFFFFFFLL) return cudaErrorInvalidConfiguration;
  const int smem = kFlightBytes<T, N> + a.teams * a.chunk * 12 + 16;
  if (cudaError_t e = allow_smem(k_embed_sum<T, G, N>, smem); e != cudaSuccess) return e;
  k_embed_sum<T, G, N><<<static_cast<unsigned>(blocks), kThreads, smem, st>>>(a);
  if (a.groups > 1) {
    const long long join = (static_cast<long long>(a.groups) * ((a.nv + 3) / 4) + kThreads / 32 - 1) / (kThreads / 32);
    k_embed_join<G, N><<<static_cast<unsigned>(join), kThreads, 0, st>>>(a);
  }
  return cudaGetLastError();
}

template <typename T, typename G>
cudaError_t embed_sum_vec(const SumArgs& a, cudaStream_t st) {
  constexpr int F = 16 / sizeof(T);
  // Elements per access of dout, and whether dtable takes as many at once.
  int vec = row_vec(a.dout, a.rs, a.d, sizeof(T));
  const int gb = std::min<int>(16, vec * sizeof(G));
  if (reinterpret_cast<uintptr_t>(a.dtable) % gb || (a.V > 1 && a.ld * static_cast<long long>(sizeof(G)) % gb)) vec = 1;
  if (vec == F) return embed_sum<T, G, F>(a, st);
  if (vec == 2) return embed_sum<T, G, 2>(a, st);
  return embed_sum<T, G, 1>(a, st);
}

struct EmbedWs {
  size_t key, idx, key2, idx2, hist, present, slots, total;
};

EmbedWs embed_ws(int V, int d, long long M) {
  EmbedWs w{};
  if (M == 0) return w;
  const SortPlan p = sort_plan(V, M);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += al256(bytes);
    return o;
  };
  w.key = take(M * 4);
  w.idx = take(M * 4);
  if (M > kTile) {
    w.key2 = take(M * 4);
    w.idx2 = take(M * 4);
    w.hist = take(static_cast<size_t>(p.passes) * std::max(p.blocks, kSortCluster) * p.bins * 4);
    w.present = take(32 * static_cast<size_t>(mark_stride(V)));
  }
  // Enough for every access width: the most groups of positions any of them makes.
  size_t slots = 0;
  for (int n = 1; n <= 8; n *= 2) {
    const int nv = (d + n - 1) / n;
    const long long per = static_cast<long long>(kThreads / tile_of(nv)) * chunk_of(M, nv);
    slots = std::max(slots, static_cast<size_t>((M + per - 1) / per) * 2 * nv * n * 4);
  }
  w.slots = take(slots);
  w.total = at;
  return w;
}

}  // namespace

size_t embed_grad_ws_bytes(int V, int d, long long M) { return embed_ws(V, d, M).total; }

cudaError_t launch_embed_grad(RowSet rs, TokenView tok, RowView dout, bool bf16_, int V, int d, float scale,
                              void* dtable, bool grad_bf16, long long ld_dtable, bool accumulate, void* ws,
                              unsigned* status, cudaStream_t st) {
  const int M = static_cast<int>(rs.rows()), es = grad_bf16 ? 2 : 4;
  if (M == 0 && accumulate) return cudaSuccess;
  const SortPlan p = sort_plan(V, M);
  const EmbedWs w = embed_ws(V, d, M);
  uint8_t* base = static_cast<uint8_t*>(ws);
  auto ints = [&](size_t at) { return reinterpret_cast<int*>(base + at); };

  ZeroArgs z{};
  z.V = V;
  z.table = static_cast<uint8_t*>(dtable);
  z.row_bytes = static_cast<size_t>(d) * es;
  z.stride = V > 1 ? static_cast<size_t>(ld_dtable) * es : z.row_bytes;
  z.unit = reinterpret_cast<uintptr_t>(dtable) % 16 == 0 && z.stride % 16 == 0 && z.row_bytes % 16 == 0 ? 16 : es;
  z.rows = static_cast<int>(std::max<size_t>(kSortWarps, 65536 / z.row_bytes));
  // Part i of n of the rows.
  auto zero_part = [&](int i, int n) {
    z.v0 = static_cast<int>(static_cast<long long>(V) * i / n);
    z.v1 = static_cast<int>(static_cast<long long>(V) * (i + 1) / n);
    z.blocks = accumulate ? 0 : (z.v1 - z.v0 + z.rows - 1) / z.rows;
    return z;
  };

  int *key = ints(w.key), *idx = ints(w.idx);
  if (M <= kTile) {
    zero_part(0, 1);
    auto k = tok.i64 ? k_sort_one<true> : k_sort_one<false>;
    k<<<1 + z.blocks, kSortThreads, 0, st>>>(rs, tok, V, M, p.passes, p.bits, key, idx, z, status);
  } else if (M <= kClusterRows) {
    zero_part(0, 1);
    ClusterSort a{rs,
                  tok,
                  V,
                  M,
                  p.passes,
                  p.bits,
                  (M + kSortCluster * 32 - 1) / (kSortCluster * 32) * 32,
                  {key, ints(w.key2)},
                  {idx, ints(w.idx2)},
                  ints(w.hist),
                  z,
                  status};
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(kSortCluster + (z.blocks + kSortCluster - 1) / kSortCluster * kSortCluster);
    cfg.blockDim = dim3(kSortThreads);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = kSortCluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaError_t e = cudaLaunchKernelEx(&cfg, tok.i64 ? k_sort_cluster<true> : k_sort_cluster<false>, a);
        e != cudaSuccess)
      return e;
    key = a.key[p.passes & 1];
    idx = a.idx[p.passes & 1];
  } else {
    int *key2 = ints(w.key2), *idx2 = ints(w.idx2), *hist = ints(w.hist);
    uint8_t* present = base + w.present;
    const int count_blocks = (M + kCount - 1) / kCount;
    // Marks and the counts of every digit, which lie together.
    if (cudaError_t e = cudaMemsetAsync(base + w.hist, 0, w.slots - w.hist, st); e != cudaSuccess) return e;
    auto k = tok.i64 ? k_sort_keys<true> : k_sort_keys<false>;
    k<<<count_blocks, kThreads, 0, st>>>(rs, tok, V, M, p.bins, p.per_block, key, present, hist, status);
    z.present = present;
    const int parts = 2 * p.passes - 1;
    for (int s = 0; s < p.passes; ++s) {
      if (s > 0) {
        zero_part(2 * s - 1, parts);
        hist += static_cast<size_t>(p.blocks) * p.bins;
        k_sort_count<<<count_blocks + z.blocks, kSortThreads, 0, st>>>(key, M, s * p.bits, p.bins, p.per_block,
                                                                       count_blocks, hist, z);
      }
      zero_part(2 * s, parts);
      k_sort_place<<<p.blocks + z.blocks, kSortThreads, 0, st>>>(key, s ? idx : nullptr, M, s * p.bits, p.bins, p.per_block,
                                                             p.blocks, hist, key2, idx2, z);
      std::swap(key, key2);
      std::swap(idx, idx2);
    }
  }
  if (M == 0) return cudaGetLastError();
  SumArgs a{};
  a.rs = flat(dout, rs) ? RowSet{1, M, nullptr} : RowSet{rs.B, rs.T, nullptr};
  a.dout = dout;
  a.key = key;
  a.idx = idx;
  a.M = M;
  a.V = V;
  a.d = d;
  a.scale = scale;
  a.dtable = dtable;
  a.ld = ld_dtable;
  a.accumulate = accumulate;
  a.slots = reinterpret_cast<float*>(base + w.slots);
  if (bf16_) return grad_bf16 ? embed_sum_vec<bf16, bf16>(a, st) : embed_sum_vec<bf16, float>(a, st);
  return grad_bf16 ? embed_sum_vec<float, bf16>(a, st) : embed_sum_vec<float, float>(a, st);
}
