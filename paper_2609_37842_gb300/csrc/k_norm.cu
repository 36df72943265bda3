// Normalisation over the channels of each row (layer norm and RMS norm) and its
// gradient. With mu = mean(x) (0 for RMS), r = (mean((x - mu)^2) + eps)^(-1/2),
// xh = (x - mu) r:
//   y  = xh w + b,
//   dx = r (g - mean(g) - xh mean(g xh)),  g = dy w  (RMS: no mean(g)),
//   dw = sum over tokens of dy xh,  db = sum over tokens of dy.
// Statistics and sums are fp32; the variance is the mean of squared differences
// from the mean, not a difference of moments. HBM-bound: a few flop per byte.
//
// A row is worked on by a team: a warp, a part of one, or a whole block, each
// thread holding vectors of the row in registers, so x (and dy) are read once.
// Rows that 16-byte accesses do not fit are loaded two or one elements at a time;
// rows too wide for registers take several passes.
#include <algorithm>

#include "rows_dev.cuh"

using namespace eogp;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kWarpTeams = 4;     // warp teams of a block
constexpr int kMaxWarps = 16;     // of a block team
constexpr int kOwnStages = 3;     // rows ahead where threads copy their own elements

// Threads of a team: 32, or the block (TEAM = 0).
template <int TEAM>
__device__ __forceinline__ int team_lane() {
  return TEAM ? threadIdx.x & (TEAM - 1) : threadIdx.x;
}
template <int TEAM>
__device__ __forceinline__ int team_threads() {
  return TEAM ? TEAM : blockDim.x;
}
template <int TEAM>
__device__ __forceinline__ void team_sync() {
  if constexpr (TEAM)
    __syncwarp();
  else
    __syncthreads();
}

// Sum over the team, the same in every thread and in a fixed order. Block teams
// synchronise once, so `part` must not be the one of the call before.
template <int TEAM, int K>
__device__ __forceinline__ void team_sum(float (&v)[K], float (*part)[kMaxWarps]) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int o = (TEAM ? TEAM : 32) / 2; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  }
  if constexpr (TEAM == 0) {
    const int nw = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) part[k][threadIdx.x >> 5] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s = 0.f;
      for (int w = 0; w < nw; ++w) s += part[k][w];
      v[k] = s;
    }
  }
}

// A team's ring of row stages in shared memory, one mbarrier each. Thread 0 of the
// team fills a stage with the rows' bulk copies; every thread waits for every stage
// in turn. A stage is filled again after the team's barrier in the row after it, by
// which time every thread is done with it; so a barrier is never more than one phase
// ahead of a thread that waits on it.
struct Ring {
  uint8_t* data;
  uint64_t* full;
  int stages, stage_bytes, slot, phase;
  bool dead;  // a wait ran out: the status word is set, results no longer matter
};

__device__ __forceinline__ void ring_wait(Ring& q, unsigned* status) {
  if (q.dead || mbar_wait(&q.full[q.slot], q.phase, status)) return;
  q.dead = true;
  // No more is filled; what is on its way arrives (again waited for with a limit)
  // before the block gives up its memory.
  for (int k = 1; k < q.stages; ++k) {
    const int s = q.slot + k;
    mbar_wait(&q.full[s % q.stages], q.phase ^ (s >= q.stages), status, EOGP_WAIT_CYCLES / 16);
  }
}
__device__ __forceinline__ void ring_next(Ring& q) {
  if (++q.slot == q.stages) {
    q.slot = 0;
    q.phase ^= 1;
  }
}

// -------------------------------------------------------------------- forward
struct NormArgs {
  RowSet rs;
  int M;
  RowView x;
  const void *w, *bias;
  bool pbf;
  float eps;
  int d;
  RowView y;
  float *mean, *rstd;
};

// A team holds a row as raw words in registers: all its loads are in flight at
// once, the passes for the mean, the variance and the result read registers, and
// other teams' loads cover the sums. Weights come from L1. At most 64 registers a
// thread, so that 1,024 threads share a multiprocessor: with 16 vectors a thread
// (164 registers) a warp waits for its sums with too few others to cover it (4096
// channels of bf16: 8 vectors a thread and two warps take 8 % less). USUAL: weight
// (and, for layer norm, bias) given and of the rows' type; the choice at each vector
// otherwise fills the issue slots (65,536 rows of 4096 bf16: 185 us with it, 161 us
// without). The limit makes ten of the bf16 kernels and one of fp32 spill, up to 96
// bytes stored and 264 loaded again a thread (8 vectors, layer norm), from and to L1.
// Measured, 0.5 GB in and out: 141 to 149 us (1.0 of the copy rate) in fp32 up to 16,384
// channels, 149 us (0.99) for 768 to 8192 channels of bf16, 153 to 233 us for 64 to 512.
template <typename T, int N, int NV, int TEAM, bool RMS, bool USUAL>
__global__ void __launch_bounds__(TEAM ? 128 : 512, TEAM ? 8 : 2) k_norm(const NormArgs a) {
  __shared__ float part[2][1][kMaxWarps];
  constexpr int teams = TEAM ? 128 / (TEAM ? TEAM : 1) : 1;
  const int lane = team_lane<TEAM>(), tt = team_threads<TEAM>();
  const int r0 = blockIdx.x * teams + (TEAM ? threadIdx.x / (TEAM ? TEAM : 1) : 0);
  const bool on = r0 < a.M;  // teams smaller than a warp stay for its shuffles
  if (TEAM != 8 && !on) return;
  const int r = on ? r0 : 0;
  int b, t;
  locate(a.rs, r, b, t);
  const bool kept = on && row_kept(a.rs, b, t);
  if (TEAM != 8 && !kept) {
    T* yr = row_out<T>(a.y, b, t);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * tt + lane) * N;
      if (c < a.d) st_vals<T, N>(yr + c, fill<N>(0.f));
    }
    if (lane == 0) {
      if (a.mean) a.mean[r] = 0.f;
      if (a.rstd) a.rstd[r] = 0.f;
    }
    return;
  }
  Raw<T, N> raw[NV];
  const T* xr = row_of<T>(a.x, b, t);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * tt + lane) * N;
    raw[j] = Raw<T, N>{};
    if (c < a.d && kept) raw[j] = ld_raw<T, N>(xr + c);
  }
  const float inv_d = 1.0f / a.d;
  float mu = 0.f;
  if (!RMS) {
    typename Vals<N>::E s = Vals<N>::all(0.f);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const Vals<N> v = unpack<T, N>(raw[j]);
#pragma unroll
      for (int i = 0; i < Vals<N>::P; ++i) s = add2(s, v.p[i]);
    }
    float m[1] = {sum2(s)};
    team_sum<TEAM>(m, part[0]);
    mu = m[0] * inv_d;
  }
  typename Vals<N>::E q = Vals<N>::all(0.f);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if ((j * tt + lane) * N < a.d) {
      const Vals<N> v = unpack<T, N>(raw[j]);
#pragma unroll
      for (int i = 0; i < Vals<N>::P; ++i) {
        const typename Vals<N>::E e = add2(v.p[i], Vals<N>::all(-mu));
        q = fma2(e, e, q);
      }
    }
  }
  float var[1] = {sum2(q)};
  team_sum<TEAM>(var, part[1]);
  const float rs_ = kept ? 1.0f / sqrtf(fmaf(var[0], inv_d, a.eps)) : 0.f;
  if (!on) return;
  T* yr = row_out<T>(a.y, b, t);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * tt + lane) * N;
    if (c < a.d) {
      const Vals<N> v = unpack<T, N>(raw[j]);
      Vals<N> w, bi = fill<N>(0.f);
      if constexpr (USUAL) {
        w = unpack<T, N>(ld_keep<T, N>(static_cast<const T*>(a.w) + c));
        if (!RMS) bi = unpack<T, N>(ld_keep<T, N>(static_cast<const T*>(a.bias) + c));
      } else {
        w = ld_param<N>(a.w, a.pbf, c, 1.f);
        bi = ld_param<N>(a.bias, a.pbf, c, 0.f);
      }
      Vals<N> o = fill<N>(0.f);
      if (kept) {
#pragma unroll
        for (int i = 0; i < Vals<N>::P; ++i) {
          typename Vals<N>::E e = v.p[i];
          if (!RMS) e = add2(e, Vals<N>::all(-mu));
          o.p[i] = fma2(mul2(e, Vals<N>::all(rs_)), w.p[i], bi.p[i]);
        }
      }
      st_vals<T, N>(yr + c, o);
    }
  }
  if (lane == 0) {
    if (a.mean) a.mean[r] = mu;
    if (a.rstd) a.rstd[r] = rs_;
  }
}

// ------------------------------------------------------------------- gradient
// Rows are numbered over groups (an example each, or the whole batch) of `rpg`
// rows, and split evenly over the blocks, `per` consecutive rows each: a block's
// rows cover whole groups and at most two pieces of groups that other blocks
// share. Sums of a whole group are final; those of a piece go to the block's
// slot 0 (the group began in an earlier block) or 1, [2][d] floats each, and
// k_norm_grad_join adds a group's pieces in order.
struct GradArgs {
  NormGrad g;
  int M, rpg, per;
  float* slots;
  bool by_work;  // rows are cut by work, not `per` a block
  int* starts;   // then: first row of each block, and M, for k_norm_grad_join; NULL without sums
  int stages;
  unsigned* status;
};

__device__ __forceinline__ void put_sums(const NormGrad& g, int e, int c, float sw, float sb) {
  const size_t at = static_cast<size_t>(e) * g.ld_dparam + c;
  if (g.dweight) g.dweight[at] = g.accumulate ? g.dweight[at] + sw : sw;
  if (g.dbias) g.dbias[at] = g.accumulate ? g.dbias[at] + sb : sb;
}

// A place in the rows: row r is token t of example b.
struct RowAt {
  int r, b, t;
};
__device__ __forceinline__ RowAt row_at(const RowSet& rs, int r) {
  RowAt p{r, 0, 0};
  locate(rs, r, p.b, p.t);
  return p;
}
__device__ __forceinline__ void advance(const RowSet& rs, RowAt& p, int by) {
  p.r += by;
  p.t += by;
  while (p.t >= rs.T) {
    p.t -= rs.T;
    ++p.b;
  }
}
// On to the first kept row of p, p + step, .. below hi.
__device__ __forceinline__ void to_kept(const RowSet& rs, RowAt& p, int step, int hi) {
  if (!rs.lengths) return;
  while (p.r < hi && p.t >= rs.lengths[p.b]) advance(rs, p, (rs.T - p.t + step - 1) / step * step);
}

// Work of an example, in accesses per element: a kept row reads x and dy and writes
// dx, one of padding writes dx at most; the sums cost about as much as a few rows.
constexpr int kSumsWork = 8;
__device__ __forceinline__ long long example_work(const RowSet& rs, int b, int kept, int padding) {
  const int n = max(0, min(rs.T, rs.lengths[b]));
  return kSumsWork + static_cast<long long>(n) * kept + static_cast<long long>(rs.T - n) * padding;
}

// Rows [at[0], at[1]) of block k of n, cut so that every block has the same work:
// block k starts where k / n of the work lies before.
__device__ __forceinline__ void cut_rows(const RowSet& rs, bool dx, int k, int n, int M, int* at) {
  __shared__ long long sums[kMaxWarps];
  const int kept = dx ? 3 : 2, padding = dx ? 1 : 0, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int each = (rs.B - 1) / static_cast<int>(blockDim.x) + 1;  // examples a thread adds up
  const int b0 = static_cast<int>(min(static_cast<long long>(rs.B), static_cast<long long>(threadIdx.x) * each));
  const int b1 = static_cast<int>(min(static_cast<long long>(rs.B), static_cast<long long>(b0) + each));
  long long own = 0;
#pragma unroll 8
  for (int b = b0; b < b1; ++b) own += example_work(rs, b, kept, padding);
  long long upto = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += u;
  }
  if (lane == 31) sums[warp] = upto;
  if (threadIdx.x < 2) at[threadIdx.x] = M;
  __syncthreads();
  long long total = 0, before = upto - own;
  for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) {
    if (w < warp) before += sums[w];
    total += sums[w];
  }
  for (int i = 0; i < 2; ++i) {
    const long long want = total * (k + i) / n;
    if (k + i == n || want < before || want >= before + own) continue;  // another thread's examples hold it
    long long left = want - before;
    for (int b = b0; b < b1; ++b) {
      const long long work = example_work(rs, b, kept, padding);
      if (left < work) {
        const long long rows = static_cast<long long>(max(0, min(rs.T, rs.lengths[b]))) * kept;
        left = max(0LL, left - kSumsWork);
        const long long t = left <= rows ? (left + kept - 1) / kept : rows / kept + (left - rows);
        at[i] = static_cast<int>(static_cast<long long>(b) * rs.T + t);
        break;
      }
      left -= work;
    }
  }
  __syncthreads();
}

// The team's lanes of a warp (for a block team: the warp); other teams of the warp may
// be elsewhere.
template <int TEAM>
__device__ __forceinline__ unsigned lane_mask() {
  constexpr int L = TEAM ? TEAM : 32;
  return L == 32 ? 0xffffffffu : ((1u << (L & 31)) - 1u) << (threadIdx.x & 31 & ~(L - 1));
}
// Sum over them.
template <int TEAM>
__device__ __forceinline__ float lane_sum(float v) {
#pragma unroll
  for (int o = (TEAM ? TEAM : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(lane_mask<TEAM>(), v, o);
  return v;
}

// Two sums over the block, the same in every thread and in a fixed order.
__device__ __forceinline__ float2 block_sum2(float2 v, float2* part) {
  v.x = warp_sum(v.x);
  v.y = warp_sum(v.y);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < static_cast<int>(blockDim.x >> 5); ++w) v = add2(v, part[w]);
  return v;
}

// Persistent teams: a team's rows arrive in a ring of shared-memory stages filled
// by bulk copies several rows ahead. A row is gone through twice in its stage: for
// the sums over channels and over rows, with p = dy (x - mu),
//   s1 = sum dy w,  s2 = sum p w,  dw += r p,  db += dy,
// then for dx = r dy w + k1 (r (x - mu)) + k0, k1 = -r (r s2 / d), k0 = -r s1 / d. x is
// centred first: k1 (r x) and k1 (r mu) apart would cancel in rows whose mean is many
// times their spread (fp32, mean 1000 times the spread: an error of 3,000 u of the
// row's scale instead of 8 u, u = 2^-24).
// The row itself is not kept in registers: with it, fewer rows are in flight. The
// weights are (WREG, of the rows' type) or lie in shared memory in fp32, 0 beyond the
// row, where threads read the row's last vector again. What a thread does once a row
// (waits, sums, addresses) is as much as the work on ten elements, so it has up to 32.
// Measured, bytes against the copy rate: 0.89 for 768 and 1024 channels of bf16, 0.85
// (layer) and 0.94 (RMS) for 4096, 0.92 for 2048 and 4096 of fp32; narrow rows 0.77 to
// 0.87 in fp32 and 0.60 to 0.87 in bf16, whose kernels for 17 to 64 vectors spill up to
// 104 bytes a thread.
template <typename T, int N, int NV, int TEAM, bool RMS, bool BULK, bool WREG, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) k_norm_grad(const GradArgs a) {
  using V = Vals<N>;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ uint64_t bars[BULK ? kWarpTeams * 8 : 1];
  __shared__ float2 part[2][kMaxWarps];
  __shared__ int cut[2];
  const NormGrad& g = a.g;
  const RowSet rs = g.rs;
  const int lane = team_lane<TEAM>(), tt = team_threads<TEAM>();
  constexpr int teams = TEAM ? 32 * kWarpTeams / (TEAM ? TEAM : 1) : 1;
  const int team = TEAM ? threadIdx.x / (TEAM ? TEAM : 1) : 0;
  const int d = g.d, width = NV * tt * N;
  const uint32_t row_bytes = static_cast<uint32_t>(d) * sizeof(T);
  int lo = static_cast<int>(blockIdx.x * static_cast<long long>(a.per));
  int hi = static_cast<int>(min(static_cast<long long>(a.M), lo + static_cast<long long>(a.per)));
  if (a.by_work) {
    cut_rows(rs, g.dx.p != nullptr, blockIdx.x, gridDim.x, a.M, cut);
    lo = cut[0];
    hi = cut[1];
    if (a.starts && threadIdx.x < 2) a.starts[blockIdx.x + threadIdx.x] = cut[threadIdx.x];
  }
  // Weights; the place where warp teams add their sums up, one after the other; rings.
  float* const ws = reinterpret_cast<float*>(smem);
  float2* const join = reinterpret_cast<float2*>(smem + (WREG ? 0 : width * 4));
  uint8_t* const ring0 = smem + width * ((WREG ? 0 : 4) + (TEAM ? 8 : 0));
  Raw<T, N> wr[WREG ? NV : 1];
  if constexpr (WREG) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * tt + lane) * N;
      wr[j] = pack_raw<T, N>(fill<N>(c < d ? 1.f : 0.f));
      if (g.weight && c < d) wr[j] = ld_keep<T, N>(static_cast<const T*>(g.weight) + c);
    }
  } else {
    for (int c = threadIdx.x; c < width; c += blockDim.x)
      ws[c] = c < d ? param_at(g.weight, g.param_bf16, c, 1.f) : 0.f;
  }
  Ring q{};
  if constexpr (BULK) {
    q = Ring{ring0 + static_cast<size_t>(team) * a.stages * 2 * row_bytes, bars + team * 8, a.stages,
             static_cast<int>(2 * row_bytes), 0, 0, false};
    if (lane == 0) {
      for (int s = 0; s < a.stages; ++s) mbar_init(&q.full[s], 1);
      fence_barrier_init();
    }
  }
  __syncthreads();
  RowAt p = row_at(rs, min(lo + team, a.M - 1));
  p.r = lo + team;
  int at[NV];  // first channel of vector j, within the row
#pragma unroll
  for (int j = 0; j < NV; ++j) at[j] = min((j * tt + lane) * N, d - N);
  RowAt ahead = p;  // next row to be copied (BULK: by thread 0)
  // Places of a thread's vectors when it copies them itself: of its own, so that it
  // needs no other thread's copies.
  T* const own = reinterpret_cast<T*>(ring0) + static_cast<size_t>(team) * kOwnStages * 2 * width + lane * N;
  auto issue = [&](int s) {
    to_kept(rs, ahead, teams, hi);
    if (ahead.r >= hi) return;
    if constexpr (!BULK) {
      const T* const xr = row_of<T>(g.x, ahead.b, ahead.t);
      const T* const dyr = row_of<T>(g.dy, ahead.b, ahead.t);
      T* const to = own + static_cast<size_t>(s) * 2 * width;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        copy_async<T, N>(reinterpret_cast<Raw<T, N>*>(to + j * tt * N), xr + at[j]);
        copy_async<T, N>(reinterpret_cast<Raw<T, N>*>(to + width + j * tt * N), dyr + at[j]);
      }
      advance(rs, ahead, teams);
      return;
    }
    mbar_arrive_expect_tx(&q.full[s], 2 * row_bytes);
    uint8_t* to = q.data + static_cast<size_t>(s) * q.stage_bytes;
    bulk_load(to, row_of<T>(g.x, ahead.b, ahead.t), row_bytes, &q.full[s]);
    bulk_load(to + row_bytes, row_of<T>(g.dy, ahead.b, ahead.t), row_bytes, &q.full[s]);
    advance(rs, ahead, teams);
  };
  if (!BULK || lane == 0)
    for (int s = 0; s < (BULK ? a.stages : kOwnStages); ++s) {
      issue(s);
      if (!BULK) commit_async();
    }
  // Moves on to the next kept row, writing the rows of padding before it.
  auto skip = [&] {
    if (!rs.lengths) return;
    while (p.r < hi && p.t >= rs.lengths[p.b]) {
      if (g.dx.p) {
        T* o = row_out<T>(g.dx, p.b, p.t);
        for (int c = lane * N; c < d; c += tt * N) st_vals<T, N>(o + c, fill<N>(0.f));
      }
      advance(rs, p, teams);
    }
  };
  skip();
  const float* const wl = ws + lane * N;
  V dw[NV], db[NV];
  const float inv_d = 1.0f / d;
  const bool sums = g.dweight || g.dbias, want_db = g.dbias != nullptr;
  int parity = 0, back = -1;  // stage of the row before
  float mu_next = 0.f, rs_next = 0.f;
  auto stats = [&](int row) {
    if (row < hi) {
      if (!RMS) mu_next = __ldg(g.mean + row);
      rs_next = __ldg(g.rstd + row);
    }
  };
  stats(p.r);
  for (int p0 = lo; p0 < hi;) {
    const int e = p0 / a.rpg;
    const int p1 = static_cast<int>(min(static_cast<long long>(hi), (e + 1LL) * a.rpg));  // end of the piece
#pragma unroll
    for (int j = 0; j < NV; ++j) dw[j] = db[j] = fill<N>(0.f);
    while (p.r < p1) {
      const float mu = mu_next, rstd = rs_next;
      T* const o = g.dx.p ? row_out<T>(g.dx, p.b, p.t) : nullptr;
      const T *xr, *dyr;
      if constexpr (BULK) {
        ring_wait(q, a.status);
        xr = reinterpret_cast<const T*>(q.data + static_cast<size_t>(q.slot) * q.stage_bytes);
        dyr = xr + d;
      } else {
        wait_async<kOwnStages - 1>();
        // dx may be x or dy: lanes beyond a row have copied its last vector for
        // themselves, which another lane writes over.
        if (TEAM && d < width) __syncwarp(lane_mask<TEAM>());
        xr = own + static_cast<size_t>(q.slot) * 2 * width;
        dyr = xr + width;
      }
      advance(rs, p, teams);
      skip();
      stats(p.r);
      auto load = [&](const T* from, int j) {
        return unpack<T, N>(*reinterpret_cast<const Raw<T, N>*>(from + (BULK ? at[j] : j * tt * N)));
      };
      auto weight = [&](int j) {
        if constexpr (WREG)
          return unpack<T, N>(wr[j]);
        else
          return ld_floats<N>(wl + j * tt * N);
      };
      typename V::E s1 = V::all(0.f), s2 = V::all(0.f);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const V x = load(xr, j), dy = load(dyr, j), w = weight(j);
#pragma unroll
        for (int i = 0; i < V::P; ++i) {
          const typename V::E pr = mul2(dy.p[i], RMS ? x.p[i] : add2(x.p[i], V::all(-mu)));
          dw[j].p[i] = fma2(pr, V::all(rstd), dw[j].p[i]);
          s2 = fma2(pr, w.p[i], s2);
          if (!RMS) s1 = fma2(dy.p[i], w.p[i], s1);
        }
        if (want_db) {
#pragma unroll
          for (int i = 0; i < V::P; ++i) db[j].p[i] = add2(db[j].p[i], dy.p[i]);
        }
      }
      float2 sum = make_float2(sum2(s1), sum2(s2));
      if (o && TEAM == 0) {
        sum = block_sum2(sum, part[parity]);
      } else if (o) {
        sum = make_float2(lane_sum<TEAM>(sum.x), lane_sum<TEAM>(sum.y));
      }
      if (BULK && !(o && TEAM == 0)) team_sync<TEAM>();
      asm volatile("" ::: "memory");  // the row is read again, not kept
      if constexpr (BULK) {
        if (lane == 0 && back >= 0 && !q.dead) issue(back);
        back = q.slot;
        ring_next(q);
      }
      if (o) {
        const float k1 = -rstd * (rstd * sum.y * inv_d), k0 = -rstd * (sum.x * inv_d);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const V x = load(xr, j), w = weight(j);
          V dy = load(dyr, j);
#pragma unroll
          for (int i = 0; i < V::P; ++i) {
            const typename V::E gv = mul2(dy.p[i], w.p[i]);
            const typename V::E xc = RMS ? x.p[i] : add2(x.p[i], V::all(-mu));
            dy.p[i] = fma2(mul2(xc, V::all(rstd)), V::all(k1), fma2(gv, V::all(rstd), V::all(RMS ? 0.f : k0)));
          }
          if ((j * tt + lane) * N < d) st_vals<T, N>(o + at[j], dy);
        }
      }
      if constexpr (!BULK) {
        issue(q.slot);
        commit_async();
        if (++q.slot == kOwnStages) q.slot = 0;
      }
      parity ^= 1;
    }
    if (sums) {
      const bool begins = static_cast<long long>(e) * a.rpg >= lo, ends = (e + 1LL) * a.rpg <= hi;
      float* slot = a.slots + (static_cast<size_t>(blockIdx.x) * 2 + (begins ? 1 : 0)) * 2 * d;
      auto put = [&](int c, float sw, float sb) {
        if (begins && ends) {
          put_sums(g, e, c, sw, sb);
        } else {
          slot[c] = sw;
          slot[d + c] = sb;
        }
      };
      if constexpr (TEAM == 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int c = (j * tt + lane) * N + i;
            if (c < d) put(c, dw[j].get(i), db[j].get(i));
          }
      } else {
        for (int k = 0; k < teams; ++k) {
          if (team == k) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
              for (int i = 0; i < N; ++i) {
                const int c = (j * tt + lane) * N + i;
                if (c < d) {
                  float2 v = make_float2(dw[j].get(i), db[j].get(i));
                  if (k > 0) v = add2(join[c], v);
                  join[c] = v;
                }
              }
          }
          __syncthreads();
        }
        for (int c = threadIdx.x; c < d; c += blockDim.x) put(c, join[c].x, join[c].y);
        __syncthreads();
      }
    }
    p0 = p1;
  }
}

// Adds the pieces of the groups that several blocks share, in block order. A group
// of many pieces: each of 16 warps of a block sums a contiguous run of them for 32
// channels, and the runs are added in order. Groups of no rows (no block) get 0.
constexpr int kJoinSlices = 16;

template <int SLICES>
__global__ void __launch_bounds__(SLICES == 1 ? kThreads : 32 * SLICES) k_norm_grad_join(const GradArgs a, int groups,
                                                                                           int blocks) {
  __shared__ float2 acc[SLICES][32];
  extern __shared__ int starts[];
  const int lane = threadIdx.x & 31, slice = SLICES == 1 ? 0 : threadIdx.x >> 5, d = a.g.d;
  const int c = SLICES == 1 ? blockIdx.x * kThreads + threadIdx.x : blockIdx.x * 32 + lane;
  if (a.starts) {
    for (int k = threadIdx.x; k <= blocks; k += blockDim.x) starts[k] = a.starts[k];
    __syncthreads();
  }
  auto start = [&](int k) {
    return a.starts ? starts[k] : static_cast<int>(min(static_cast<long long>(a.M), static_cast<long long>(k) * a.per));
  };
  // The first block that starts at row r or later.
  auto from = [&](long long r) {
    if (!a.starts) return static_cast<int>((r + a.per - 1) / a.per);
    int k0 = 0, k1 = blocks;
    while (k0 < k1) {
      const int k = (k0 + k1) / 2;
      if (starts[k] >= r)
        k1 = k;
      else
        k0 = k + 1;
    }
    return k0;
  };
  for (int e = blockIdx.y; e < groups; e += gridDim.y) {
    const long long r0 = static_cast<long long>(e) * a.rpg, r1 = r0 + a.rpg;
    // Blocks b0 .. b1 - 1, of which some may have no rows.
    const int b0 = a.rpg ? from(r0 + 1) - 1 : 0, b1 = a.rpg ? from(r1) : 0;
    if (b1 > b0 && start(b0 + 1) >= r1) continue;  // one block had it whole
    const int each = (b1 - b0 + SLICES - 1) / SLICES;
    float2 s = make_float2(0.f, 0.f);
    if (c < d)
#pragma unroll 4
      for (int k = b0 + slice * each; k < min(b1, b0 + (slice + 1) * each); ++k) {
        const float* slot = a.slots + (static_cast<size_t>(k) * 2 + (k == b0)) * 2 * d;  // it began in block b0
        const float2 v = make_float2(slot[c], slot[d + c]);
        s = add2(s, !a.starts || starts[k] < starts[k + 1] ? v : make_float2(0.f, 0.f));
      }
    if constexpr (SLICES > 1) {
      acc[slice][lane] = s;
      __syncthreads();
      if (slice == 0)
        for (int k = 1; k < SLICES; ++k) s = add2(s, acc[k][lane]);
      __syncthreads();
    }
    if (slice == 0 && c < d) put_sums(a.g, e, c, s.x, s.y);
  }
}

// ---------------------------------------------- rows too wide for registers
// One block per row, three passes over the row (the later ones from cache), an element
// a load: 20,001 channels of bf16 0.28 of the copy rate.
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

// dx: one block per row, two passes over the row. With the sums below, which read x and
// dy again: 12,288 and 16,384 channels of fp32 0.26 of the copy rate, 24,576 of bf16 0.19.
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

// dw, db: one thread per channel sums the rows of a block's run, with the pieces
// and slots of k_norm_grad. Channels along grid.x, which has room for any width; the runs,
// at most kGradOcc a multiprocessor, along grid.y.
template <typename T, bool RMS>
__global__ void __launch_bounds__(kThreads) k_norm_dparam_rows(const GradArgs a) {
  const NormGrad& g = a.g;
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= g.d) return;
  const long long first = static_cast<long long>(blockIdx.y) * a.per;
  const int hi = static_cast<int>(min(static_cast<long long>(a.M), first + a.per)), lo = static_cast<int>(first);
  for (int p0 = lo; p0 < hi;) {
    const int e = p0 / a.rpg;
    const int p1 = static_cast<int>(min(static_cast<long long>(hi), (e + 1LL) * a.rpg));
    float sw = 0.f, sb = 0.f;
    for (int r = p0; r < p1; ++r) {
      int b, t;
      locate(g.rs, r, b, t);
      if (!row_kept(g.rs, b, t)) continue;
      const float dy = to_f32(row_of<T>(g.dy, b, t)[c]);
      const float xh = (to_f32(row_of<T>(g.x, b, t)[c]) - (RMS ? 0.f : g.mean[r])) * g.rstd[r];
      sw = fmaf(dy, xh, sw);
      sb += dy;
    }
    const bool begins = static_cast<long long>(e) * a.rpg >= lo, ends = (e + 1LL) * a.rpg <= hi;
    if (begins && ends) {
      put_sums(g, e, c, sw, sb);
    } else {
      float* slot = a.slots + (static_cast<size_t>(blockIdx.y) * 2 + (begins ? 1 : 0)) * 2 * g.d;
      slot[c] = sw;
      slot[g.d + c] = sb;
    }
    p0 = p1;
  }
}

// ------------------------------------------------------------------ launching
int ceil_div(long long a, long long b) { return static_cast<int>((a + b - 1) / b); }

// How a row of d elements is worked on by the gradient: NV vectors of n elements a
// thread by a warp (team 32) or a block of `threads`; n = 0: too wide.
struct Shape {
  int n, nv, team, threads;
};

// `vec`: elements per access the arrays allow; es: element bytes. 16-byte vectors:
// a warp of up to `warp_nv` of them a thread, or a block of `block_nv` a thread.
Shape grad_shape(int d, int vec, int es, int warp_nv, int block_nv) {
  const int nv = ceil_div(d, vec);
  if (vec == 16 / es) {
    if (nv <= 32 * warp_nv) return Shape{vec, ceil_div(nv, 32), 32, 32 * kWarpTeams};
    const int th = ceil_div(nv, 32 * block_nv) * 32;
    return th <= 512 ? Shape{vec, block_nv, 0, th} : Shape{0, 0, 0, 0};
  }
  const int th = ceil_div(nv, 32 * 8) * 32;
  return th <= 512 ? Shape{vec, 8, 0, th} : Shape{0, 0, 0, 0};
}

// Shared memory that the blocks of a multiprocessor share: 228 KB less 1 KB and the
// static arrays of each.
constexpr size_t kSmemPerSm = 220 * 1024;

// Blocks of `threads` that a multiprocessor's registers and threads hold, at most
// `most`: persistent blocks beyond the resident ones would run as a second wave.
template <typename F>
int resident(F k, int threads, int most) {
  cudaFuncAttributes at;
  if (cudaFuncGetAttributes(&at, k) != cudaSuccess || at.numRegs < 1) return 1;
  // Each of the four parts of a multiprocessor gives its warps 16,384 registers.
  const int warps = 4 * (16384 / ((at.numRegs + 7) / 8 * 8 * 32));
  return std::max(1, std::min({most, warps / (threads / 32), 2048 / threads}));
}

// Examples as one run of rows where no lengths and no strides tell them apart.
template <typename... V>
RowSet flatten(const RowSet& rs, const V&... v) {
  if (!rs.lengths && (flat(v, rs) && ...)) return RowSet{1, static_cast<int>(rs.rows()), nullptr};
  return rs;
}

template <typename T, int N, int NV, int TEAM>
cudaError_t norm_team(bool rms, const NormArgs& a, int threads, cudaStream_t st) {
  const bool usual = a.w && a.pbf == (sizeof(T) == 2) && (rms ? !a.bias : a.bias != nullptr);
  auto k = rms ? (usual ? k_norm<T, N, NV, TEAM, true, true> : k_norm<T, N, NV, TEAM, true, false>)
               : (usual ? k_norm<T, N, NV, TEAM, false, true> : k_norm<T, N, NV, TEAM, false, false>);
  k<<<ceil_div(a.M, TEAM ? 128 / (TEAM ? TEAM : 1) : 1), threads, 0, st>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t norm_launch(bool rms, const NormArgs& a, int num_sms, cudaStream_t st) {
  constexpr int F = 16 / sizeof(T);
  const int es = sizeof(T);
  int vec = std::min(row_vec(a.x, a.rs, a.d, es), row_vec(a.y, a.rs, a.d, es));
  const RowSet one{1, 1, nullptr};
  const int pes = a.pbf ? 2 : 4;
  const int pvec = std::min(row_vec(a.w, 0, 0, one, 8, pes), row_vec(a.bias, 0, 0, one, 8, pes));
  if (vec > 1 && pvec < 2) vec = 1;
  if (vec == F && pvec < 16 / pes) vec = 2;
  const int nv = ceil_div(a.d, vec);
  if (vec == F) {
    // Few rows: their latency counts, so a row gets a block of two vectors a thread
    // (one row of 4096 bf16: 2.3 us against 5.6 us for 16 vectors a thread).
    if (nv > 64 && nv <= 1024 && a.M <= 4 * num_sms) return norm_team<T, F, 2, 0>(rms, a, ceil_div(nv, 64) * 32, st);
    if (nv <= 8) return norm_team<T, F, 1, 8>(rms, a, 128, st);
    if (nv <= 16) return norm_team<T, F, 2, 8>(rms, a, 128, st);
    if (nv <= 32) return norm_team<T, F, 4, 8>(rms, a, 128, st);
    if (nv <= 64) return norm_team<T, F, 2, 32>(rms, a, 128, st);
    if (nv <= 96) return norm_team<T, F, 3, 32>(rms, a, 128, st);
    if (nv <= 128) return norm_team<T, F, 4, 32>(rms, a, 128, st);
    if (nv <= 192) return norm_team<T, F, 6, 32>(rms, a, 128, st);
    if (nv <= 256) return norm_team<T, F, 8, 32>(rms, a, 128, st);
    // A block team of as few warps as hold the row at 8 vectors a thread.
    const int warps = ceil_div(nv, 8 * 32), th = warps * 32;
    if (warps <= kMaxWarps) {
      const int per = ceil_div(nv, th);
      if (per <= 5) return norm_team<T, F, 5, 0>(rms, a, th, st);
      if (per == 6) return norm_team<T, F, 6, 0>(rms, a, th, st);
      if (per == 7) return norm_team<T, F, 7, 0>(rms, a, th, st);
      return norm_team<T, F, 8, 0>(rms, a, th, st);
    }
  } else if (vec == 2) {
    if (nv <= 256) return norm_team<T, 2, 8, 32>(rms, a, 128, st);
    if (nv <= 512) return norm_team<T, 2, 16, 32>(rms, a, 128, st);
    const int th = ceil_div(nv, 16 * 32) * 32;
    if (th <= 512) return norm_team<T, 2, 16, 0>(rms, a, th, st);
  } else {
    if (nv <= 256) return norm_team<T, 1, 8, 32>(rms, a, 128, st);
    const int th = ceil_div(nv, 16 * 32) * 32;
    if (th <= 512) return norm_team<T, 1, 16, 0>(rms, a, th, st);
  }
  auto k = rms ? k_norm_rows<T, true> : k_norm_rows<T, false>;
  k<<<a.M, kThreads, 0, st>>>(a.rs, a.x, a.w, a.bias, a.pbf, a.eps, a.d, a.y, a.mean, a.rstd);
  return cudaGetLastError();
}

// Rows of a block of the gradient: blocks for `occ` a multiprocessor, and at least
// 4 rows each so that joining their sums stays small beside forming them.
int grad_rows(long long M, int num_sms, int occ) {
  return std::max(4, ceil_div(M, static_cast<long long>(num_sms) * occ));
}
constexpr int kGradOcc = 8;  // most blocks a multiprocessor is given
int grad_blocks(long long M, int num_sms) { return ceil_div(M, grad_rows(M, num_sms, kGradOcc)); }

template <typename T, int N, int NV, int TEAM, bool BULK, bool WREG, int MAXT, int MINB>
cudaError_t grad_team(GradArgs& a, int threads, int num_sms, cudaStream_t st) {
  auto k = a.g.rms ? k_norm_grad<T, N, NV, TEAM, true, BULK, WREG, MAXT, MINB>
                   : k_norm_grad<T, N, NV, TEAM, false, BULK, WREG, MAXT, MINB>;
  const int teams = TEAM ? 32 * kWarpTeams / (TEAM ? TEAM : 1) : 1;
  const size_t width = static_cast<size_t>(NV) * (TEAM ? TEAM : threads) * N;
  const size_t stage = static_cast<size_t>(teams) * 2 * (BULK ? a.g.d : width) * sizeof(T);
  const size_t extra = width * ((WREG ? 0 : 4) + (TEAM ? 8 : 0));
  // Fewer blocks where the rings would have less than two or three rows each.
  constexpr int kMinStages = !BULK ? kOwnStages : sizeof(T) == 2 ? 3 : 2;
  const int occ = std::max(1, std::min(resident(k, threads, kGradOcc),
                                       static_cast<int>(kSmemPerSm / (extra + kMinStages * stage))));
  a.stages = !BULK ? kOwnStages
                   : std::max(2, std::min<int>(8, static_cast<int>((kSmemPerSm / occ - extra) / stage)));
  const size_t smem = extra + a.stages * stage;
  if (cudaError_t e = allow_smem(k, smem); e != cudaSuccess) return e;
  a.per = grad_rows(a.M, num_sms, occ);
  // Rows of padding are less work than others: 512 examples of 512 x 768 bf16, a
  // quarter to all tokens kept, 200 us in blocks of equally many rows and 170 us of
  // equal work.
  // Every block reads all lengths for its share, so examples of fewer than 64 tokens,
  // whose lengths would be a tenth of the traffic, are cut by rows.
  a.by_work = a.g.rs.lengths && a.g.rs.T >= 64;
  if (a.by_work && (a.g.dweight || a.g.dbias))
    a.starts = reinterpret_cast<int*>(a.slots + static_cast<size_t>(grad_blocks(a.M, num_sms)) * 4 * a.g.d);
  k<<<ceil_div(a.M, a.per), threads, smem, st>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t grad_launch(GradArgs& a, int num_sms, cudaStream_t st) {
  constexpr int F = 16 / sizeof(T);
  const NormGrad& g = a.g;
  const int es = sizeof(T), pes = g.param_bf16 ? 2 : 4;
  int vec = std::min(row_vec(g.x, g.rs, g.d, es), row_vec(g.dy, g.rs, g.d, es));
  if (g.dx.p) vec = std::min(vec, row_vec(g.dx, g.rs, g.d, es));
  const int pvec = row_vec(g.weight, 0, 0, RowSet{1, 1, nullptr}, 8, pes);
  if (vec > 1 && pvec < 2) vec = 1;
  if (vec == F && pvec < 16 / pes) vec = 2;
  constexpr int WNV = sizeof(T) == 2 ? 4 : 6, BNV = 4;
  // Weights in registers: not for warps of bf16, whose unpacking costs more than
  // reading them from shared memory (768 channels: 277 us against 249 us).
  constexpr bool WREG = sizeof(T) == 4;
  const bool own_type = g.param_bf16 == (sizeof(T) == 2);
  const Shape s = grad_shape(g.d, vec, es, WNV, BNV);
  // Narrow rows, several to a warp, whose lanes copy their own vectors.
  if (s.n == F && s.team == 32) {
    const int nv = g.d / F;
    if (nv <= 8) return grad_team<T, F, 1, 8, false, false, 128, 4>(a, 128, num_sms, st);
    if (nv <= 16) return grad_team<T, F, 2, 8, false, false, 128, 4>(a, 128, num_sms, st);
    if (nv <= 32) return grad_team<T, F, 4, 8, false, false, 128, 3>(a, 128, num_sms, st);
    if (nv <= 64) return grad_team<T, F, 4, 16, false, false, 128, 3>(a, 128, num_sms, st);
  }
  if (s.n == F && s.team == 32 && (own_type || !WREG)) {
    if (s.nv == 3) return grad_team<T, F, 3, 32, true, WREG, 128, 4>(a, s.threads, num_sms, st);
    if (s.nv == 4) return grad_team<T, F, 4, 32, true, WREG, 128, 4>(a, s.threads, num_sms, st);
    if constexpr (WNV > 4) return grad_team<T, F, WNV, 32, true, WREG, 128, 3>(a, s.threads, num_sms, st);
  }
  if (s.n == F && s.team == 0 && own_type) {
    // bf16, 32 elements a thread: few blocks of many registers, except where a row is
    // only two warps (2048 channels: 292 us with 8 blocks, 398 us with 4). fp32, 16
    // elements: 768 threads a multiprocessor.
    if constexpr (sizeof(T) == 2) {
      if (s.threads <= 64) return grad_team<T, F, BNV, 0, true, true, 64, 8>(a, s.threads, num_sms, st);
      if (s.threads <= 128) return grad_team<T, F, BNV, 0, true, true, 128, 2>(a, s.threads, num_sms, st);
      if (s.threads <= 192) return grad_team<T, F, BNV, 0, true, true, 256, 2>(a, s.threads, num_sms, st);
      if (s.threads <= 256) return grad_team<T, F, BNV, 0, true, true, 256, 1>(a, s.threads, num_sms, st);
    } else {
      if (s.threads <= 128) return grad_team<T, F, BNV, 0, true, true, 128, 6>(a, s.threads, num_sms, st);
      if (s.threads <= 256) return grad_team<T, F, BNV, 0, true, true, 256, 3>(a, s.threads, num_sms, st);
    }
    return grad_team<T, F, BNV, 0, true, true, 512, 1>(a, s.threads, num_sms, st);
  }
  if (s.n == F && s.team == 32) return grad_team<T, F, WNV, 32, true, false, 128, 4>(a, s.threads, num_sms, st);
  if (s.n == F) return grad_team<T, F, BNV, 0, true, false, 512, 1>(a, s.threads, num_sms, st);
  if (s.n == 2) return grad_team<T, 2, 8, 0, false, false, 512, 1>(a, s.threads, num_sms, st);
  if (s.n == 1) return grad_team<T, 1, 8, 0, false, false, 512, 1>(a, s.threads, num_sms, st);
  // The sums read dy and x before dx may be written over them.
  a.per = grad_rows(a.M, num_sms, kGradOcc);
  if (g.dweight || g.dbias) {
    auto k = g.rms ? k_norm_dparam_rows<T, true> : k_norm_dparam_rows<T, false>;
    k<<<dim3(ceil_div(g.d, kThreads), ceil_div(a.M, a.per)), kThreads, 0, st>>>(a);
    // dx may go over dy or x: not after sums that did not start.
    if (cudaError_t e = cudaGetLastError(); e != cudaSuccess) return e;
  }
  if (g.dx.p) {
    auto k = g.rms ? k_norm_dx_rows<T, true> : k_norm_dx_rows<T, false>;
    k<<<a.M, kThreads, 0, st>>>(g);
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_norm(bool rms, RowSet rs, RowView x, bool bf16_, const void* weight, const void* bias,
                        bool param_bf16, float eps, int d, RowView y, float* mean, float* rstd, int num_sms,
                        cudaStream_t st) {
  const NormArgs a{flatten(rs, x, y), static_cast<int>(rs.rows()), x, weight, bias, param_bf16, eps, d, y, mean, rstd};
  return bf16_ ? norm_launch<bf16>(rms, a, num_sms, st) : norm_launch<float>(rms, a, num_sms, st);
}

size_t norm_grad_ws_bytes(int B, int T, int d, int num_sms) {
  const long long M = static_cast<long long>(B) * T;
  if (M == 0) return 0;
  const size_t blocks = grad_blocks(M, num_sms);
  return blocks * 4 * d * 4 + (blocks + 1) * 4;  // two slots of two sums a block; where the blocks start
}

cudaError_t launch_norm_grad(const NormGrad& g, void* ws, unsigned* status, int num_sms, cudaStream_t st) {
  const int M = static_cast<int>(g.rs.rows()), groups = g.per_example ? g.rs.B : 1;
  const bool sums = (g.dweight || g.dbias) && groups > 0;
  if (!sums && (!g.dx.p || M == 0)) return cudaSuccess;
  GradArgs a{g, M, g.per_example ? g.rs.T : M, 1, static_cast<float*>(ws), false, nullptr, 0, status};
  a.g.rs = g.dx.p ? flatten(g.rs, g.x, g.dy, g.dx) : flatten(g.rs, g.x, g.dy);
  if (M > 0) {
    const cudaError_t e = g.bf16 ? grad_launch<bf16>(a, num_sms, st) : grad_launch<float>(a, num_sms, st);
    if (e != cudaSuccess) return e;
    if (!sums || (!a.by_work && a.per % a.rpg == 0) || M <= a.per) return cudaSuccess;  // no group is shared by blocks
  }
  const int rows = std::min(groups, 65535), blocks = M > 0 ? ceil_div(M, a.per) : 0;
  const size_t smem = a.starts ? (blocks + 1) * sizeof(int) : 0;
  if (ceil_div(a.rpg, a.per) <= 8)
    k_norm_grad_join<1><<<dim3(ceil_div(g.d, kThreads), rows), kThreads, smem, st>>>(a, groups, blocks);
  else
    k_norm_grad_join<kJoinSlices>
        <<<dim3(ceil_div(g.d, 32), rows), 32 * kJoinSlices, smem, st>>>(a, groups, blocks);
  return cudaGetLastError();
}
