// Token loss through the output matrix and its gradient. Per counted position, with
// z = scale x W^T over the V classes:
//   lse = log sum_v exp(z_v),  loss = w (lse - z_target),
//   D = w scale (exp(z - lse) - e_target),  dx = D W,  dW (+)= sum D^T x.
//
// The counted positions (inside their example's length, target not ignored, weight not
// 0) are found first and their rows of x gathered, a piece of them at a time: what is
// left out costs no products. The logits of one piece lie in the workspace in fp32 and
// become D in place; those of narrow rows of bf16 are formed again for D instead.
//
// Bound by the products, 6 m V d operations with both gradients (GB300: 4 x 2048 positions, 3,979 of them counted,
// 4096 columns, 100,000 classes: 6.7 ms), for few rows by the launches, one after the other, and the
// matrix's way through the multiprocessors (511 positions, 768 columns, 50,001 classes: 171 us); the loss of
// one position by reading the matrix (50,000 x 768: 33 us).
#include <algorithm>

#include "head_dev.cuh"

using namespace eogp;

namespace {

constexpr int kFindThreads = 1024;
constexpr int kFindBlocks = 1024;
constexpr int kFewRows = 1024;
constexpr int kAgainRows = 256, kAgainWidth = 1024;
constexpr int kDSegment = 8192;  // columns of a row of D that a block forms at a time
constexpr size_t kSlabBytes = size_t(512) << 20;
constexpr size_t kPieceBytes = size_t(4) << 30;  // logits of a piece

size_t al256(size_t x) { return (x + 255) & ~size_t(255); }
long long up(long long x, long long a) { return (x + a - 1) / a * a; }

// Where everything lies in the workspace, and how the products are cut.
struct Plan {
  int find_blocks, per_block;  // blocks of the search, positions of each
  bool few;                    // positions are found and gathered in one launch
  int piece, pieces;           // rows of a piece, most pieces
  int ldz, ldx, ldw;           // row strides of the logits, of the gathered rows and of the matrix (bf16 elements)
  int parts;                   // bf16 parts of D
  bool again;                  // the logits are not kept but formed again for D
  int bn_z, bn_d;              // columns of a tile of the logits, of dx and dW
  int ld_slab;
  size_t slab_bytes;
  size_t counts, idx, target, w, x, z, D, acc, W, part, zt, row, rest, rest_w, slabs, total;
};

bool w_fits(const HeadArgs& a) {
  return a.bf16 && reinterpret_cast<uintptr_t>(a.weight) % 16 == 0 &&
         (a.V == 1 || (a.ld_weight % 8 == 0 && a.ld_weight >= a.d));
}

Plan plan_of(const HeadArgs& a) {
  Plan p{};
  const long long M = a.rs.rows();
  if (M == 0) return p;
  const bool grad = a.dx.p || a.dweight;
  const long long tiles = (M + kFindThreads - 1) / kFindThreads;
  const long long each = (tiles + kFindBlocks - 1) / kFindBlocks;
  p.per_block = static_cast<int>(each * kFindThreads);
  p.find_blocks = static_cast<int>((tiles + each - 1) / each);
  p.ldz = static_cast<int>(up(a.V, 64));
  p.ldx = p.ldw = static_cast<int>(a.bf16 ? up(a.d, 8) : up(a.d, 64) * 3);
  p.parts = !a.bf16 ? 3 : a.dweight && !a.grad_bf16 ? 2 : 1;
  // Narrow rows: the logits are not kept, D is formed from them where they are computed a second time. That costs
  // 2 d operations a logit and spares 8 bytes of traffic, 6 or 4 where D has one part or two. us, kept / formed again, of
  // 16,384 rows and 50,000 classes, dW in bf16 and in fp32 (two parts):
  //   64 columns 2,437 / 1,319 and 2,802 / 2,163, 256 2,562 / 1,538 and 2,937 / 2,307, 768 3,598 / 3,414 and
  //   4,598 / 4,416, 896 4,202 / 4,072 and 5,469 / 5,418, 1024 4,380 / 4,308 and 5,789 / 5,798, 1536 6,020 / 6,502 and
  //   7,879 / 8,431;
  // 511 rows, in bf16: 256 columns 124 / 101, 768 169 / 173. For few rows the matrix, read once more, counts too.
  p.again = grad && a.bf16 && M >= kAgainRows && a.d <= std::min<long long>(kAgainWidth, M);
  // A row of a piece: logits (and D, where it is not in their place), or the sums of its half tiles; and the gathered row.
  const size_t row_bytes = static_cast<size_t>(p.ldx) * 2 + (grad ? static_cast<size_t>(p.ldz) * (p.again ? p.parts * 2 : a.bf16 ? 4 : 10) : 0) +
                           p.ldz / 64 * 16;
  const long long most = std::max<long long>(256, static_cast<long long>(kPieceBytes / row_bytes) / 256 * 256);
  p.pieces = static_cast<int>((M + most - 1) / most);
  p.piece = static_cast<int>(std::min(most, up((M + p.pieces - 1) / p.pieces, 256)));
  p.few = p.pieces == 1 && M <= kFewRows;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += al256(bytes);
    return o;
  };
  p.counts = take((kFindBlocks + 1) * 4);
  p.idx = take(M * 4);
  p.target = take(M * 4);
  p.w = take(M * 4);
  p.x = take(static_cast<size_t>(p.piece) * p.ldx * 2);
  if (!w_fits(a)) p.W = take(static_cast<size_t>(a.V) * p.ldw * 2);
  // Columns of a tile of the logits: those with which the pairs have the least in their rounds, a tile costing
  // about 24 columns more than it has (50,000 classes, one row, 76 pairs: 3 rounds of 224 instead of 256). fp32: two
  // accumulators of 128 at most.
  const long long mt = (std::min<long long>(M, p.piece) + 255) / 256;
  long long least = 0;
  for (int bn = a.bf16 ? 256 : 128; bn >= 64; bn -= 32) {
    const long long cost = (mt * ((a.V + bn - 1) / bn) + a.clusters - 1) / a.clusters * (bn + 24);
    if (p.bn_z == 0 || cost < least) p.bn_z = bn, least = cost;
  }
  p.bn_d = !a.bf16 || up(a.d, 128) * 1.15 < up(a.d, 256) ? 128 : 256;
  p.part = take(static_cast<size_t>((a.V + p.bn_z - 1) / p.bn_z) * 2 * p.piece * 8);
  p.zt = take(static_cast<size_t>(p.piece) * 4);
  p.row = take(static_cast<size_t>(p.piece) * 8);
  p.rest = p.rest_w = take(static_cast<size_t>(p.piece) * 4);
  if (p.parts == 2) p.rest_w = take(static_cast<size_t>(p.piece) * 4);
  if (grad) {
    if (!p.again) p.z = take(static_cast<size_t>(p.piece) * p.ldz * 4);
    if (!a.bf16 || p.again) p.D = take(static_cast<size_t>(p.piece) * p.ldz * p.parts * 2);
    if (a.dweight && a.grad_bf16 && p.pieces > 1) p.acc = take(static_cast<size_t>(a.V) * a.d * 4);
    p.ld_slab = static_cast<int>(up(a.d, 8));
    // Room for split sums: as many as there may be, of dx for any number of rows, half a GB at most.
    const long long most = std::min<long long>(M, p.piece), across = (a.d + p.bn_d - 1) / p.bn_d;
    size_t floats = 0;
    if (a.dweight)
      floats = head_slab_floats((a.V + 255ll) / 256 * across, (most + 63) / 64, p.parts == 2 ? 2 : 1,
                                static_cast<size_t>(a.V) * p.ld_slab, a.clusters);
    for (long long m = 1; a.dx.p && (m - 1) * 256 < most && head_split_at_all(m * across, a.clusters); ++m)
      floats = std::max(floats, head_slab_floats(m * across, (a.V + 63ll) / 64, 1,
                                                 static_cast<size_t>(std::min(m * 256, most)) * p.ld_slab, a.clusters));
    p.slab_bytes = std::min(kSlabBytes, floats * 4);
    p.slabs = take(p.slab_bytes);
  }
  p.total = at;
  return p;
}

// ------------------------------------------------------------ counted positions
struct Job {
  int target;
  float w;
  bool kept;
};
__device__ __forceinline__ Job job_of(const HeadArgs& a, int r, unsigned* status) {
  int b, t;
  locate(a.rs, r, b, t);
  const int len = a.rs.lengths ? a.rs.lengths[b] : a.rs.T;
  const long long target = token_at(a.targets, b, t);
  const float w = a.weights ? a.weights[r] : 1.f;
  bool kept = t < len && target != a.ignore && w != 0.f;
  if (kept && (target < 0 || target >= a.V)) {
    flag_status(status, EOGP_ST_DEVICE);
    kept = false;
  }
  return Job{static_cast<int>(target), w, kept};
}

__global__ void __launch_bounds__(kFindThreads) k_head_count(const HeadArgs a, int M, int per, int* counts) {
  after_previous();
  const int r0 = blockIdx.x * per, r1 = min(M, r0 + per);
  int n = 0;
  for (int r = r0; r < r1; r += kFindThreads) {
    const int i = r + threadIdx.x;
    n += __syncthreads_count(i < r1 && job_of(a, i, nullptr).kept);
  }
  if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// idx[i], target[i], w[i] of counted position i, in ascending order of (b, t); their
// number in counts[kFindBlocks]. Losses of the others are 0.
__global__ void __launch_bounds__(kFindThreads) k_head_place(const HeadArgs a, int M, int per, int* counts, int* idx,
                                                             int* target, float* w, unsigned* status) {
  after_previous();
  __shared__ int part[kFindThreads / 32], base;
  const int tid = threadIdx.x, lane = tid & 31;
  int before = 0;
  if (gridDim.x > 1) {
    before = tid < blockIdx.x ? counts[tid] : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    if (lane == 0) part[tid >> 5] = before;
    __syncthreads();
    before = 0;
    for (int i = 0; i < kFindThreads / 32; ++i) before += part[i];
    __syncthreads();
  }
  const int r0 = blockIdx.x * per, r1 = min(M, r0 + per);
  for (int r = r0; r < r1; r += kFindThreads) {
    const int i = r + tid;
    Job j{0, 0.f, false};
    if (i < r1) j = job_of(a, i, status);
    const unsigned mask = __ballot_sync(0xffffffffu, j.kept);
    if (lane == 0) part[tid >> 5] = __popc(mask);
    __syncthreads();
    int at = before + __popc(mask & ((1u << lane) - 1u)), all = 0;
    for (int k = 0; k < kFindThreads / 32; ++k) {
      if (k < tid >> 5) at += part[k];
      all += part[k];
    }
    if (j.kept) {
      idx[at] = i;
      target[at] = j.target;
      w[at] = j.w;
    } else if (i < r1) {
      a.loss[i] = 0.f;
      if (a.lse) a.lse[i] = 0.f;
    }
    before += all;
    __syncthreads();
  }
  if (blockIdx.x == gridDim.x - 1 && tid == 0) counts[kFindBlocks] = before;
}

// Zeros in the rows of dx that are left out.
template <typename T>
__global__ void __launch_bounds__(256) k_head_zero(const HeadArgs a, int M) {
  after_previous();
  const int lane = threadIdx.x & 31;
  for (int r = blockIdx.x * 8 + (threadIdx.x >> 5); r < M; r += gridDim.x * 8) {
    if (job_of(a, r, nullptr).kept) continue;
    int b, t;
    locate(a.rs, r, b, t);
    T* const g = row_out<T>(a.dx, b, t);
    for (int c = lane; c < a.d; c += 32) g[c] = from_f32<T>(0.f);
  }
}

// fp32 as the sum of three bf16, exactly: 8 bits of the mantissa each, the first two cut off. What is not finite
// is its first part alone.
__device__ __forceinline__ void split3(float v, bf16 (&p)[3]) {
  if (!(fabsf(v) <= kLargest)) {
    p[0] = from_f32<bf16>(v);
    p[1] = p[2] = from_f32<bf16>(0.f);
    return;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const float top = k < 2 ? __uint_as_float(__float_as_uint(v) & 0xffff0000u) : v;
    p[k] = from_f32<bf16>(top);
    v -= top;
  }
}
// Place of part k of column c in a row of three parts.
__device__ __forceinline__ int place3(int c, int k) { return (c >> 6) * 192 + k * 64 + (c & 63); }

// A row as the products read it, by a warp: x (NULL: zeros) and zeros from d on; fp32 in three parts.
__device__ __forceinline__ void put_row(const bf16* x, int d, int ldx, bool vec, bf16* o) {
  const int lane = threadIdx.x & 31, nv = vec && x ? d / 8 : 0;
#pragma unroll 4
  for (int c = lane; c < nv; c += 32)
    *reinterpret_cast<uint4*>(o + c * 8) = __ldcs(reinterpret_cast<const uint4*>(x) + c);
  for (int c = nv * 8 + lane; c < ldx; c += 32) o[c] = x && c < d ? x[c] : from_f32<bf16>(0.f);
}
__device__ __forceinline__ void put_row(const float* x, int d, int ldx, bool, bf16* o) {
  // Two columns a lane: 64 at a time, a block of each part.
  const int lane = threadIdx.x & 31;
#pragma unroll 4
  for (int c = lane * 2; c < ldx / 3; c += 64) {
    bf16 p[3] = {}, q[3] = {};
    if (x && c < d) split3(x[c], p);
    if (x && c + 1 < d) split3(x[c + 1], q);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      __nv_bfloat162 v;
      v.x = p[k], v.y = q[k];
      *reinterpret_cast<__nv_bfloat162*>(o + place3(c, k)) = v;
    }
  }
}

// Rows first .. of the counted positions, dense; zeros up to the next multiple of 64.
template <typename T>
__global__ void __launch_bounds__(256) k_head_gather(const HeadArgs a, const int* counts, const int* idx, int first,
                                                     int piece, int ldx, bool vec, bf16* out) {
  after_previous();
  const int n = min(piece, counts[kFindBlocks] - first), n64 = (max(n, 0) + 63) & ~63;
  for (int i = blockIdx.x * 8 + (threadIdx.x >> 5); i < n64; i += gridDim.x * 8) {
    const T* x = nullptr;
    if (i < n) {
      int b, t;
      locate(a.rs, idx[first + i], b, t);
      x = row_of<T>(a.x, b, t);
    }
    put_row(x, a.d, ldx, vec, out + static_cast<size_t>(i) * ldx);
  }
}

// Up to kFewRows positions: the search, the gathering and the zeros in one launch. Every block looks at all of
// them, and each of its warps then has one.
template <typename T>
__global__ void __launch_bounds__(256) k_head_few(const HeadArgs a, int M, int* counts, int* idx, int* target, float* w,
                                                  int ldx, bool vec, bf16* out, unsigned* status) {
  after_previous();
  __shared__ unsigned kept[kFewRows / 32];
  const int tid = threadIdx.x, lane = tid & 31, r = blockIdx.x * 8 + (tid >> 5);
#pragma unroll
  for (int k = 0; k < kFewRows / 256; ++k) {
    const int i = tid + k * 256;
    const unsigned mask = __ballot_sync(0xffffffffu, i < M && job_of(a, i, nullptr).kept);
    if (lane == 0) kept[i >> 5] = mask;
  }
  __syncthreads();
  int before = 0, n = 0;
  for (int k = lane; k < kFewRows / 32; k += 32) {
    const unsigned m = kept[k];
    n += __popc(m);
    before += __popc(k * 32 + 32 <= r ? m : k * 32 <= r ? m & ((1u << (r & 31)) - 1u) : 0u);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    n += __shfl_xor_sync(0xffffffffu, n, o);
    before += __shfl_xor_sync(0xffffffffu, before, o);
  }
  if (r == 0 && lane == 0) counts[kFindBlocks] = n;
  for (int i = n + r; i < ((n + 63) & ~63); i += gridDim.x * 8)
    put_row(static_cast<const T*>(nullptr), a.d, ldx, vec, out + static_cast<size_t>(i) * ldx);
  if (r >= M) return;
  const Job j = job_of(a, r, status);
  int b, t;
  locate(a.rs, r, b, t);
  if (j.kept) {
    if (lane == 0) {
      idx[before] = r;
      target[before] = j.target;
      w[before] = j.w;
    }
    put_row(row_of<T>(a.x, b, t), a.d, ldx, vec, out + static_cast<size_t>(before) * ldx);
  } else {
    if (lane == 0) {
      a.loss[r] = 0.f;
      if (a.lse) a.lse[r] = 0.f;
    }
    if (a.dx.p) {
      T* const g = row_out<T>(a.dx, b, t);
      for (int c = lane; c < a.d; c += 32) g[c] = from_f32<T>(0.f);
    }
  }
}

// ------------------------------------------------------------ between the products
// The matrix with rows that TMA can read; fp32 in three parts.
template <typename T>
__global__ void __launch_bounds__(256) k_head_matrix(const T* W, long long ld, int V, int d, bf16* out, int ldo) {
  after_previous();
  for (long long r = blockIdx.x * 8 + (threadIdx.x >> 5); r < V; r += gridDim.x * 8)
    put_row(W + r * ld, d, ldo, false, out + r * ldo);
}

// 32 rows a block: the (maximum, sum) pairs of a row's half tiles joined to its loss and lse,
// and what D needs of them: maximum and w scale / sum.
__global__ void __launch_bounds__(1024) k_head_join(const HeadArgs a, const int* counts, const int* idx, const float* ws,
                                                    int first, int piece, const float2* parts, int n_parts,
                                                    const float* zt, float2* row) {
  after_previous();
  __shared__ float2 all[32][33];
  const int n = min(piece, counts[kFindBlocks] - first), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int i = blockIdx.x * 32 + lane;
  if (blockIdx.x * 32 >= n) return;
  float m = kLowest, s = 0.f;
  if (i < n) {
    const float2* const v = parts + i;
    for (int p = warp; p < n_parts; p += 32 * 8) {
      float2 x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[e] = p + 32 * e < n_parts ? v[static_cast<size_t>(p + 32 * e) * piece] : make_float2(kLowest, 0.f);
      float top = m;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e].x);
      s *= exp2f((m - top) * kLog2e);
      m = top;
#pragma unroll
      for (int e = 0; e < 8; ++e) s += x[e].y * exp2f((x[e].x - m) * kLog2e);
    }
  }
  all[warp][lane] = make_float2(m, s);
  __syncthreads();
  const int mine = blockIdx.x * 32 + warp;  // a row a warp
  if (mine >= n) return;
  const float2 x = all[lane][warp];
  m = x.x;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  s = warp_sum(x.y * exp2f((x.x - m) * kLog2e));
  if (lane > 0) return;
  const float ls = s > 0.f ? logf(s) : NAN;  // no finite logit: NaN
  const int r = idx[first + mine];
  const float w = ws[first + mine];
  a.loss[r] = w * ((m - zt[mine]) + ls);
  if (a.lse) a.lse[r] = m + ls;
  if (row) row[mine] = make_float2(m, w * a.scale / s);
}

// D over the logits, in place: the 256 bytes of 64 columns become the 64 first bf16 parts and, with PARTS = 2,
// the 64 second ones. Eight columns a thread, eight threads on such a block, which read it before one writes.
// With PARTS = 3 (fp32) the parts go to an array of their own.
// Zeros in the rows up to the next multiple of 64, which the sum over rows runs over. (4,096 x 50,000 to two parts: 255 us,
// 6.4 TB/s.)
template <int PARTS>
__global__ void __launch_bounds__(256) k_head_d(const HeadArgs a, const int* counts, const int* targets,
                                                const float* ws, int first, int piece, float* z, int ldz,
                                                const float2* row, bf16* D, float* rest,
                                                float* rest_w) {
  after_previous();
  const int n = min(piece, counts[kFindBlocks] - first), n64 = (max(n, 0) + 63) & ~63;
  const unsigned segments = (ldz + kDSegment - 1) / kDSegment, items = n64 * segments;
  for (unsigned item = blockIdx.x; item < items; item += gridDim.x) {
    const int i = item / segments, c0 = (item - i * segments) * kDSegment, c1 = min(ldz, c0 + kDSegment);
    float* const x = z + static_cast<size_t>(i) * ldz;
    const bool real = i < n;
    const float2 mi = real ? row[i] : make_float2(0.f, 0.f);
    const int target = real ? targets[first + i] : -1;
    const float g = real ? ws[first + i] * a.scale : 0.f;
    for (int c = c0 + threadIdx.x * 8; (c & ~255) < c1; c += 256 * 8) {
      Vals<8> v = fill<8>(0.f);
      if (real && c < c1) {
        v = ld_floats<8>(x + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v.p[e].x = exp2f((v.p[e].x - mi.x) * kLog2e) * mi.y;
          v.p[e].y = exp2f((v.p[e].y - mi.x) * kLog2e) * mi.y;
        }
        if (c + 8 > a.V) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + e >= a.V) v.set(e, 0.f);
        }
        if (static_cast<unsigned>(target - c) < 8u) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (target - c == e) v.set(e, v.get(e) - g);
          float at = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (target - c == e) at = v.get(e);
          if (PARTS < 3) {
            const float left = at - to_f32(from_f32<bf16>(at));
            rest[i] = left;
            if (PARTS == 2) rest_w[i] = left - to_f32(from_f32<bf16>(left));
          }
        }
      }
      __syncwarp();
      if (c >= c1) continue;
      bf16* const o = PARTS == 3 ? D + (static_cast<size_t>(i) * ldz + (c & ~63)) * 3 + (c & 63)
                                 : reinterpret_cast<bf16*>(x + (c & ~63)) + (c & 63);
      if (PARTS == 3) {
        __align__(16) bf16 w[3][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          bf16 q[3];
          split3(v.get(e), q);
          w[0][e] = q[0], w[1][e] = q[1], w[2][e] = q[2];
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(o + 64 * p) = *reinterpret_cast<const uint4*>(w[p]);
        continue;
      }
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        const Raw<bf16, 8> r = pack_raw<bf16, 8>(v);
        *reinterpret_cast<uint4*>(o + 64 * p) = r.w;
        if (p + 1 < PARTS) {
          const Vals<8> h = unpack<bf16, 8>(r);
#pragma unroll
          for (int e = 0; e < 4; ++e) v.p[e] = make_float2(v.p[e].x - h.p[e].x, v.p[e].y - h.p[e].y);
        }
      }
    }
  }
}

// The slabs of a split sum joined, in order, four columns a thread: rows of dx by position, or rows of dW.
__global__ void __launch_bounds__(256) k_head_slabs(const HeadTc h, bool to_dx) {
  after_previous();
  const int there = *h.count - h.first, some = max(0, min(h.piece, there)), rows = to_dx ? some : h.V;
  if ((to_dx || h.first > 0) && some == 0) return;
  const int steps = ((to_dx ? h.V : some) + 63) / 64, lane = threadIdx.x & 31;
  const int splits = head_splits(h, static_cast<long long>((rows + 255) / 256) * ((h.d + h.bn - 1) / h.bn), steps, rows);
  if (splits == 1) return;
  const bool to_acc = !to_dx && h.acc && there > h.piece;
  const size_t slab = static_cast<size_t>(rows) * h.ld_slab;
  // A warp has 128 columns of a row at a time.
  const long long chunks = (h.d + 127) / 128, items = rows * chunks;
  for (long long k = blockIdx.x * 8ll + (threadIdx.x >> 5); k < items; k += gridDim.x * 8ll) {
    const int i = items <= 0x7fffffff ? static_cast<int>(static_cast<unsigned>(k) / static_cast<unsigned>(chunks))
                                      : static_cast<int>(k / chunks);
    const int c = static_cast<int>(k - i * chunks) * 128 + lane * 4;
    if (c >= h.d) continue;
    int b = 0, t = 0;
    if (to_dx) locate(h.rs, h.idx[h.first + i], b, t);
    const float* const from = h.slabs + static_cast<size_t>(i) * h.ld_slab + c;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int s = 0; s < splits; ++s) {
      const float4 x = __ldcs(reinterpret_cast<const float4*>(from + s * slab));
      v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
    }
    const float w[4] = {v.x, v.y, v.z, v.w};
    const long long at = to_dx ? b * h.dx.bs + t * h.dx.ld : to_acc ? static_cast<long long>(i) * h.d : i * h.ld_out;
    void* const out = to_dx ? const_cast<void*>(h.dx.p) : to_acc ? h.acc : h.out;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (c + e >= h.d) break;
      float x = w[e];
      if (h.add) {
        const long long a = i * h.ld_add + c + e;
        x += h.add_bf16 ? to_f32(static_cast<const bf16*>(h.add)[a]) : static_cast<const float*>(h.add)[a];
      }
      if (h.out_bf16 && !to_acc)
        static_cast<bf16*>(out)[at + c + e] = from_f32<bf16>(x);
      else
        static_cast<float*>(out)[at + c + e] = x;
    }
  }
}

// Whether rows of `es`-byte elements begin on 16 bytes.
bool vec_rows(const RowView& v, int es) {
  return reinterpret_cast<uintptr_t>(v.p) % 16 == 0 && v.bs * es % 16 == 0 && v.ld * es % 16 == 0;
}

#define TRY(x)                                             \
  do {                                                     \
    if (cudaError_t e_ = (x); e_ != cudaSuccess) return e_; \
  } while (0)

// The counted positions of the batch, zeros for the others, and, where there are few, their rows at `x`.
template <typename T>
cudaError_t find(const HeadArgs& a, const Plan& p, uint8_t* ws, bf16* x, bool vec, bool next, unsigned* status,
                 int num_sms, cudaStream_t st) {
  const int M = static_cast<int>(a.rs.rows());
  int* const counts = reinterpret_cast<int*>(ws + p.counts);
  int* const idx = reinterpret_cast<int*>(ws + p.idx);
  int* const target = reinterpret_cast<int*>(ws + p.target);
  float* const w = reinterpret_cast<float*>(ws + p.w);
  if (p.few)
    return head_launch(k_head_few<T>, next, (M + 7) / 8, 256, 0, st, a, M, counts, idx, target, w, p.ldx, vec, x, status);
  if (p.find_blocks > 1) {
    TRY(head_launch(k_head_count, next, p.find_blocks, kFindThreads, 0, st, a, M, p.per_block, counts));
    next = true;
  }
  TRY(head_launch(k_head_place, next, p.find_blocks, kFindThreads, 0, st, a, M, p.per_block, counts, idx, target, w,
                  status));
  if (a.dx.p) TRY(head_launch(k_head_zero<T>, true, std::min((M + 7) / 8, num_sms * 8), 256, 0, st, a, M));
  return cudaSuccess;
}

// Bytes that rows of es-byte elements are aligned to, 32 at most.
int row_align(const void* p, long long bs, long long ld, int es) {
  int v = 32;
  while (v > es && (reinterpret_cast<uintptr_t>(p) % v || bs * es % v || ld * es % v)) v /= 2;
  return v;
}

template <typename T>
cudaError_t run(const HeadArgs& a, uint8_t* ws, unsigned* status, cudaStream_t st) {
  const Plan p = plan_of(a);
  const int num_sms = 2 * a.clusters;
  const int M = static_cast<int>(a.rs.rows());
  const bool grad = a.dx.p || a.dweight;
  int* const counts = reinterpret_cast<int*>(ws + p.counts);
  int* const idx = reinterpret_cast<int*>(ws + p.idx);
  int* const target = reinterpret_cast<int*>(ws + p.target);
  float* const w = reinterpret_cast<float*>(ws + p.w);
  bf16* const x = reinterpret_cast<bf16*>(ws + p.x);
  float2* const row = reinterpret_cast<float2*>(ws + p.row);
  const bf16* W = static_cast<const bf16*>(a.weight);
  long long ldw = a.V == 1 ? p.ldw : a.ld_weight;
  constexpr bool f32 = sizeof(T) == 4;
  if (!w_fits(a)) {
    bf16* const copy = reinterpret_cast<bf16*>(ws + p.W);
    TRY(head_launch(k_head_matrix<T>, false, std::min((a.V + 7) / 8, num_sms * 8), 256, 0, st,
                    static_cast<const T*>(a.weight), a.ld_weight, a.V, a.d, copy, p.ldw));
    W = copy;
    ldw = p.ldw;
  }
  const bool vec = vec_rows(a.x, sizeof(T));
  TRY(find<T>(a, p, ws, x, vec, !w_fits(a), status, num_sms, st));
  HeadTc h{};
  h.count = counts + kFindBlocks;
  h.piece = p.piece;
  h.d = a.d;
  h.V = a.V;
  h.scale = a.scale;
  h.z = grad && !p.again ? reinterpret_cast<float*>(ws + p.z) : nullptr;
  h.ldz = p.ldz;
  h.part = reinterpret_cast<float2*>(ws + p.part);
  h.zt = reinterpret_cast<float*>(ws + p.zt);
  h.rest = reinterpret_cast<float*>(ws + p.rest);
  h.rest_w = reinterpret_cast<float*>(ws + p.rest_w);
  h.target = target;
  h.rs = a.rs;
  h.idx = idx;
  h.parts_a = h.used_a = f32 ? 3 : 1;
  bf16* const D = reinterpret_cast<bf16*>(ws + (f32 || p.again ? p.D : p.z));  // else in the logits' place
  const int parts_d = f32 ? 3 : p.again ? p.parts : 2;  // as they lie
  h.ld_slab = p.ld_slab;
  h.slabs = reinterpret_cast<float*>(ws + p.slabs);
  h.slab_bytes = p.slab_bytes;
  h.clusters = a.clusters;
  h.piece_rows = static_cast<int>(std::min<long long>(M, p.piece));
  h.rows_box = static_cast<int>(std::min<long long>(128, up(h.piece_rows, 8)));
  const uint64_t xcols = f32 ? p.ldx : a.d, uv = a.V, rows = p.piece, dcols = static_cast<uint64_t>(p.ldz) * parts_d;
  for (int c = 0; c < p.pieces; ++c) {
    h.first = c * p.piece;
    if (!p.few)
      TRY(head_launch(k_head_gather<T>, true, std::min(p.piece / 8, num_sms * 8), 256, 0, st, a, counts, idx, h.first,
                      p.piece, p.ldx, vec, x));
    HeadTc z = h;
    z.A = x, z.inner_a = xcols, z.rows_a = rows, z.lda = p.ldx;
    z.B = W, z.inner_b = xcols, z.rows_b = uv, z.ldb = ldw;
    z.bn = p.bn_z, z.run = 8;
    TRY(launch_head_logits(z, status, st));
    TRY(head_launch(k_head_join, true, (p.piece + 31) / 32, 1024, 0, st, a, counts, idx, w, h.first, p.piece, h.part,
                    (a.V + p.bn_z - 1) / p.bn_z * 2, h.zt, grad ? row : nullptr));
    if (!grad) continue;
    if (p.again) {
      z.bn = 256;
      z.D = D, z.parts_d = parts_d, z.row = row, z.w = w;
      TRY(launch_head_d(z, status, st));
    } else {
      auto d = f32 ? k_head_d<3> : p.parts == 2 ? k_head_d<2> : k_head_d<1>;
      const long long segments = static_cast<long long>(p.piece) * ((p.ldz + kDSegment - 1) / kDSegment);
      TRY(head_launch(d, true, std::min<long long>(segments, num_sms * 8), 256, 0, st, a, counts, target, w, h.first,
                      p.piece, h.z, p.ldz, row, D, h.rest, h.rest_w));
    }
    if (a.dx.p) {
      HeadTc g = h;
      g.A = D, g.inner_a = dcols, g.rows_a = rows, g.lda = dcols, g.parts_a = parts_d;
      g.B = W, g.inner_b = xcols, g.rows_b = uv, g.ldb = ldw;
      g.bn = p.bn_d, g.run = f32 ? 8 : 64;
      g.dx = a.dx, g.out_bf16 = !f32, g.out_vec = row_align(a.dx.p, a.dx.bs, a.dx.ld, sizeof(T));
      TRY(launch_head_dx(g, status, st));
      TRY(head_launch(k_head_slabs, true, num_sms * 8, 256, 0, st, g, true));
    }
    if (a.dweight) {
      HeadTc g = h;
      g.A = D, g.inner_a = dcols, g.rows_a = rows, g.lda = dcols, g.parts_a = parts_d;
      g.B = x, g.inner_b = xcols, g.rows_b = rows, g.ldb = p.ldx;
      g.used_a = p.parts;
      g.bn = p.bn_d, g.run = f32 || p.parts == 2 ? 8 : 64;
      // Sums of several pieces stay in fp32, in dweight itself or beside it; the last piece that has rows
      // ends them, and those after it do nothing.
      g.out = a.dweight, g.ld_out = a.ld_dweight, g.out_bf16 = a.grad_bf16;
      float* const acc = p.acc ? reinterpret_cast<float*>(ws + p.acc) : nullptr;
      if (c > 0)
        g.add = acc ? static_cast<void*>(acc) : a.dweight, g.ld_add = acc ? a.d : a.ld_dweight;
      else if (a.accumulate)
        g.add = a.dweight, g.ld_add = a.ld_dweight, g.add_bf16 = a.grad_bf16;
      g.acc = c < p.pieces - 1 ? acc : nullptr;
      g.out_vec = row_align(g.out, 0, g.ld_out, g.out_bf16 ? 2 : 4);
      g.add_vec = row_align(g.add, 0, g.ld_add, g.add_bf16 ? 2 : 4);
      TRY(launch_head_dw(g, status, st));
      if (head_split_at_all((a.V + 255ll) / 256 * ((a.d + g.bn - 1) / g.bn), g.clusters))
        TRY(head_launch(k_head_slabs, true, num_sms * 8, 256, 0, st, g, false));
    }
  }
  return cudaSuccess;
}

// dweight of a batch without positions.
template <typename T>
__global__ void __launch_bounds__(256) k_head_clear(T* p, long long ld, int V, int d) {
  for (long long r = blockIdx.x; r < V; r += gridDim.x)
    for (int c = threadIdx.x; c < d; c += 256) p[r * ld + c] = from_f32<T>(0.f);
}

}  // namespace

size_t head_loss_ws_bytes(const HeadArgs& a) { return plan_of(a).total; }

cudaError_t launch_head_loss(const HeadArgs& a, void* ws, unsigned* status, cudaStream_t st) {
  if (a.rs.rows() == 0) {
    if (a.accumulate) return cudaSuccess;
    const int blocks = std::min(a.V, a.clusters * 16);
    if (a.grad_bf16)
      k_head_clear<bf16><<<blocks, 256, 0, st>>>(static_cast<bf16*>(a.dweight), a.ld_dweight, a.V, a.d);
    else
      k_head_clear<float><<<blocks, 256, 0, st>>>(static_cast<float*>(a.dweight), a.ld_dweight, a.V, a.d);
    return cudaGetLastError();
  }
  return a.bf16 ? run<bf16>(a, static_cast<uint8_t*>(ws), status, st)
                : run<float>(a, static_cast<uint8_t*>(ws), status, st);
}
