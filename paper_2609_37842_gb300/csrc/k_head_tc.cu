// The products of the token loss through the output matrix, on the tensor cores (see
// k_head.cu for the formulas): z = scale x W^T with the sums of the loss, or once more as D of
// them, dx = D W and dW = D^T x, all sums in fp32.
//
// k_head_tc: a pair of CTAs (tcgen05 cta_group::2) works on tiles of 256 x BN outputs, one
// after the other. Each CTA loads its 128 rows of A and its half of B's columns, 64 steps of the
// sum at a time, by TMA into a ring; the leader's MMA warp issues M = 256 instructions, whose
// accumulators (two, in turn) lie in both CTAs' tensor memory; eight warps a CTA take a finished
// one while the next is filled. An operand is read as it lies: K-major (x and W for the logits, D
// for dx) or MN-major (W for dx, D and x for dW), so nothing is transposed.
// Tensor cores cut an accumulator off where they add to it: towards 0, by up to 2^-23 of it every
// 16 products. So a long sum goes through several accumulators, `run` steps of 64 each, which are
// added up in registers, rounded.
// An operand may come in several bf16 parts, blocks of 64 columns of each in turn. D of two parts (PARTS = 2): both
// are in a stage and meet the same x. fp32 operands are sums of three parts of 8 bits each, exactly; of the
// nine products of parts the six down to 2^-16 are formed (PARTS = 3), the first parts' in one accumulator and
// the others', 2^-8 and less of it, in a second one, where cutting off costs nothing that counts.
//
// Warps (384 threads): 0 issues TMA, 1 owns tensor memory and issues MMAs, 4-11 end tiles; these
// take over registers from the first four (168 x 384 = 56 x 128 + 224 x 256).
// Every wait is bounded; after one that ran out each role goes to the common end.
//
// 875 rows, 4096 columns, 50,000 classes: z 457 us, dx 404, dW 416 (73, 85, 74 % of the tensor cores' cycles) at 15 to
// 17 TB/s from L2 to shared memory, which bounds them; dW of two parts, with 3/4 of those bytes a product, 96 %. Many
// such launches in a row meet the power limit.
// Tried without gain: operands asked for in L2 ten steps ahead (7.2 against 6.7 ms for that batch), a thread of its
// own for each operand's copies.
#include <algorithm>

#include "head_dev.cuh"

using namespace eogp;

namespace {

constexpr int kThreads = 384;
constexpr int kMostStages = 16;
constexpr size_t kRingBytes = 221184;  // 6 stages of 32 KB, 3 of 72 KB
constexpr uint32_t kABytes = 128u * 64u * 2u;
constexpr int kNear = 1024;

enum { kLogits = 0, kDx = 1, kDw = 2, kD = 3 };

struct TcArgs {
  HeadTc h;
  int nN;      // tiles along N
  int stages;  // of the ring
  unsigned* status;
};

// What a tile is about: its place, the steps of its sum, and which slab of a split sum it gives.
struct Tile {
  int m0, n0, split, i0, i1;
};
// Outputs of a thread: a row's half tile, in registers while a sum goes through several accumulators.
struct Sums {
  float v[4][32];
};
struct Shape {
  int rows, M, mt, steps, splits, per, tiles;
  bool last;  // no piece with rows follows
};
// By whole warps.
template <int MODE>
__device__ __forceinline__ Shape shape_of(const TcArgs& g) {
  Shape s;
  const int left = *g.h.count - g.h.first;
  s.rows = max(0, min(g.h.piece, left));
  s.last = left <= g.h.piece;
  s.M = MODE == kDw ? g.h.V : s.rows;
  s.mt = (s.M + 255) / 256;
  const int K = MODE == kDx ? g.h.V : MODE == kDw ? s.rows : g.h.d;
  s.steps = (K + 63) / 64;
  s.splits = MODE == kLogits || MODE == kD ? 1 : head_splits(g.h, s.mt * g.nN, s.steps, s.M);
  s.per = (s.steps + s.splits - 1) / s.splits;
  s.tiles = s.rows == 0 && g.h.first > 0 ? 0 : s.mt * g.nN * s.splits;
  return s;
}
template <int MODE>
__device__ __forceinline__ Tile tile_of(const TcArgs& g, const Shape& s, int t) {
  Tile r;
  // Tiles that run together share what is read from far: the logits' W, and D for the others.
  const int mn = s.mt * g.nN;
  r.split = t / mn;
  t -= r.split * mn;
  constexpr bool by_n = MODE == kLogits || MODE == kD;
  const int m = by_n ? t % s.mt : t / g.nN, n = by_n ? t / s.mt : t % g.nN;
  r.m0 = m * 256;
  r.n0 = n * g.h.bn;
  r.i0 = r.split * s.per;
  r.i1 = min(s.steps, r.i0 + s.per);
  return r;
}

// Up to 32 outputs of one row, of which `left` are stored; `vec`: bytes that its start is aligned to (32 at most).
__device__ __forceinline__ void put_row(float* p, int left, int vec, const float (&v)[32]) {
  if (left >= 32 && vec >= 8) {
    if (vec == 32) {
#pragma unroll
      for (int q = 0; q < 32; q += 8) {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(v[q + e]);
        st_global_v8(p + q, w);
      }
    } else if (vec == 16) {
#pragma unroll
      for (int q = 0; q < 32; q += 4)
        *reinterpret_cast<float4*>(p + q) = make_float4(v[q], v[q + 1], v[q + 2], v[q + 3]);
    } else {
#pragma unroll
      for (int q = 0; q < 32; q += 2) *reinterpret_cast<float2*>(p + q) = make_float2(v[q], v[q + 1]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if (e < left) p[e] = v[e];
  }
}
__device__ __forceinline__ void put_row(bf16* p, int left, int vec, const float (&v)[32]) {
  if (left >= 32 && vec >= 4) {
    uint32_t w[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e] = pack_bf16(make_float2(v[2 * e], v[2 * e + 1]));
    if (vec == 32) {
#pragma unroll
      for (int q = 0; q < 16; q += 8) {
        const uint32_t u[8] = {w[q], w[q + 1], w[q + 2], w[q + 3], w[q + 4], w[q + 5], w[q + 6], w[q + 7]};
        st_global_v8(p + 2 * q, u);
      }
    } else if (vec == 16) {
#pragma unroll
      for (int q = 0; q < 16; q += 4)
        *reinterpret_cast<uint4*>(p + 2 * q) = make_uint4(w[q], w[q + 1], w[q + 2], w[q + 3]);
    } else if (vec == 8) {
#pragma unroll
      for (int q = 0; q < 16; q += 2) *reinterpret_cast<uint2*>(p + 2 * q) = make_uint2(w[q], w[q + 1]);
    } else {
#pragma unroll
      for (int q = 0; q < 16; ++q) *reinterpret_cast<uint32_t*>(p + 2 * q) = w[q];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if (e < left) p[e] = from_f32<bf16>(v[e]);
  }
}

template <typename T>
__device__ __forceinline__ void add_row(const T* p, int left, bool wide, float (&v)[32]) {
  constexpr int N = 16 / sizeof(T);
  if (left >= 32 && wide) {
#pragma unroll
    for (int q = 0; q < 32; q += N) {
      const Vals<N> a = unpack<T, N>(ld_raw<T, N>(p + q));
#pragma unroll
      for (int e = 0; e < N; ++e) v[q + e] += a.get(e);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if (e < left) v[e] += to_f32(p[e]);
  }
}

// What the sums of a thread's row of its side's columns of the tile become: logits, with the maximum and the sum of
// exponentials of the row's columns here. Two warps a scheduler run this: the chains are kept short.
__device__ __forceinline__ void end_logits(const TcArgs& g, const Shape& s, const Tile& t, int row, int side, int target,
                                           Sums& sums) {
  const HeadTc& h = g.h;
  if (row >= s.M) return;
  const int half = h.bn / 2, c0 = t.n0 + side * half, cols = min(half, h.V - c0);
  float top[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float(&v)[32] = sums.v[k];
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
      const float2 z = mul2(make_float2(v[e], v[e + 1]), pair(h.scale));
      v[e] = z.x, v[e + 1] = z.y;
    }
    if (cols < k * 32 + 32) {
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] = k * 32 + e < cols ? v[e] : -INFINITY;
    }
    if (h.z) {
      float* const z = h.z + static_cast<size_t>(row) * h.ldz + c0 + k * 32;
      const int left = min(half, h.ldz - c0) - k * 32;  // a multiple of 8
#pragma unroll
      for (int q = 0; q < 32; q += 8) {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(v[q + e]);
        if (q < left) st_global_v8(z + q, w);
      }
    }
    float a[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = fmaxf(fmaxf(v[e], v[e + 8]), fmaxf(v[e + 16], v[e + 24]));
    top[k] = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(a[4], a[5]), fmaxf(a[6], a[7])));
  }
  if (static_cast<unsigned>(target - c0) < static_cast<unsigned>(half)) {
    float zt = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 32; ++e) zt = target - c0 == k * 32 + e ? sums.v[k][e] : zt;
    h.zt[row] = zt;
  }
  const float m = fmaxf(kLowest, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
  float2 sum[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    sum[k] = pair(0.f);
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
      const float2 d = mul2(add2(make_float2(sums.v[k][e], sums.v[k][e + 1]), pair(-m)), pair(kLog2e));
      sum[k] = add2(sum[k], make_float2(exp2_fast(d.x), exp2_fast(d.y)));
    }
  }
  const float2 all = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
  h.part[static_cast<size_t>(t.n0 / h.bn * 2 + side) * h.piece + row] = make_float2(m, all.x + all.y);
}

// Or D of logits that are not kept, in one or two bf16 parts: zeros from V on and in the rows up to the next multiple
// of 64. Sixteen columns of a part are 32 bytes of a block of 64.
__device__ __forceinline__ void end_d(const TcArgs& g, const Shape& s, const Tile& t, int row, int side, int target,
                                      Sums& sums) {
  const HeadTc& h = g.h;
  if (row >= ((s.M + 63) & ~63)) return;
  const bool real = row < s.M;
  const float2 mi = real ? h.row[row] : make_float2(0.f, 0.f);
  const int c0 = t.n0 + side * (h.bn / 2), cols = real ? h.V - c0 : 0, out = h.ldz - c0;
  bf16* const D = static_cast<bf16*>(h.D) + static_cast<size_t>(row) * h.ldz * h.parts_d;
  const float gt = static_cast<unsigned>(target - c0) < 128u ? h.w[h.first + row] * h.scale : 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float(&v)[32] = sums.v[k];
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
      const float2 z = mul2(make_float2(v[e], v[e + 1]), pair(h.scale));
      const float2 x = mul2(add2(z, pair(-mi.x)), pair(kLog2e));
      const float2 p = mul2(make_float2(exp2_fast(x.x), exp2_fast(x.y)), pair(mi.y));
      v[e] = p.x, v[e + 1] = p.y;
    }
    if (cols < k * 32 + 32) {
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] = k * 32 + e < cols ? v[e] : 0.f;
    }
    if (static_cast<unsigned>(target - c0 - k * 32) < 32u) {
      float at = 0.f;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        if (target - c0 == k * 32 + e) at = v[e] -= gt;
      }
      const float rest = at - to_f32(from_f32<bf16>(at));
      h.rest[row] = rest;
      if (h.parts_d == 2) h.rest_w[row] = rest - to_f32(from_f32<bf16>(rest));
    }
    if (out < k * 32 + 32) continue;
    bf16* const o = D + static_cast<size_t>((c0 + k * 32) >> 6) * 64 * h.parts_d + (c0 + k * 32 & 63);
#pragma unroll
    for (int q = 0; q < 32; q += 16) {
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = pack_bf16(make_float2(v[q + 2 * e], v[q + 2 * e + 1]));
      st_global_v8(o + q, w);
      if (h.parts_d == 1) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        w[e] = pack_bf16(make_float2(v[q + 2 * e] - __uint_as_float(w[e] << 16),
                                     v[q + 2 * e + 1] - __uint_as_float(w[e] & 0xffff0000u)));
      st_global_v8(o + 64 + q, w);
    }
  }
}

// A thread's row and side of a tile with r times row `b` of the B operand added; r = 0: not.
__device__ __forceinline__ void add_rest(const HeadTc& h, const Tile& t, int side, float r, long long b, Sums& sums) {
  const int c0 = t.n0 + side * (h.bn / 2);
  if (r == 0.f) return;
  const bf16* const p = static_cast<const bf16*>(h.B) + b * static_cast<long long>(h.ldb) + c0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int left = h.d - c0 - k * 32;
    if (k * 64 >= h.bn || left <= 0) continue;
    if (left >= 32) {
      Raw<bf16, 8> w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = ld_keep<bf16, 8>(p + k * 32 + q * 8);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const Vals<8> x = unpack<bf16, 8>(w[q]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sums.v[k][q * 8 + e] = fmaf(r, x.get(e), sums.v[k][q * 8 + e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 32; ++e)
        if (e < left) sums.v[k][e] = fmaf(r, to_f32(p[k * 32 + e]), sums.v[k][e]);
    }
  }
}

// D enters the products rounded to bf16 (one part), as a batch's dlogits of the same type would. That tells most at the
// target, whose entry is among the largest of its row: a class whose gradient is one position's would have two
// roundings in place of one. So what was rounded off there is added in fp32 (3,979 rows, 100,000 classes: 0.0017 of dW's
// and dx's norms off float64, as products in fp32 rounded once; 0.0024 without; 447 rows of 768 columns: 10 of 171 us).
// Another class with most of a row's mass keeps its one rounding more (x along wrong classes, 1,024 rows of 256 columns,
// 4,000 classes: 0.0019 for 0.0017). Two parts of D in every product would take 195 us for 172 (511 tokens, 50,001 x
// 768) and 10.2 ms for 6.6 (those 3,979 rows).
// dx: a thread's row has one target. dW: targets and rests of the first positions lie in shared memory.
struct Near {
  int target[kNear];
  float rest[kNear];
};
// Positions of a lane's class, first ones first, as offsets of 10 bits: six in each word.
struct Queue {
  unsigned long long a, b;
  int n;
  __device__ __forceinline__ void push(unsigned at) {
    const unsigned long long v = at;
    if (n < 6)
      a |= v << 10 * n;
    else
      b |= v << 10 * (n - 6);
    ++n;
  }
  // From r0 on; -1: none.
  __device__ __forceinline__ int pop(int r0) {
    if (n == 0) return -1;
    const int at = static_cast<int>(a & 1023u);
    a = a >> 10 | (b & 1023u) << 50;
    b >>= 10;
    --n;
    return r0 + at;
  }
};
// What is added first, found before the sums are there.
struct Found {
  bool more;           // dW: a class of the warp's has another position among the same 1024
  int mine;            // row of B: dx: the target; dW: the first position of the lane's class; -1: none
  float rest;
  Raw<bf16, 8> x[16];  // that row's part, on its way
};
__device__ __forceinline__ void ask_rest(const HeadTc& h, const Tile& t, int side, Found& f) {
  const int c0 = t.n0 + side * (h.bn / 2);
  const bf16* const p = static_cast<const bf16*>(h.B) + f.mine * static_cast<long long>(h.ldb) + c0;
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    f.x[q] = {};
    const int left = q * 16 < h.bn ? h.d - c0 - q * 8 : 0;
    if (f.mine < 0 || left <= 0) continue;
    if (left >= 8) {
      f.x[q] = ld_keep<bf16, 8>(p + q * 8);
    } else {
      // A row's end: what lies behind it may not be there.
      uint32_t w[4] = {};
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < left) w[e / 2] |= static_cast<uint32_t>(__bfloat16_as_ushort(p[q * 8 + e])) << (e & 1) * 16;
      f.x[q].w = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}
__device__ __forceinline__ void add_found(const Found& f, Sums& sums) {
  if (!__any_sync(0xffffffffu, f.mine >= 0)) return;
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    const Vals<8> x = unpack<bf16, 8>(f.x[q]);
#pragma unroll
    for (int e = 0; e < 8; ++e) sums.v[q / 4][q % 4 * 8 + e] = fmaf(f.rest, x.get(e), sums.v[q / 4][q % 4 * 8 + e]);
  }
}
__device__ __forceinline__ float rest_of(const HeadTc& h, const Near& near, int r) {
  return r < 0 ? 0.f : r < kNear ? near.rest[r] : h.rest_w[r];
}
// Most positions of a class that are added to its row, in each part of a split sum: turns that a tile's MMAs cover.
// (Queues have room for 12.)
__device__ __forceinline__ int share_of(const Shape& s) { return min(12, 4 + s.steps / 4); }

// Of 1024 positions from r0 on, below r1, the first `share` of each of the warp's 32 classes: a queue a lane, for its class.
// A warp goes through the positions of its classes once, in a fixed order; those of a class that has its share are passed
// over from the next 32 on. (Targets of probability 1 / rank, 20,484 positions, 50,000 classes of 768 columns, dW in
// fp32: 5.8 ms, 8.2 by a scan of the positions left at each turn.)
__device__ __forceinline__ Queue queue_of(const HeadTc& h, const Near& near, int row0, int r0, int r1, int share) {
  const int lane = threadIdx.x & 31;
  Queue q{};
  unsigned done = __ballot_sync(0xffffffffu, share <= 0);
  for (int i = 0; i < 8 && r0 + i * 128 < r1; ++i) {
    const int r = r0 + i * 128 + lane * 4;
    int4 t = make_int4(-1, -1, -1, -1);
    if (r < r1) t = *reinterpret_cast<const int4*>(r < kNear ? &near.target[r] : &h.target[h.first + r]);
    const int c[4] = {t.x - row0, t.y - row0, t.z - row0, t.w - row0};
    bool hit[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) hit[e] = r + e < r1 && static_cast<unsigned>(c[e]) < 32u;
    if (!__any_sync(0xffffffffu, hit[0] || hit[1] || hit[2] || hit[3])) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      unsigned left = __ballot_sync(0xffffffffu, hit[e] && !(done >> (c[e] & 31) & 1u));
      if (left == 0) continue;
      for (; left; left &= left - 1) {
        const int b = __ffs(left) - 1;
        if (__shfl_sync(0xffffffffu, c[e], b) == lane && q.n < share) q.push(i * 128 + b * 4 + e);
      }
      done = __ballot_sync(0xffffffffu, q.n >= share);
    }
  }
  return q;
}

__device__ __forceinline__ void find_rest(const TcArgs& g, const Shape& s, const Tile& t, int row, const Near& near,
                                          Found& f) {
  const int row0 = row - static_cast<int>(threadIdx.x & 31), r0 = t.i0 * 64;
  Queue q = queue_of(g.h, near, row0, r0, min(s.rows, t.i1 * 64), 2);
  f.more = __any_sync(0xffffffffu, q.n > 1);
  f.mine = q.pop(r0);
  f.rest = rest_of(g.h, near, f.mine);
}
// The others: in a turn, the next one of every class that has one. So a class with many positions, whose roundings go
// either way, neither holds up the tile for long nor takes anything from its neighbours.
__device__ __forceinline__ void add_rest_dw(const TcArgs& g, const Shape& s, const Tile& t, int row, int side,
                                            const Near& near, const Found& f, Sums& sums) {
  const HeadTc& h = g.h;
  const int row0 = row - static_cast<int>(threadIdx.x & 31), r1 = min(s.rows, t.i1 * 64);
  int share = share_of(s);
  for (int r0 = t.i0 * 64; r0 < r1 && !__all_sync(0xffffffffu, share <= 0); r0 += 1024) {
    const bool first = r0 == t.i0 * 64;  // its first positions are added already
    if (first && !f.more) {
      share -= f.mine >= 0;
      continue;
    }
    Queue q = queue_of(h, near, row0, r0, r1, share);
    share -= q.n;
    if (first) q.pop(r0);
    while (__any_sync(0xffffffffu, q.n > 0)) {
      const int mine = q.pop(r0);
      add_rest(h, t, side, rest_of(h, near, mine), mine, sums);
    }
  }
}

// Or outputs of dx or dW, or of a slab of them.
template <int MODE>
__device__ __forceinline__ void end_tile(const TcArgs& g, const Shape& s, const Tile& t, int row, int side,
                                         Sums& sums) {
  const HeadTc& h = g.h;
  if (row >= s.M) return;
  bf16* out16 = nullptr;
  float* out32 = nullptr;
  int vec = 32;
  if (s.splits > 1) {
    out32 = h.slabs + (static_cast<size_t>(t.split) * s.M + row) * h.ld_slab;
  } else if (MODE == kDx) {
    int b, tt;
    locate(h.rs, h.idx[h.first + row], b, tt);
    if (h.out_bf16)
      out16 = row_out<bf16>(h.dx, b, tt);
    else
      out32 = row_out<float>(h.dx, b, tt);
    vec = h.out_vec;
  } else if (h.acc && !s.last) {
    out32 = h.acc + static_cast<size_t>(row) * h.d;
    vec = h.d % 8 == 0 ? 32 : 4;
  } else {
    const long long at = static_cast<long long>(row) * h.ld_out;
    if (h.out_bf16)
      out16 = static_cast<bf16*>(h.out) + at;
    else
      out32 = static_cast<float*>(h.out) + at;
    vec = h.out_vec;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int col = t.n0 + side * (h.bn / 2) + k * 32, left = h.d - col;
    if (k * 64 < h.bn && left > 0) {
      float(&v)[32] = sums.v[k];
      if (MODE == kDw && s.splits == 1 && h.add) {
        const long long at = static_cast<long long>(row) * h.ld_add + col;
        if (h.add_bf16)
          add_row(static_cast<const bf16*>(h.add) + at, left, h.add_vec >= 16, v);
        else
          add_row(static_cast<const float*>(h.add) + at, left, h.add_vec >= 16, v);
      }
      if (out16)
        put_row(out16 + col, left, vec, v);
      else
        put_row(out32 + col, left, vec, v);
    }
  }
}

// An accumulator, in place of the sums or added to them.
__device__ __forceinline__ void add_sums(uint32_t tmem, int bn, Sums& sums) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (k * 64 < bn) {
#pragma unroll
      for (int c = 0; c < 32; c += 16) {
        float v[16];
        tmem_ld16(tmem + k * 32 + c, v);
#pragma unroll
        for (int e = 0; e < 16; ++e) sums.v[k][c + e] += v[e];
      }
    }
  }
}
template <int PARTS>
__device__ __forceinline__ void take_sums(uint32_t tmem, int bn, bool more, Sums& sums) {
  if (more) {
    add_sums(tmem, bn, sums);
  } else {
    // All loads are under way before the first is waited for. Columns past the side's (the allocation has them: 512
    // for every width) are not used.
    uint32_t r[4][32];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      tmem_ld32_issue(tmem + k * 32, r[k]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      tmem_wait_ld(r[k]);
#pragma unroll
      for (int e = 0; e < 32; ++e) sums.v[k][e] = __uint_as_float(r[k][e]);
    }
  }
  if (PARTS == 3) add_sums(tmem + bn, bn, sums);
}

template <int MODE, int PARTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    k_head_tc(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const TcArgs g) {
  constexpr bool kAmn = MODE == kDw, kBmn = MODE == kDx || MODE == kDw;
  constexpr int kPartsB = PARTS == 3 ? 3 : 1;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = align1024(smem_raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int half = g.h.bn / 2;  // columns of B in this CTA
  const uint32_t a_bytes = kAmn ? kABytes : g.h.rows_box * 128u;
  const uint32_t b_bytes = static_cast<uint32_t>(half) * 128u, b_at = PARTS * a_bytes;
  const uint32_t stage_bytes = b_at + kPartsB * b_bytes;
  const int stages = g.stages;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + static_cast<size_t>(stages) * stage_bytes + (kABytes - a_bytes));
  uint64_t* empty = full + stages;
  uint64_t* tfull = empty + stages;
  uint64_t* tempty = tfull + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tempty + 2);
  Near& near = *reinterpret_cast<Near*>(tmem_slot + 4);
  const uint32_t buf_cols = static_cast<uint32_t>(g.h.bn) * (PARTS == 3 ? 2u : 1u);
  constexpr uint32_t tcols = 512;
  const int cl = blockIdx.x >> 1, ncl = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    for (int s = 0; s < stages; ++s) {
      mbar_init(&full[s], 2);   // one expect_tx arrive from each CTA (the leader's copy is used)
      mbar_init(&empty[s], 1);  // MMA completion, in both CTAs
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], 16);  // 8 warps of 2 CTAs (the leader's copy is used)
    }
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc_pair(tmem_slot, tcols);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  after_previous();
  const Shape sh = shape_of<MODE>(g);

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  if (warp == 0) {
    if (lane == 0) {
      // Few rows: those of A that there are, and none of the second CTA's. What the MMAs read in the others' place
      // (the stage's B, the next stage, at the ring's end the space behind it) only reaches outputs that are not taken.
      const bool a_there = kAmn || static_cast<int>(rank) * 128 < g.h.piece_rows;
      const uint32_t bytes = PARTS * (a_there ? a_bytes : 0u) + kPartsB * b_bytes;
      const uint32_t ring = smem_u32(smem), full0 = mapa_shared(smem_u32(full), 0);
      int s = 0;
      uint32_t ph = 1;
      bool ok = true;
      for (int t = cl; t < sh.tiles && ok; t += ncl) {
        const Tile tl = tile_of<MODE>(g, sh, t);
        const int am = tl.m0 + static_cast<int>(rank) * 128, bn = tl.n0 + static_cast<int>(rank) * half;
        const int ac = kAmn ? am * g.h.parts_a : 0, bc = kBmn ? bn * kPartsB : 0;
        const int ai = 64 * g.h.parts_a;
        for (int i = tl.i0; i < tl.i1; ++i) {
          if (!mbar_wait(&empty[s], ph, g.status)) {
            ok = false;
            break;
          }
          const uint32_t st = ring + s * stage_bytes, fl = full0 + s * 8;
          mbar_arrive_expect_tx_cluster(fl, bytes);
#pragma unroll
          for (int q = 0; q < PARTS; ++q) {
            const uint32_t a = st + q * a_bytes;
            if (kAmn) {
              tma_load_2d_pair(a, &tmA, ac + q * 64, i * 64, fl);
              tma_load_2d_pair(a + 8192, &tmA, ac + ai + q * 64, i * 64, fl);
            } else if (a_there) {
              tma_load_2d_pair(a, &tmA, i * ai + q * 64, am, fl);
            }
          }
#pragma unroll
          for (int q = 0; q < kPartsB; ++q) {
            const uint32_t b = st + b_at + q * b_bytes;
            if (kBmn) {
              tma_load_2d_pair(b, &tmB, bc + q * 64, i * 64, fl);
              if (half > 64) tma_load_2d_pair(b + 8192, &tmB, bc + (kPartsB + q) * 64, i * 64, fl);
            } else {
              tma_load_2d_pair(b, &tmB, (i * kPartsB + q) * 64, bn, fl);
            }
          }
          if (++s == stages) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      // The copies under way are not left behind: every stage is free again, or its wait has run out meanwhile.
      for (int k = 0; k < stages; ++k) {
        if (!mbar_wait(&empty[s], ph, g.status)) break;
        if (++s == stages) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      const uint32_t idesc = idesc_bf16_f32(256, g.h.bn, kAmn, kBmn);
      // Step of 16 along the sum: 32 bytes of a K-major row, 16 rows of 128 bytes of MN-major ones.
      constexpr uint64_t ka = kAmn ? 128 : 2, kb_ = kBmn ? 128 : 2;
      const uint32_t st = smem_u32(smem);
      const uint64_t a0 = kAmn ? sdesc_sw128(st, 8192, 1024) : sdesc_sw128(st, 16, 1024);
      const uint64_t b0 = kBmn ? sdesc_sw128(st + b_at, 8192, 1024) : sdesc_sw128(st + b_at, 16, 1024);
      int rs = 0, i = 0;
      uint32_t rph = 0;
      bool ok = true;
      for (int t = cl; t < sh.tiles && ok; t += ncl) {
        const Tile tl = tile_of<MODE>(g, sh, t);
        for (int k0 = tl.i0; k0 < tl.i1 && ok; k0 += g.h.run) {
          const int buf = i & 1, k1 = min(tl.i1, k0 + g.h.run);
          if (!mbar_wait(&tempty[buf], (static_cast<uint32_t>(i >> 1) & 1u) ^ 1u, g.status)) {
            ok = false;
            break;
          }
          ++i;
          tc_fence_after();
          const uint32_t d = tmem + buf * buf_cols;
          for (int k = k0; k < k1; ++k) {
            const int s = rs;
            const uint32_t ph = rph;
            if (++rs == stages) {
              rs = 0;
              rph ^= 1u;
            }
            if (!mbar_wait(&full[s], ph, g.status)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint32_t at = static_cast<uint32_t>(s) * stage_bytes >> 4;
            const uint64_t a = a0 + at, b = b0 + at;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              const uint64_t ak = a + ka * kk, bk = b + kb_ * kk;
              const uint32_t on = (k != k0 || kk != 0) ? 1u : 0u;
              tc_mma_f16_pair(d, ak, bk, idesc, on);
              if (PARTS == 2) tc_mma_f16_pair(d, ak + (a_bytes >> 4), bk, idesc, 1u);
              if (PARTS == 3) {
                const uint64_t a1 = a_bytes >> 4, b1 = b_bytes >> 4;
                const uint32_t rest = d + g.h.bn;
                tc_mma_f16_pair(rest, ak, bk + b1, idesc, on);
                tc_mma_f16_pair(rest, ak + a1, bk, idesc, 1u);
                tc_mma_f16_pair(rest, ak + a1, bk + b1, idesc, 1u);
                tc_mma_f16_pair(rest, ak, bk + 2 * b1, idesc, 1u);
                tc_mma_f16_pair(rest, ak + 2 * a1, bk, idesc, 1u);
              }
            }
            tc_commit_pair_mc(&empty[s], 0x3);
          }
          tc_commit_pair_mc(&tfull[buf], 0x3);
        }
      }
    }
    __syncwarp();
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    const int q = warp & 3, side = (warp - 4) >> 2;
    if (MODE == kDw && PARTS < 3) {
      for (int r = threadIdx.x - 128; r < min(kNear, sh.rows); r += 256) {
        near.target[r] = g.h.target[g.h.first + r];
        near.rest[r] = g.h.rest_w[r];
      }
      named_bar_sync(1, 256);
    }
    int i = 0;
    bool ok = true;
    for (int t = cl; t < sh.tiles && ok; t += ncl) {
      const Tile tl = tile_of<MODE>(g, sh, t);
      const int row = tl.m0 + static_cast<int>(rank) * 128 + q * 32 + lane;
      const uint32_t lanes = tmem + (static_cast<uint32_t>(q * 32) << 16);
      // Asked for before the accumulator is waited for.
      const bool one = MODE == kLogits || MODE == kD || (MODE == kDx && PARTS == 1 && tl.split == 0);
      const int target = one && row < sh.M ? g.h.target[g.h.first + row] : -1;
      Found found;
      if constexpr (PARTS < 3 && (MODE == kDx || MODE == kDw)) {
        if (MODE == kDw) {
          find_rest(g, sh, tl, row, near, found);
        } else {
          found.mine = target;
          found.rest = target >= 0 ? g.h.rest[row] : 0.f;
        }
        if (found.rest == 0.f) found.mine = -1;
        ask_rest(g.h, tl, side, found);
      }
      Sums sums;
      if (tl.i0 >= tl.i1) {  // a sum without terms
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int e = 0; e < 32; ++e) sums.v[k][e] = 0.f;
      }
      for (int k0 = tl.i0; k0 < tl.i1; k0 += g.h.run, ++i) {
        const int buf = i & 1;
        uint32_t there = 1;
        if (lane == 0) there = mbar_wait(&tfull[buf], static_cast<uint32_t>(i >> 1) & 1u, g.status) ? 1u : 0u;
        there = __shfl_sync(0xffffffffu, there, 0);
        if (!there) {
          ok = false;
          break;
        }
        tc_fence_after();
        take_sums<PARTS>(lanes + buf * buf_cols + side * half, g.h.bn, k0 > tl.i0, sums);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_relaxed_cluster(mapa_shared(smem_u32(&tempty[buf]), 0));
      }
      if (!ok) break;
      if constexpr (MODE == kLogits)
        end_logits(g, sh, tl, row, side, target, sums);
      else if constexpr (MODE == kD)
        end_d(g, sh, tl, row, side, target, sums);
      else {
        if constexpr (PARTS < 3) add_found(found, sums);
        if constexpr (MODE == kDw && PARTS < 3) add_rest_dw(g, sh, tl, row, side, near, found, sums);
        end_tile<MODE>(g, sh, tl, row, side, sums);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // neither CTA leaves while its peer may still signal it
  tc_fence_after();
  if (warp == 1) tmem_dealloc_pair(tmem, tcols);
}

int tmap(CUtensorMap* tm, const void* base, uint64_t inner, uint64_t rows, uint64_t ld, uint32_t box_rows) {
  const uint64_t dims[2] = {inner, rows};
  const uint64_t strides[1] = {ld * 2};
  const uint32_t box[2] = {64, box_rows};
  return make_tmap(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int MODE, int PARTS>
cudaError_t launch_parts(const HeadTc& h, int most_m, int N, unsigned* status, cudaStream_t st) {
  const size_t a_bytes = MODE == kDw ? kABytes : h.rows_box * 128u, stage = PARTS * a_bytes + (PARTS == 3 ? 3 : 1) * (h.bn / 2 * 128u);
  const size_t behind = (kABytes - a_bytes) + (MODE == kDw && PARTS < 3 ? sizeof(Near) : 0);  // the ring
  TcArgs g{h, (N + h.bn - 1) / h.bn, static_cast<int>(std::min<size_t>(kMostStages, (kRingBytes - behind) / stage)), status};
  CUtensorMap ta, tb;
  const bool a_mn = MODE == kDw, b_mn = MODE == kDx || MODE == kDw;
  if (tmap(&ta, h.A, h.inner_a, h.rows_a, h.lda, a_mn ? 64 : h.rows_box) ||
      tmap(&tb, h.B, h.inner_b, h.rows_b, h.ldb, b_mn ? 64 : h.bn / 2))
    return cudaErrorInvalidValue;
  const long long tiles = static_cast<long long>((most_m + 255) / 256) * g.nN * (b_mn ? kMostSplits : 1);
  if (tiles > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  const size_t smem = 1024 + g.stages * stage + behind + (2 * g.stages + 4) * 8 + 16;
  if (cudaError_t e = allow_smem(k_head_tc<MODE, PARTS>, smem); e != cudaSuccess) return e;
  const unsigned grid = 2u * static_cast<unsigned>(std::min<long long>(tiles, h.clusters));
  return head_launch(k_head_tc<MODE, PARTS>, true, grid, kThreads, smem, st, ta, tb, g);
}

}  // namespace

cudaError_t launch_head_logits(const HeadTc& h, unsigned* status, cudaStream_t st) {
  return h.used_a == 3 ? launch_parts<kLogits, 3>(h, h.piece_rows, h.V, status, st)
                       : launch_parts<kLogits, 1>(h, h.piece_rows, h.V, status, st);
}
cudaError_t launch_head_d(const HeadTc& h, unsigned* status, cudaStream_t st) {
  return launch_parts<kD, 1>(h, h.piece_rows, h.V, status, st);
}
cudaError_t launch_head_dx(const HeadTc& h, unsigned* status, cudaStream_t st) {
  return h.used_a == 3 ? launch_parts<kDx, 3>(h, h.piece_rows, h.d, status, st)
                       : launch_parts<kDx, 1>(h, h.piece_rows, h.d, status, st);
}
cudaError_t launch_head_dw(const HeadTc& h, unsigned* status, cudaStream_t st) {
  return h.used_a == 3   ? launch_parts<kDw, 3>(h, h.V, h.d, status, st)
         : h.used_a == 2 ? launch_parts<kDw, 2>(h, h.V, h.d, status, st)
                         : launch_parts<kDw, 1>(h, h.V, h.d, status, st);
}
