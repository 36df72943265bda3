// Distillation from a teacher's top logits and the gradient of the losses' sum. Per row
// x of V logits and list of classes j_k with the teacher's logits y_k, h the temperature:
//   p = softmax(x / h), q_k = exp(y_k / h - whole), whole the teacher's log-sum (given, or
//   the list's own),
//   loss = w sum q_k (log q_k - log p_jk),  dx = (w / h) (p - sum_k q_k e_jk);
// with a given log-sum the classes not listed are one more class on both sides,
//   q_r = max(0, 1 - sum q_k), p_r = sum of their p: loss += w q_r (log q_r - log p_r), and, with
//   Q = q_r + sum q_k the teacher's whole mass, dx = (w / h) (Q p - sum_k q_k e_jk) for the listed classes and
//   dx = (w / h) p (Q - q_r / p_r) for the others. Q is 1 unless the list's mass is above 1 (rounded logits beside the
//   log-sum of others, say) or all classes are listed.
// The sum over the classes not listed has its own maximum m_r, and that over the listed ones theirs, m_l; the
// difference m_l - m_r is formed before it is scaled, and logarithms are taken against the larger of the two: each
// keeps all its digits however far the two lie apart. With e = 2^(x f - c), f = log2(e) / h, c = m_r f rounded, and
// s_r = sum e over the classes not listed, dx = (w / h) (Q p_r - q_r) e / s_r there, whatever the sizes: p_r is no
// difference, and may be too small for a float.
//
// HBM-bound: a row is read once and its gradient written once.
// k_distill: a row lies in the shared memory of a CTA, or in slices in that of the CTAs
// of a cluster, as in k_loss. The listed classes' places there are set to -inf before the sum, so that
// the passes over the row know nothing of the list; the threads that have its entries write those
// elements of the gradient last. A warp of its own works through the next row's list while the others have a row.
// k_distill_rows: rows too long for a cluster's shared memory, in passes over global memory. Its
// passes, in which every difference x - max is formed before it is scaled, also serve rows whose
// maximum is too far from 0 for the reference c (kNearLogit), or infinite.
#include "loss_dev.cuh"

using namespace eogp;

namespace {

constexpr int kListMax = EOGP_DISTILL_MAX;
constexpr int kSeen = 8192;
constexpr int kRowThreads = 512;

// A row's list in shared memory, and what it comes to by itself: log q of an entry is (y - top) / h - whole; `sum` of q;
// the largest of the student's logits m, and t = sum q (log q - (x - m) / h), so that the loss's sum over the list
// is t + sum * (lse - m / h); s = sum 2^((x - m) f) over its classes, each once.
struct __align__(16) List {
  int cls[kListMax];       // -1: no entry
  float x[kListMax];       // the student's logit
  float q_all[kListMax];   // sum of q of the entries of this class
  uint8_t first[kListMax]; // the first entry of its class
  float sum, m, t, s, log_s;  // log_s = log2 s
  float rest, mass;        // q_r and Q
  bool live;               // the row takes part
};
using Seen = unsigned[kSeen / 32];  // of slow_row: bit c % kSeen: a class like c is listed
struct Lists {
  List l[2];
  Seen seen;
  uint8_t end[(128 - (2 * sizeof(List) + sizeof(Seen)) % 128) % 128 + 128];  // slices begin on 128 bytes
};
static_assert(sizeof(Lists) % 128 == 0, "slices begin on 128 bytes");

struct Job {
  int b, t;
  float w, lse;  // lse: the teacher's
  bool kept;
};
// Its loads do not wait for each other.
__device__ __forceinline__ Job job_of(const DistillArgs& a, int r) {
  Job j;
  locate(a.rs, r, j.b, j.t);
  const int len = a.rs.lengths ? a.rs.lengths[j.b] : a.rs.T;
  j.w = a.weights ? a.weights[r] : 1.f;
  j.lse = a.teacher_lse ? a.teacher_lse[r] : 0.f;
  j.kept = j.t < len && j.w != 0.f;
  return j;
}

__device__ __forceinline__ float term(float q, float log_q, float log_p) {
  return q > 0.f || q != q ? q * (log_q - log_p) : 0.f;
}
__device__ __forceinline__ float warp_max(float m) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
}

// (a - b) k of k2 = 2 k: the difference first, which keeps its digits, and of halves, for it may be no float. (What
// halving takes from numbers below 2^-125 is below 2^-22 even at the largest k2.)
__device__ __forceinline__ float scaled(float a, float b, float k2) { return fmaf(a, 0.5f, -0.5f * b) * k2; }
// hi += x; lo += what that rounds off.
__device__ __forceinline__ void add_exactly(float& hi, float& lo, float x) {
  const float s = hi + x, b = s - hi;
  lo += (hi - (s - b)) + (x - b);
  hi = s;
}

// One warp makes row r's list.
template <typename T>
__device__ __forceinline__ void make_list(const DistillArgs& a, const Job& j, List& l, float inv2, bool flag,
                                          unsigned* status) {
  constexpr int E = kListMax / 32;
  const int lane = threadIdx.x & 31;
  if (!j.kept) {
    if (lane == 0) l.live = false;
    return;
  }
  const long long at = j.b * a.classes.bs + j.t * a.classes.ld + lane, aty = j.b * a.teacher.bs + j.t * a.teacher.ld + lane;
  const T* const row = row_of<T>(a.logits, j.b, j.t);
  long long raw[E];
  float y[E], x[E];
  int c[E];
  // Loads of a kind are all under way before one is looked at.
#pragma unroll
  for (int e = 0; e < E; ++e) {
    raw[e] = -1;
    y[e] = 0.f;
    if (lane + 32 * e < a.K) {
      raw[e] = a.classes_i64 ? static_cast<const long long*>(a.classes.p)[at + 32 * e]
                             : static_cast<const int*>(a.classes.p)[at + 32 * e];
      y[e] = a.teacher_bf16 ? to_f32(static_cast<const bf16*>(a.teacher.p)[aty + 32 * e])
                            : static_cast<const float*>(a.teacher.p)[aty + 32 * e];
    }
  }
  bool bad = false, any = false;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    bad |= raw[e] >= a.V;
    c[e] = raw[e] < 0 || raw[e] >= a.V ? -1 : static_cast<int>(raw[e]);
    x[e] = c[e] >= 0 ? to_f32(row[c[e]]) : 0.f;
    any |= c[e] >= 0 && !(y[e] == -INFINITY);
    l.cls[lane + 32 * e] = c[e];
  }
  bad = __any_sync(0xffffffffu, bad);
  any = __any_sync(0xffffffffu, any) || a.teacher_lse;
  if (bad && lane == 0 && flag) flag_status(status, EOGP_ST_DEVICE);
  if (bad || !any) {
    if (lane == 0) l.live = false;
    return;
  }
  float top = -INFINITY, m = kLowest;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (c[e] < 0) continue;
    top = fmaxf(top, y[e]);
    m = fmaxf(m, x[e]);
  }
  m = warp_max(m);
  float whole = j.lse, sum = 0.f, t = 0.f;
  if (a.teacher_lse) {
    top = 0.f;
  } else {
    top = warp_max(top);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (c[e] >= 0) s += expf(scaled(y[e], top, inv2));
    whole = logf(warp_sum(s));
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float lq = scaled(y[e], top, inv2) - whole, q = c[e] >= 0 ? expf(lq) : 0.f;
    sum += q;
    t += term(q, lq, scaled(x[e], m, inv2));
    y[e] = q;
    l.x[lane + 32 * e] = x[e];
    l.q_all[lane + 32 * e] = q;
  }
  float rest = 0.f;
  if (a.teacher_lse) {
    // q_r may be a small difference: what the sum's additions round off is summed too. (In fp64 the list's warp took
    // 8 % of the time of 4 x 2048 rows of 100,096 with 128 entries.)
    float hi = 0.f, lo = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (32 * e < a.K) add_exactly(hi, lo, y[e]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      lo += __shfl_xor_sync(0xffffffffu, lo, o);
      add_exactly(hi, lo, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    sum = hi + lo;
    rest = fmaxf(0.f, (1.f - hi) - lo);
  } else {
    sum = warp_sum(sum);
  }
  __syncwarp();
  // Entries of the same class: how many, and whether one comes before.
  int same[E];
  bool first[E];
#pragma unroll
  for (int e = 0; e < E; ++e) same[e] = 0, first[e] = c[e] >= 0;
  for (int i = 0; i < a.K; i += 4) {  // past K: no entries
    const int4 o = *reinterpret_cast<const int4*>(&l.cls[i]);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (32 * e >= a.K) break;
      const int k = lane + 32 * e;
      same[e] += (o.x == c[e]) + (o.y == c[e]) + (o.z == c[e]) + (o.w == c[e]);
      first[e] &= !((o.x == c[e] && i < k) || (o.y == c[e] && i + 1 < k) || (o.z == c[e] && i + 2 < k) ||
                    (o.w == c[e] && i + 3 < k));
    }
  }
  bool twice = false;
  float s = 0.f, classes = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    twice |= c[e] >= 0 && same[e] > 1;
    l.first[lane + 32 * e] = first[e];
    if (first[e]) {
      s += expf(scaled(x[e], m, inv2));
      classes += 1.f;
    }
  }
  if (__any_sync(0xffffffffu, twice)) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      y[e] = 0.f;
      if (c[e] >= 0)
        for (int i = 0; i < a.K; ++i)
          if (l.cls[i] == c[e]) y[e] += l.q_all[i];
    }
    __syncwarp();
#pragma unroll
    for (int e = 0; e < E; ++e) l.q_all[lane + 32 * e] = y[e];
  }
  t = warp_sum(t);
  s = warp_sum(s);
  classes = warp_sum(classes);
  if (lane == 0) {
    l.sum = sum;
    l.m = m;
    l.t = t;
    l.s = s;
    l.log_s = log2f(s);
    l.live = true;
    l.rest = classes != static_cast<float>(a.V) ? rest : 0.f;
    l.mass = a.teacher_lse && !(l.rest > 0.f) ? sum : 1.f;
  }
  __syncwarp();
}
// The loss's sum over the list; none for a list of q = 0, whose maximum may be as far away as it likes.
__device__ __forceinline__ float list_loss(const List& l, float lse_against_m) {
  return l.sum == 0.f ? 0.f : fmaf(l.sum, lse_against_m, l.t);
}

__device__ __forceinline__ void put_loss(const DistillArgs& a, int r, float loss, float lse) {
  a.loss[r] = loss;
  if (a.lse) a.lse[r] = lse;
}

// -------------------------------------------------------------- any row, slowly
// Threads 0 .. nt - 1 of a block, which may have others.
__device__ __forceinline__ void meet(int nt) { named_bar_sync(1, nt); }
__device__ __forceinline__ float block_max(float m, float* part, int nt) {
  m = warp_max(m);
  meet(nt);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  meet(nt);
  m = part[0];
  for (int w = 1; w < nt >> 5; ++w) m = fmaxf(m, part[w]);
  return m;
}
__device__ __forceinline__ float block_add(float s, float* part, int nt) {
  s = warp_sum(s);
  meet(nt);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  meet(nt);
  s = 0.f;
  for (int w = 0; w < nt >> 5; ++w) s += part[w];
  return s;
}

// nt threads on row r, whose list is complete in shared memory.
template <typename T>
__device__ __noinline__ void slow_row(const DistillArgs& a, int r, const Job& j, const List& l, Seen& seen, int nt) {
  __shared__ float part[kRowThreads / 32];
  const int tid = threadIdx.x;
  const T* const x = row_of<T>(a.logits, j.b, j.t);
  const float inv_h = 1.f / a.temperature, f = kLog2e * inv_h, inv2 = 2.f * inv_h, f2 = 2.f * f;
  for (int k = tid; k < kSeen / 32; k += nt) seen[k] = 0u;
  meet(nt);
  for (int k = tid; k < a.K; k += nt) {
    const int c = l.cls[k];
    if (c >= 0) atomicOr(&seen[c % kSeen / 32], 1u << c % 32);
  }
  meet(nt);
  auto listed = [&](int c) {
    if (!(seen[c % kSeen / 32] >> c % 32 & 1u)) return -1;
    for (int k = 0; k < a.K; ++k)
      if (l.cls[k] == c) return k;
    return -1;
  };
  float m = kLowest;
  for (int c = tid; c < a.V; c += nt) {
    const float v = to_f32(x[c]);
    if (v > m && listed(c) < 0) m = v;
  }
  const float m_r = block_max(m, part, nt);
  float s = 0.f;
  for (int c = tid; c < a.V; c += nt) {
    const float v = to_f32(x[c]);
    if (v != -INFINITY && listed(c) < 0) s += exp2_fast(scaled(v, m_r, f2));
  }
  const float s_r = block_add(s, part, nt);
  m = fmaxf(l.m, m_r);
  s = l.s * exp2_fast(scaled(l.m, m, f2)) + s_r * exp2_fast(scaled(m_r, m, f2));
  const float ls = s > 0.f ? logf(s) : NAN;  // no finite logit: NaN
  const float log_pr = scaled(m_r, m, inv2) + (logf(s_r) - ls);
  if (tid == 0)
    put_loss(a, r, j.w * (list_loss(l, scaled(m, l.m, inv2) + ls) + term(l.rest, logf(l.rest), log_pr)), m * inv_h + ls);
  if (!a.dlogits.p) return;
  T* const g = row_out<T>(a.dlogits, j.b, j.t);
  const float wt = j.w * inv_h;
  const float out = s_r > 0.f ? wt * (l.mass * expf(log_pr) - l.rest) / s_r : ls * 0.f;
  for (int c = tid; c < a.V; c += nt) {
    const float xc = to_f32(x[c]);
    const int k = listed(c);
    g[c] = from_f32<T>(k >= 0 ? wt * (l.mass * expf(scaled(xc, m, inv2) - ls) - l.q_all[k]) : exp2_fast(scaled(xc, m_r, f2)) * out);
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_distill_rows(const DistillArgs a, unsigned* status) {
  __shared__ List l;
  __shared__ Seen seen;
  const int r = blockIdx.x, tid = threadIdx.x;
  const Job j = job_of(a, r);
  if (tid < 32) make_list<T>(a, j, l, 2.f * (1.f / a.temperature), true, status);
  __syncthreads();
  if (l.live) return slow_row<T>(a, r, j, l, seen, kRowThreads);
  if (tid == 0) put_loss(a, r, 0.f, 0.f);
  if (!a.dlogits.p) return;
  T* const g = row_out<T>(a.dlogits, j.b, j.t);
  for (int c = tid; c < a.V; c += kRowThreads) g[c] = from_f32<T>(0.f);
}

// ----------------------------------------------------------------- slices of rows
// A cluster works on `rows` consecutive rows; what k_loss says of its copies, its exchange and an expired wait
// holds here. Every CTA has the whole list, made by its last warp; the other nt threads meet at barrier 1, and all
// of them at barrier 2 at the start of a row: its list is there, and that of the row before has been read.
template <typename T, bool GRAD>
__global__ void __launch_bounds__(kSliceThreads + 32, 2) k_distill(const DistillArgs a, int M, int rows, int per, int cs,
                                                                   unsigned* status) {
  constexpr int N = 16 / sizeof(T), K = 4;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ MaxSum part[kSliceThreads / 32], peers[2][kMaxCluster], all;
  __shared__ volatile int lost;  // the row whose exchange ran out; r1: none
  __shared__ uint64_t bar[2];
  const int tid = threadIdx.x, nt = blockDim.x - 32, nw = nt >> 5;
  const int rank = cs > 1 ? static_cast<int>(blockIdx.x % cs) : 0;
  const int r0 = static_cast<int>(blockIdx.x / cs) * rows, r1 = min(M, r0 + rows);
  const bool first_cta = rank == 0;
  Lists& ls_ = *reinterpret_cast<Lists*>(smem);
  Raw<T, N>* const slice = reinterpret_cast<Raw<T, N>*>(smem + sizeof(Lists));
  const float inv_h = 1.f / a.temperature, f = kLog2e * inv_h, inv2 = 2.f * inv_h, f2 = 2.f * f;
  if (tid == 0) lost = r1;
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
  if (tid >= nt) {
    for (int r = r0; r < r1; ++r) {
      make_list<T>(a, job_of(a, r), ls_.l[(r - r0) & 1], inv2, first_cta, status);
      named_bar_sync(2, nt + 32);
      // Of an earlier row: the others came to barrier 2 once more, with that written before, and not again. Of this
      // row, which may be written meanwhile: they will come once more.
      if (lost < r) break;
    }
    if (cs > 1) cluster_wait();
    return;
  }
  bool met = cs == 1;
  int turn = 0;  // exchanges so far: they alternate between two sets of slots

  struct Part {
    Job j;
    RowVecs<T> row;
    const T* x;
    int v0, n;  // first vector and number of vectors of the slice; n = 0 for a row left out
  };
  auto part_of = [&](const Job& j) {
    const T* const x = row_of<T>(a.logits, j.b, j.t);
    const RowVecs<T> row(x, a.V);
    const int v0 = row.f0 + rank * per;
    return Part{j, row, x, v0, j.kept ? max(0, min(row.f1 - v0, per)) : 0};
  };
  auto ask = [&](const Part& p, int k) { copy_async<T, N>(slice + k, p.x + p.row.col(p.v0 + k)); };
  auto edge_of = [&](const Part& p) { return p.j.kept && first_cta ? p.row.edge(tid) : -1; };

  Part p = part_of(job_of(a, r0));
  for (int k = tid; k < p.n; k += nt) ask(p, k);
  int ce = edge_of(p);
  float xe = ce >= 0 ? to_f32(p.x[ce]) : 0.f;
  int r = r0;
  for (; r < r1; ++r) {
    Job jn = p.j;
    jn.kept = false;
    if (r + 1 < r1) jn = job_of(a, r + 1);
    T* const g = GRAD ? row_out<T>(a.dlogits, p.j.b, p.j.t) : nullptr;
    const List& l = ls_.l[(r - r0) & 1];
    commit_async();
    wait_async<0>();
    named_bar_sync(2, nt + 32);  // the list, and all threads' copies of the slice
    const Part next = part_of(jn);
    if (!l.live) {  // in every CTA of the cluster
      if (GRAD) {
        const RowVecs<T> out(g, a.V);
        const int v0 = out.f0 + rank * per;
        zero_vecs<T>(g, out, v0, min(out.f1, v0 + per), tid, nt, first_cta);
      }
      if (tid == 0 && first_cta) put_loss(a, r, 0.f, 0.f);
      for (int k = tid; k < next.n; k += nt) ask(next, k);
    } else {
      const int col0 = p.row.col(p.v0);
      for (int k = tid; k < a.K; k += nt) {
        const int at = l.cls[k] - col0;
        if (l.first[k] && static_cast<unsigned>(at) < static_cast<unsigned>(p.n * N))
          reinterpret_cast<T*>(slice)[at] = from_f32<T>(-INFINITY);
      }
      if (ce >= 0) {
        for (int k = 0; k < a.K; k += 4) {
          const int4 o = *reinterpret_cast<const int4*>(&l.cls[k]);
          if (o.x == ce || o.y == ce || o.z == ce || o.w == ce) xe = -INFINITY;
        }
      }
      meet(nt);  // the listed classes' places
      MaxSum v{-INFINITY, 0.f};
      int k = tid;
      for (; k + (K - 1) * nt < p.n; k += K * nt) {
        Raw<T, N> w[K];
#pragma unroll
        for (int u = 0; u < K; ++u) w[u] = slice[k + u * nt];
        add_vecs<T, N, K>(v, w, f);
      }
      for (; k < p.n; k += nt) {
        const Raw<T, N> w[1] = {slice[k]};
        add_vecs<T, N, 1>(v, w, f);
      }
      if (ce >= 0) add_one(v, xe, f);
      if (!GRAD)
        for (int i = tid; i < next.n; i += nt) ask(next, i);
      v = warp_join(v, f);
      if ((tid & 31) == 0) part[tid >> 5] = v;
      meet(nt);
      v = join_all(part, nw, f);
      if (cs > 1) {
        const int set = turn & 1;
        if (!met) cluster_wait();  // every CTA of the cluster runs, its mbarriers set
        met = true;
        if (tid < 32) {
          if (tid < cs) put_peer(&peers[set][rank], &bar[set], tid, v);
          const bool came = __all_sync(0xffffffffu, mbar_wait_cluster(&bar[set], (turn >> 1) & 1, status));
          if (tid == 0) {
            if (!came) lost = r;
            if (came) {
              mbar_arrive_expect_tx(&bar[set], cs * sizeof(MaxSum));  // for the turn after next
              all = join_all(peers[set], cs, f);
            }
          }
        }
        meet(nt);
        if (lost < r1) break;
        v = all;
        ++turn;
      }
      if (!(fabsf(v.m) * f <= kNearLogit * kLog2e)) {  // in every CTA of the cluster
        if (first_cta) slow_row<T>(a, r, p.j, l, ls_.seen, nt);
        if (GRAD)
          for (int i = tid; i < next.n; i += nt) ask(next, i);
      } else {
        // How far the list's maximum and the others' lie below the larger of the two, and logarithms to base 2 against
        // that: of the sums over the list, over the others (which knows what c was rounded by), and over both.
        const float c = ref(v.m, f), gap = scaled(l.m, v.m, inv2), to_list = fminf(gap, 0.f), to_rest = fminf(-gap, 0.f);
        const float log_s = log2f(v.s) + fmaf(-v.m, f, c);
        const float to_l = fmaf(to_list, kLog2e, l.log_s), to_r = fmaf(to_rest, kLog2e, log_s);
        const float ls = fmaxf(to_l, to_r) + log2f(1.f + exp2_fast(-fabsf(to_l - to_r)));  // = to_r beside an empty list
        const float log_pr = fmaf(kLn2, log_s - ls, to_rest);
        if (tid == 0 && first_cta)
          put_loss(a, r, p.j.w * (list_loss(l, fmaf(kLn2, ls, -to_list)) + term(l.rest, logf(l.rest), log_pr)),
                   fmaf(kLn2, ls, fmaxf(l.m, v.m) * inv_h));
        if (GRAD) {
          const RowVecs<T> out(g, a.V);
          const float wt = p.j.w * inv_h, to = wt * (l.mass * exp2_fast(to_r - ls) - l.rest) / v.s;
          const float at = fmaf(to_list, kLog2e, -ls);
          if (ce >= 0) g[ce] = from_f32<T>(exp2_fast(fmaf(xe, f, -c)) * to);
          if (out.ph == p.row.ph) {
            T* o = g + col0 + tid * N;
            const int both = min(p.n, next.n);
            int i = tid;
#pragma unroll 4
            for (; i < both; i += nt, o += nt * N) {
              st_vals<T, N>(o, grad_of<T, N>(slice[i], c, to, f));
              ask(next, i);
            }
#pragma unroll 4
            for (; i < p.n; i += nt, o += nt * N) st_vals<T, N>(o, grad_of<T, N>(slice[i], c, to, f));
            for (; i < next.n; i += nt) ask(next, i);
          } else {
            // dlogits lies otherwise to 16 bytes than logits: by way of shared memory,
            // an element a thread.
            for (int i = tid; i < p.n; i += nt) slice[i] = pack_raw<T, N>(grad_of<T, N>(slice[i], c, to, f));
            meet(nt);
            const T* const from = reinterpret_cast<const T*>(slice);
            for (int i = tid; i < p.n * N; i += nt) g[col0 + i] = from[i];
            meet(nt);
            for (int i = tid; i < next.n; i += nt) ask(next, i);
          }
          meet(nt);  // the row's other elements, which the listed ones go over
          const int inner = p.row.head + (p.row.f1 - p.row.f0) * N;
          for (int k = tid; k < a.K; k += nt) {
            const int ck = l.cls[k];
            const bool edge = ck < p.row.head || ck >= inner;
            if (l.first[k] && (edge ? first_cta : static_cast<unsigned>(ck - col0) < static_cast<unsigned>(p.n * N)))
              g[ck] = from_f32<T>(wt * (l.mass * exp2_fast(scaled(l.x[k], l.m, f2) + at) - l.q_all[k]));
          }
        }
      }
    }
    p = next;
    ce = edge_of(p);
    xe = ce >= 0 ? to_f32(p.x[ce]) : 0.f;
  }
  if (!met) cluster_wait();
  if (cs > 1 && met && lost < r1) {
    if (r + 1 < r1) named_bar_sync(2, nt + 32);  // the last warp stops too
    commit_async();
    wait_async<0>();
    cluster_arrive();
    cluster_wait();  // for the threads of the cluster that have not ended
  }
}

template <typename T>
cudaError_t distill_launch(const DistillArgs& a, unsigned* status, int num_sms, cudaStream_t st) {
  constexpr int N = 16 / sizeof(T);
  const int M = static_cast<int>(a.rs.rows());
  const int nv = a.V / N;  // whole vectors of a row at most
  // Rows of up to 101 KB stay in one CTA, two of which share a multiprocessor beside their lists; longer ones are
  // cut into slices of up to that: every CTA of a cluster works through the whole list (4 x 2048 rows of 100,096 with
  // 128 entries: 0.79 ms in slices of 48 KB, 0.54 ms so). Few rows: spread over the multiprocessors.
  const long long bytes = nv * 16ll;
  int cs = 1;
  while (cs < kMaxCluster && bytes > 101 * 1024ll * cs) cs *= 2;
  while (cs < kMaxCluster && static_cast<long long>(M) * cs * 2 <= num_sms && nv / cs >= 512) cs *= 2;
  const int per = (nv + cs - 1) / cs;
  const bool grad = a.dlogits.p != nullptr;
  const long long smem = sizeof(Lists) + per * 16ll;
  if (smem > 220 * 1024 || static_cast<long long>(M) * cs > 0x7FFFFFFFLL) {
    k_distill_rows<T><<<M, kRowThreads, 0, st>>>(a, status);
    return cudaGetLastError();
  }
  const int each = static_cast<long long>(M) * cs < 2 * num_sms ? 12 : 14;
  const int threads = std::min(kSliceThreads, std::max(64, (per / each + 31) / 32 * 32));
  const int rows = loss_rows(M, cs, threads, num_sms);
  auto k = grad ? k_distill<T, true> : k_distill<T, false>;
  if (cudaError_t e = allow_smem(k, smem); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>((M + rows - 1) / rows) * cs);
  cfg.blockDim = dim3(threads + 32);
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

cudaError_t launch_distill(const DistillArgs& a, bool bf16_, unsigned* status, int num_sms, cudaStream_t st) {
  return bf16_ ? distill_launch<bf16>(a, status, num_sms, st) : distill_launch<float>(a, status, num_sms, st);
}
