// Distillation from a teacher's top logits and the gradient of the losses' sum. Per row
// x of V logits and list of classes j_k with the teacher's logits y_k, h the temperature:
//   p = softmax(x / h), q_k = exp(y_k / h - whole), whole the teacher's log-sum (given, or
//   the list's own),
//   loss = w sum q_k (log q_k - log p_jk),  dx = (w / h) (p - sum_k q_k e_jk);
// with a given log-sum the classes not listed are one more class on both sides,
//   q_r = max(0, 1 - sum q_k), p_r = sum of their p: loss += w q_r (log q_r - log p_r), and
//   dx = (w / h) p (1 - q_r / p_r) for them.
// The sum over the classes not listed has its own maximum m_r, and so log p_r has all its digits; with
// e = 2^(x f - c), f = log2(e) / h, c = m_r f, and s_r = sum e over those classes,
// dx = (w / h) (p_r - q_r) e / s_r there, whatever the sizes: p_r is no difference, and may be too
// small for a float.
//
// HBM-bound: a row is read once and its gradient written once.
// k_distill: a row lies in the shared memory of a CTA, or in slices in that of the CTAs
// of a cluster, as in k_loss. The listed classes' places there are set to -inf before the sum, so that
// the passes over the row know nothing of the list; the threads that have its entries write those
// elements of the gradient last. The next row's entries are asked for while a row is worked on.
// k_distill_rows: rows too long for a cluster's shared memory, in passes over global memory. Its
// passes, in which every difference x - max is formed before it is scaled, also serve rows whose
// maximum is too far from 0 for the reference c (kNearLogit), or infinite.
#include "loss_dev.cuh"

using namespace eogp;

namespace {

constexpr int kListMax = EOGP_DISTILL_MAX;
constexpr int kSeen = 8192;
constexpr int kRowThreads = 512;
constexpr float kLowest = -3.402823466e38f;

// A row's list in shared memory.
struct __align__(16) List {
  int cls[kListMax];         // -1: no entry; -2: out of range
  float y[kListMax];         // the teacher's logit
  float x[kListMax];         // the student's
  float q_all[kListMax];     // sum of q of the entries of this class
  uint8_t first[kListMax];   // the first entry of its class
  unsigned seen[kSeen / 32]; // of slow_row: bit c % kSeen: a class like c is listed
};

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

// An entry as it lies in memory; looked at only when it is needed.
struct RawEntry {
  long long c;
  uint32_t y;
};
__device__ __forceinline__ RawEntry ask_entry(const DistillArgs& a, const Job& j, int k) {
  RawEntry e;
  const long long c = j.b * a.classes.bs + j.t * a.classes.ld + k, y = j.b * a.teacher.bs + j.t * a.teacher.ld + k;
  e.c = a.classes_i64 ? static_cast<const long long*>(a.classes.p)[c] : static_cast<const int*>(a.classes.p)[c];
  e.y = a.teacher_bf16 ? static_cast<const uint16_t*>(a.teacher.p)[y] : static_cast<const uint32_t*>(a.teacher.p)[y];
  return e;
}
struct Entry {
  int c;
  float y, x;
};
template <typename T>
__device__ __forceinline__ Entry entry_of(const DistillArgs& a, const Job& j, const RawEntry& e) {
  Entry r;
  r.c = e.c < 0 ? -1 : e.c >= a.V ? -2 : static_cast<int>(e.c);
  r.y = __uint_as_float(a.teacher_bf16 ? e.y << 16 : e.y);
  r.x = r.c >= 0 ? to_f32(row_of<T>(a.logits, j.b, j.t)[r.c]) : 0.f;
  return r;
}

// What a list comes to by itself, by every warp alone: log q of an entry is (y - top) / h - whole; sum of q; the
// largest of the student's logits m, and t = sum q (log q - (x - m) / h), so that the loss's sum over
// the list is t + sum * (lse - m / h).
struct Sums {
  float top, whole, sum, m, t;
  bool bad, some;  // a class out of range; something to learn from
};
__device__ __forceinline__ float log_q_of(const Sums& t, float y, float inv_h) { return (y - t.top) * inv_h - t.whole; }
__device__ __forceinline__ float term(float q, float log_q, float log_p) {
  return q > 0.f || q != q ? q * (log_q - log_p) : 0.f;
}
__device__ __forceinline__ Sums sums_of(const DistillArgs& a, const List& l, const Job& j, float inv_h) {
  const int lane = threadIdx.x & 31;
  Sums t;
  float top = -INFINITY, m = kLowest;
  bool bad = false, any = false;
  for (int k = lane; k < a.K; k += 32) {
    const int c = l.cls[k];
    const float y = l.y[k];
    bad |= c == -2;
    if (c < 0) continue;
    any |= !(y == -INFINITY);
    top = fmaxf(top, y);
    m = fmaxf(m, l.x[k]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  t.bad = __any_sync(0xffffffffu, bad);
  t.some = __any_sync(0xffffffffu, any) || a.teacher_lse;
  t.m = m;
  t.top = 0.f;
  t.whole = j.lse;
  if (!a.teacher_lse) {
    float s = 0.f;
    for (int k = lane; k < a.K; k += 32)
      if (l.cls[k] >= 0) s += expf((l.y[k] - top) * inv_h);
    t.top = top;
    t.whole = logf(warp_sum(s));
  }
  float sum = 0.f, v = 0.f;
  for (int k = lane; k < a.K; k += 32) {
    if (l.cls[k] < 0) continue;
    const float lq = log_q_of(t, l.y[k], inv_h), q = expf(lq);
    sum += q;
    v += term(q, lq, (l.x[k] - m) * inv_h);
  }
  t.sum = warp_sum(sum);
  t.t = warp_sum(v);
  return t;
}

// The loss's sum over the list; none for a list of q = 0, whose maximum may be as far away as it likes.
__device__ __forceinline__ float list_loss(const Sums& t, float lse_against_m) {
  return t.sum == 0.f ? 0.f : fmaf(t.sum, lse_against_m, t.t);
}

// Whether entry k, of class c, is its class's first, and the sum of q over the class's entries, q its own.
__device__ __forceinline__ bool look_up(const List& l, const Sums& t, int K, int k, int c, float q, float inv_h,
                                        float& q_all) {
  int same = 0;
  bool first = c >= 0;
  for (int i = 0; i < K; i += 4) {  // past K: no entries
    const int4 o = *reinterpret_cast<const int4*>(&l.cls[i]);
    same += (o.x == c) + (o.y == c) + (o.z == c) + (o.w == c);
    first &= !((o.x == c && i < k) || (o.y == c && i + 1 < k) || (o.z == c && i + 2 < k) || (o.w == c && i + 3 < k));
  }
  q_all = q;
  if (c >= 0 && same > 1) {
    q_all = 0.f;
    for (int i = 0; i < K; ++i)
      if (l.cls[i] == c) q_all += expf(log_q_of(t, l.y[i], inv_h));
  }
  return first;
}

__device__ __forceinline__ void put_loss(const DistillArgs& a, int r, float loss, float lse) {
  a.loss[r] = loss;
  if (a.lse) a.lse[r] = lse;
}

// -------------------------------------------------------------- any row, slowly
__device__ __forceinline__ float block_max(float m, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
  m = part[0];
  for (unsigned w = 1; w < blockDim.x >> 5; ++w) m = fmaxf(m, part[w]);
  return m;
}
__device__ __forceinline__ float block_add(float s, float* part) {
  s = warp_sum(s);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  s = 0.f;
  for (unsigned w = 0; w < blockDim.x >> 5; ++w) s += part[w];
  return s;
}

// One block on row r, whose list is complete in shared memory.
template <typename T>
__device__ __noinline__ void slow_row(const DistillArgs& a, int r, const Job& j, List& l, const Sums& t) {
  __shared__ float part[kRowThreads / 32];
  const int tid = threadIdx.x, nt = blockDim.x;
  const T* const x = row_of<T>(a.logits, j.b, j.t);
  const float inv_h = 1.f / a.temperature, f = kLog2e * inv_h;
  for (int k = tid; k < kSeen / 32; k += nt) l.seen[k] = 0u;
  __syncthreads();
  float classes = 0.f;
  for (int k = tid; k < a.K; k += nt) {
    const int c = l.cls[k];
    if (c >= 0) atomicOr(&l.seen[c % kSeen / 32], 1u << c % 32);
    classes += l.first[k];
  }
  const bool whole = block_add(classes, part) == static_cast<float>(a.V);
  auto listed = [&](int c) {
    if (!(l.seen[c % kSeen / 32] >> c % 32 & 1u)) return -1;
    for (int k = 0; k < a.K; ++k)
      if (l.cls[k] == c) return k;
    return -1;
  };
  float m = kLowest;
  for (int c = tid; c < a.V; c += nt) {
    const float v = to_f32(x[c]);
    if (v > m && listed(c) < 0) m = v;
  }
  const float m_r = block_max(m, part);
  float s = 0.f;
  for (int c = tid; c < a.V; c += nt) {
    const float v = to_f32(x[c]);
    if (v != -INFINITY && listed(c) < 0) s += exp2_fast((v - m_r) * f);
  }
  const float s_r = block_add(s, part);
  m = fmaxf(t.m, m_r);
  s = 0.f;
  for (int k = tid; k < a.K; k += nt)
    if (l.first[k]) s += exp2_fast((l.x[k] - m) * f);
  s = block_add(s, part) + s_r * exp2_fast((m_r - m) * f);
  const float ls = s > 0.f ? logf(s) : NAN;  // no finite logit: NaN
  const float log_pr = (m_r - m) * inv_h + (logf(s_r) - ls);
  const float q_r = a.teacher_lse && !whole ? fmaxf(0.f, 1.f - t.sum) : 0.f;
  if (tid == 0)
    put_loss(a, r, j.w * (list_loss(t, (m - t.m) * inv_h + ls) + term(q_r, logf(q_r), log_pr)), m * inv_h + ls);
  if (!a.dlogits.p) return;
  T* const g = row_out<T>(a.dlogits, j.b, j.t);
  const float wt = j.w * inv_h;
  const float out = s_r > 0.f ? wt * (expf(log_pr) - q_r) / s_r : ls * 0.f;
  for (int c = tid; c < a.V; c += nt) {
    const float xc = to_f32(x[c]);
    const int k = listed(c);
    g[c] = from_f32<T>(k >= 0 ? wt * (expf((xc - m) * inv_h - ls) - l.q_all[k]) : exp2_fast((xc - m_r) * f) * out);
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_distill_rows(const DistillArgs a, unsigned* status) {
  __shared__ List l;
  const int r = blockIdx.x, tid = threadIdx.x;
  const Job j = job_of(a, r);
  const float inv_h = 1.f / a.temperature;
  Sums t{};
  if (j.kept) {
    if (tid < kListMax) {
      Entry e{-1, 0.f, 0.f};
      if (tid < a.K) e = entry_of<T>(a, j, ask_entry(a, j, tid));
      l.cls[tid] = e.c;
      l.y[tid] = e.y;
      l.x[tid] = e.x;
    }
    __syncthreads();
    t = sums_of(a, l, j, inv_h);
    if (t.bad && tid == 0) flag_status(status, EOGP_ST_DEVICE);
  }
  if (!j.kept || t.bad || !t.some) {
    if (tid == 0) put_loss(a, r, 0.f, 0.f);
    if (!a.dlogits.p) return;
    T* const g = row_out<T>(a.dlogits, j.b, j.t);
    for (int c = tid; c < a.V; c += kRowThreads) g[c] = from_f32<T>(0.f);
    return;
  }
  if (tid < a.K)
    l.first[tid] = look_up(l, t, a.K, tid, l.cls[tid], expf(log_q_of(t, l.y[tid], inv_h)), inv_h, l.q_all[tid]);
  __syncthreads();
  slow_row<T>(a, r, j, l, t);
}

// ----------------------------------------------------------------- slices of rows
// A cluster works on `rows` consecutive rows; what k_loss says of its copies, its exchange and an expired wait
// holds here. Every CTA has the whole list. Two entries a thread at most.
constexpr int kEach = 2;

template <typename T, bool GRAD>
__global__ void __launch_bounds__(kSliceThreads, 2) k_distill(const DistillArgs a, int M, int rows, int per, int cs,
                                                              unsigned* status) {
  constexpr int N = 16 / sizeof(T), K = 4;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ MaxSum part[kSliceThreads / 32], peers[2][kMaxCluster], all;
  __shared__ bool lost;
  __shared__ uint64_t bar[2];
  const int tid = threadIdx.x, nt = blockDim.x, nw = nt >> 5, lane = tid & 31;
  const int rank = cs > 1 ? static_cast<int>(blockIdx.x % cs) : 0;
  const int r0 = static_cast<int>(blockIdx.x / cs) * rows, r1 = min(M, r0 + rows);
  const bool first_cta = rank == 0;
  List& l = *reinterpret_cast<List*>(smem);
  Raw<T, N>* const slice = reinterpret_cast<Raw<T, N>*>(smem + sizeof(List));
  const float inv_h = 1.f / a.temperature, f = kLog2e * inv_h;
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
  auto ask_list = [&](const Job& j, RawEntry (&e)[kEach]) {
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int k = tid + u * nt;
      e[u] = RawEntry{-1, 0u};
      if (j.kept && k < a.K) e[u] = ask_entry(a, j, k);
    }
  };
  auto take_list = [&](const Job& j, const RawEntry (&e)[kEach], Entry (&o)[kEach]) {
#pragma unroll
    for (int u = 0; u < kEach; ++u) o[u] = entry_of<T>(a, j, e[u]);
  };

  Part p = part_of(job_of(a, r0));
  RawEntry raw[kEach];
  Entry own[kEach];
  ask_list(p.j, raw);
  for (int k = tid; k < p.n; k += nt) ask(p, k);
  int ce = edge_of(p);
  float xe = ce >= 0 ? to_f32(p.x[ce]) : 0.f;
  take_list(p.j, raw, own);
  if (tid < kListMax - a.K) l.cls[a.K + tid] = -1;  // no entries beyond the list
  if (nt + tid < kListMax - a.K) l.cls[a.K + nt + tid] = -1;
  for (int r = r0; r < r1; ++r) {
    Job jn = p.j;
    jn.kept = false;
    if (r + 1 < r1) jn = job_of(a, r + 1);
    ask_list(jn, raw);
    Entry nxt[kEach];
    T* const g = GRAD ? row_out<T>(a.dlogits, p.j.b, p.j.t) : nullptr;
    Sums t{};
    if (p.j.kept) {  // in every CTA of the cluster
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const int k = tid + u * nt;
        if (k < a.K) {
          l.cls[k] = own[u].c;
          l.y[k] = own[u].y;
          l.x[k] = own[u].x;
        }
      }
      commit_async();
      __syncthreads();  // the list; what is done with it comes while the slice's copies arrive
      t = sums_of(a, l, p.j, inv_h);
      if (t.bad && tid == 0 && first_cta) flag_status(status, EOGP_ST_DEVICE);
    }
    if (!p.j.kept || t.bad || !t.some) {  // likewise
      if (GRAD) {
        const RowVecs<T> out(g, a.V);
        const int v0 = out.f0 + rank * per;
        zero_vecs<T>(g, out, v0, min(out.f1, v0 + per), tid, nt, first_cta);
      }
      if (tid == 0 && first_cta) put_loss(a, r, 0.f, 0.f);
      wait_async<0>();  // no copy lands on the next one
      take_list(jn, raw, nxt);
      p = part_of(jn);
      for (int k = tid; k < p.n; k += nt) ask(p, k);
      __syncthreads();  // the list has been read
    } else {
      const int col0 = p.row.col(p.v0);
      bool first[kEach];
      float q_all[kEach];
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const int k = tid + u * nt;
        first[u] = false;
        if (k < a.K) {
          first[u] = look_up(l, t, a.K, k, own[u].c, expf(log_q_of(t, own[u].y, inv_h)), inv_h, q_all[u]);
          l.first[k] = first[u];
          l.q_all[k] = q_all[u];
        }
      }
      wait_async<0>();
      __syncthreads();  // all threads' copies of the slice
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        if (first[u]) {
          const int at = own[u].c - col0;
          if (static_cast<unsigned>(at) < static_cast<unsigned>(p.n * N))
            reinterpret_cast<T*>(slice)[at] = from_f32<T>(-INFINITY);
        }
      }
      if (ce >= 0) {
        for (int k = 0; k < a.K; k += 4) {
          const int4 o = *reinterpret_cast<const int4*>(&l.cls[k]);
          if (o.x == ce || o.y == ce || o.z == ce || o.w == ce) xe = -INFINITY;
        }
      }
      // The list's own sum, against its maximum, and its classes.
      float s_l = 0.f, classes = 0.f;
      for (int i = lane; i < a.K; i += 32)
        if (l.first[i]) {
          s_l += exp2_fast((l.x[i] - t.m) * f);
          classes += 1.f;
        }
      s_l = warp_sum(s_l);
      const bool whole = warp_sum(classes) == static_cast<float>(a.V);
      __syncthreads();  // the listed classes' places
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
      take_list(jn, raw, nxt);
      const Part next = part_of(jn);
      if (!GRAD)
        for (int i = tid; i < next.n; i += nt) ask(next, i);
      v = warp_join(v, f);
      if (lane == 0) part[tid >> 5] = v;
      __syncthreads();
      v = join_all(part, nw, f);
      if (cs > 1) {
        const int set = turn & 1;
        if (!met) cluster_wait();  // every CTA of the cluster runs, its mbarriers set
        met = true;
        if (tid < 32) {
          if (tid < cs) put_peer(&peers[set][rank], &bar[set], tid, v);
          const bool came = __all_sync(0xffffffffu, mbar_wait_cluster(&bar[set], (turn >> 1) & 1, status));
          if (tid == 0) {
            lost = !came;
            if (came) {
              mbar_arrive_expect_tx(&bar[set], cs * sizeof(MaxSum));  // for the turn after next
              all = join_all(peers[set], cs, f);
            }
          }
        }
        __syncthreads();
        if (lost) break;
        v = all;
        ++turn;
      }
      const bool is_near = fabsf(v.m) * f <= kNearLogit * kLog2e;
      if (!is_near) {  // in every CTA of the cluster
        if (first_cta) slow_row<T>(a, r, p.j, l, t);
        if (GRAD)
          for (int i = tid; i < next.n; i += nt) ask(next, i);
      } else {
        // Logarithms to base 2 against c: of the list's maximum, of the sum over all classes, of the remainder's share.
        const float c = ref(v.m, f), to_list = fmaf(t.m, f, -c), top = fmaxf(0.f, to_list);
        const float ls = top + log2f(s_l * exp2_fast(to_list - top) + v.s * exp2_fast(-top)), log_r = log2f(v.s) - ls;
        const float q_r = a.teacher_lse && !whole ? fmaxf(0.f, 1.f - t.sum) : 0.f;
        if (tid == 0 && first_cta)
          put_loss(a, r, p.j.w * (list_loss(t, kLn2 * (ls - to_list)) + term(q_r, logf(q_r), kLn2 * log_r)),
                   kLn2 * (c + ls));
        if (GRAD) {
          const RowVecs<T> out(g, a.V);
          const float wt = p.j.w * inv_h, to = wt * (exp2_fast(log_r) - q_r) / v.s;
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
            __syncthreads();
            const T* const from = reinterpret_cast<const T*>(slice);
            for (int i = tid; i < p.n * N; i += nt) g[col0 + i] = from[i];
            __syncthreads();
            for (int i = tid; i < next.n; i += nt) ask(next, i);
          }
          __syncthreads();  // the row's other elements, which the listed ones go over; the list has been read
          const int inner = p.row.head + (p.row.f1 - p.row.f0) * N;
#pragma unroll
          for (int u = 0; u < kEach; ++u) {
            const int cu = own[u].c;
            const bool edge = cu < p.row.head || cu >= inner;
            if (first[u] && (edge ? first_cta : static_cast<unsigned>(cu - col0) < static_cast<unsigned>(p.n * N)))
              g[cu] = from_f32<T>(wt * (exp2_fast(fmaf(own[u].x, f, -c) - ls) - q_all[u]));
          }
        }
      }
      if (!GRAD || !is_near) __syncthreads();  // `part` and the list have been read
      p = next;
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u) own[u] = nxt[u];
    ce = edge_of(p);
    xe = ce >= 0 ? to_f32(p.x[ce]) : 0.f;
  }
  if (!met) cluster_wait();
  if (cs > 1 && met && lost) {
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
  // Rows of up to 103 KB stay in one CTA, two of which share a multiprocessor beside their lists; longer ones are
  // cut into slices of up to that: every CTA of a cluster works through the whole list (4 x 2048 rows of 100,096 with
  // 128 entries: 0.79 ms in slices of 48 KB, 0.54 ms so). Few rows: spread over the multiprocessors.
  const long long bytes = nv * 16ll;
  int cs = 1;
  while (cs < kMaxCluster && bytes > 103 * 1024ll * cs) cs *= 2;
  while (cs < kMaxCluster && static_cast<long long>(M) * cs * 2 <= num_sms && nv / cs >= 512) cs *= 2;
  const int per = (nv + cs - 1) / cs;
  const bool grad = a.dlogits.p != nullptr;
  const long long smem = sizeof(List) + per * 16ll;
  if (smem > 220 * 1024 || static_cast<long long>(M) * cs > 0x7FFFFFFFLL) {
    k_distill_rows<T><<<M, kRowThreads, 0, st>>>(a, status);
    return cudaGetLastError();
  }
  const int each = static_cast<long long>(M) * cs < 2 * num_sms ? 12 : 14;
  const int threads = std::min(kSliceThreads, std::max(kListMax / kEach, (per / each + 31) / 32 * 32));
  const int rows = loss_rows(M, cs, threads, num_sms);
  auto k = grad ? k_distill<T, true> : k_distill<T, false>;
  if (cudaError_t e = allow_smem(k, smem); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>((M + rows - 1) / rows) * cs);
  cfg.blockDim = dim3(threads);
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
