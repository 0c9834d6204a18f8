// Scores of tokens under rows of logits (kf_op_token_scores) and their
// gradient (kf_op_token_scores_grad).
//
// With x = logits / tau and a reference m near max x, one pass over a row gives
//   S = sum exp(x - m),  T = sum (x - m) exp(x - m),
//   lse = m + log S,     entropy = log S - T / S
// (against a near reference no term cancels against a much larger one).
// A thread keeps (m, S, T) of the 16-byte vectors it reads; they move to another
// reference as S' = f S, T' = f (T + d S) with d = m - m' and f = exp(d).  All of it is
// fp32, in base-2 units: 2^d with d = x log2(e) - m log2(e).
//
// What bounds it: the logits' bytes, read once (scores) or read and written once
// (gradient), and close behind them the instructions: 8.3 an element without alternatives, 11.6 with
// eight, ten a pass of the gradient, most of the arithmetic on pairs (fma.rn.f32x2).  CTAs walk over the rows, and each thread streams its
// vectors through slots of shared memory that are its own (cp.async, batches of four; no thread
// waits for another's), the next row's while this one is reduced.
//   Scores: a ring of three batches a thread, four CTAs of 256 threads a SM (many rows that are
//   not wide: sixteen of 64 with two batches).
//   Gradient: the row stays in the slots for the second pass, two CTAs of 512 threads a SM (a
//   second pass from L2 found only half of the lines there: 369 MB read instead of 206 at
//   2048 x 50257); a row wider than that is split over a cluster.
//
// Top alternatives: the threads of a row form 64 groups, and the
// n-th largest of the 64 groups' maxima is at or below the n-th largest logit (n
// groups have an element at or above it).  So only the vectors of threads whose own
// maximum reaches that bound are looked at again (from L2, a warp per such thread), and their
// elements at or above it listed, a few dozen of a vocabulary; each one's rank among
// them is its place.  Where masks close too many groups, the threads' own maxima give the
// bound; rows where the list would not fit all the same (ties in the hundreds) raise the bound.
//
// Measured: 4096 bf16 rows of 50257 in 96 us with eight alternatives (4.3 TB/s), 72 without (5.7); 8 fp32
// rows 7.5; the gradient of 2048 bf16 rows 86 us (4.8 TB/s).
#include <algorithm>
#include <cooperative_groups.h>

#include "kf_mma.cuh"
#include "kf_serving.cuh"
#include "kf_tc.cuh"

namespace cg = cooperative_groups;

namespace kf {
namespace {

constexpr int kBatch = 4;          // vectors of a batch
// scores: batches under way or in use (two for CTAs of two warps, so that sixteen of them fit an SM)
template <int THREADS> constexpr int kRing = THREADS == 64 ? 2 : 3;
constexpr int kResident = 4;       // gradient: batches of a row, at most
constexpr int kPairBytes = 13 * 512 * 16;    // gradient: slots of a CTA that leave room for a second one on the SM
constexpr int kGroups = 64;        // groups whose maxima bound the n-th largest logit
constexpr int kMaxTop = kGroups;
// Alternatives that the groups' maxima bound well; for more, CTAs of over 64 threads take their
// threads' own (4096 bf16 rows, groups and threads, us: 56 of 18000  116  144, 64 of them 260  152;
// 56 of 50257  190  191, 64 of them 380  198)
constexpr int kFew = 56;
template <int THREADS> constexpr int kList = THREADS == 64 ? 512 : 768;      // listed candidates of a row
constexpr int kMostRow = 8 * kResident * kBatch * 512 * 16;      // bytes of a row: the gradient's slots in eight CTAs
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -300.f;   // 2^-300 is 0 in fp32: stands for -inf where it multiplies that 0
constexpr float kRaise = 20.f;
constexpr float kLarge = 16777216.f;      // 2^24: from there on the rounding of a reference in base-2 units passes 1

struct Args {
  const void* logits;
  int64_t stride;
  const int64_t* tokens;
  const float *g_logp, *g_entropy;
  float *logp, *entropy, *lse, *top_logp;
  int32_t* top_ids;
  void* grad;
  int64_t grad_stride, R;
  int V, top;
  float inv_tau, c2, margin;       // 1 / tau, log2(e) / tau, kRaise / c2
  int* err;
};

// 2^x on the special-function unit: relative error about 2^-22
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What scores are taken against: a logit `raw` that no element exceeds by more than
// 2^kRaise.  (The maximum itself changes for some lane of a warp at almost every
// vector; the entropy's cancellation, 2^-24 of kRaise, stays below 2e-6.)  In base-2 units one fused
// multiply-add gives an element's difference, and what the reference lost in rounding is a factor of S and T alike that
// cancels; past kLarge (rows at a mask's value, a small tau) that factor would leave fp32's range,
// so there the logits' difference is formed first and scaled after
struct Ref {
  float raw, nm;                   // nm: minus the reference, base-2 units (a logit where big)
  float limit;                     // a logit past this raises the reference
  bool big;
  static __device__ __forceinline__ bool large(const Args& a, float r) {
    const float m = fabsf(r * a.inv_tau);
    return m >= kLarge && m < INFINITY;
  }
  __device__ __forceinline__ void set(const Args& a, float r) {
    const float m = r * a.inv_tau;
    raw = r;
    limit = r == -INFINITY ? r : r + a.margin;
    big = large(a, r);
    nm = m == -INFINITY ? 0.f : big ? -r : -__fmul_rn(r, a.c2);
  }
  __device__ __forceinline__ bool open(const Args& a) const { return raw * a.inv_tau != -INFINITY; }
  // log2 of exp(x - m)
  __device__ __forceinline__ float less(const Args& a, float v) const {
    return big ? (v + nm) * a.c2 : fmaf(v, a.c2, nm);
  }
  // log2 of exp(m' - m) for an open reference m' of the logit `from`, both as they were rounded
  __device__ __forceinline__ float less_ref(const Args& a, float from) const {
    if (large(a, from)) return less(a, from);
    const float was = __fmul_rn(from, a.c2);
    return big ? fmaf(nm, a.c2, was) : __fadd_rn(was, nm);      // (no fused multiply-add)
  }
};

// S and T (base-2 units) of some elements against the reference `raw`; without an open element
// they are 0 (or NaN)
struct Sums {
  float raw, s, t;
  // against the reference r (at or above this one)
  __device__ __forceinline__ void move_to(const Args& a, const Ref& r) {
    const float d = raw * a.inv_tau == -INFINITY ? 0.f : fmaxf(r.less_ref(a, raw), kLeast), f = ex2(d);
    t = f * fmaf(d, s, t);
    s *= f;
    raw = r.raw;
  }
};

// one thread's pass over its elements
struct Pass {
  Ref r;
  float most = -INFINITY;          // the largest logit
  uint64_t s = 0ull, t = 0ull;     // S and T, in two lanes each
  __device__ __forceinline__ Pass() : r{-INFINITY, 0.f, -INFINITY, false} {}
  __device__ __forceinline__ void raise(const Args& a, float to) {
    const Ref was = r;
    r.set(a, to);
    if (was.open(a)) {
      const float d = fmaxf(r.less_ref(a, was.raw), kLeast), f = ex2(d);
      t = mul_f2(f2(f, f), fma_f2(f2(d, d), s, t));
      s = mul_f2(f2(f, f), s);
    }
  }
  __device__ __forceinline__ void pair(float2 d) {
    const uint64_t e = f2(ex2(d.x), ex2(d.y));
    s = add_f2(s, e);
    t = fma_f2(e, f2(fmaxf(d.x, kLeast), fmaxf(d.y, kLeast)), t);
  }
  template <int N>
  __device__ __forceinline__ void add(const Args& a, const float* v) {
    float top = fmaxf(v[0], v[1]);
#pragma unroll
    for (int i = 2; i < N; i += 2) top = max3f(top, v[i], v[i + 1]);
    most = fmaxf(most, top);
    if (top > r.limit) raise(a, top);
    const uint64_t c = f2(a.c2, a.c2), nm = f2(r.nm, r.nm);
    if (!r.big) {
#pragma unroll
      for (int i = 0; i < N; i += 2) pair(f2_split(fma_f2(f2(v[i], v[i + 1]), c, nm)));
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2) pair(f2_split(mul_f2(add_f2(f2(v[i], v[i + 1]), nm), c)));
    }
  }
  __device__ __forceinline__ void add_one(const Args& a, float v) {
    most = fmaxf(most, v);
    if (v > r.limit) raise(a, v);
    pair(make_float2(r.less(a, v), -INFINITY));
  }
  __device__ __forceinline__ Sums sums() const {
    const float2 x = f2_split(s), y = f2_split(t);
    return Sums{r.raw, x.x + x.y, y.x + y.y};
  }
};

// A row's elements in 16-byte vectors: `head` elements lie before the first
// aligned one, then nvec vectors, then the rest.
template <typename T>
struct Row {
  const T* p;
  int head, nvec, V;
  __device__ __forceinline__ Row(const T* q, int V_) : p(q), V(V_) {
    head = min((int)((16 - (reinterpret_cast<uintptr_t>(q) & 15)) & 15) / (int)sizeof(T), V);
    nvec = (V - head) / Vec16<T>::N;
  }
  __device__ __forceinline__ const T* vec(int i) const { return p + head + (size_t)i * Vec16<T>::N; }
  __device__ __forceinline__ int edge() const { return V - nvec * Vec16<T>::N; }        // elements outside the vectors
  __device__ __forceinline__ int edge_id(int j) const { return j < head ? j : j + nvec * Vec16<T>::N; }
};

struct Cand {
  float x;
  int id;
};
__device__ __forceinline__ bool before(Cand a, Cand b) { return a.x > b.x || (a.x == b.x && a.id < b.id); }

template <int THREADS>
struct Shared {
  float ref[THREADS / 32], cta_ref;
  float2 warp[THREADS / 32], cta;
  float group[kGroups];
  float bound;
  int count, again;
  uint16_t thread[THREADS];        // threads whose vectors are looked at again
  int tied[THREADS / 32];
  Cand list[kList<THREADS>];
};

// A row's numbers, the same in all of its threads
struct Scores {
  Ref ref;
  float logs, lse, H;              // log2 S; H: the entropy
  bool none, bad;                  // every token closed; a NaN or +inf in the row
  // log p of a logit: from the difference to the reference, not from lse, which loses log S where the
  // reference is large (the last form where a difference leaves fp32's range before it is scaled)
  __device__ __forceinline__ float lp(const Args& a, float v) const {
    const float d = ref.big ? v + ref.nm : ref.less(a, v);
    if (fabsf(d) < INFINITY) return ref.big ? d * a.inv_tau - logs * kLn2 : (d - logs) * kLn2;
    return (v * a.inv_tau - ref.raw * a.inv_tau) - logs * kLn2;
  }
};
// The row's sums against its largest reference, added in one fixed order; with `groups` the
// groups' maxima in sh.group (of every CTA)
template <int THREADS, int CS, bool GROUPS>
__device__ __forceinline__ Scores reduce_row(const Args& a, Shared<THREADS>& sh, const Pass& ps) {
  constexpr int WARPS = THREADS / 32, LANES = THREADS * CS / kGroups;      // LANES: threads of a group
  static_assert(!GROUPS || (LANES >= 1 && LANES <= 32), "a group lies in a warp");
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  Sums su = ps.sums();
  Scores o;
  float m = su.raw;
#pragma unroll
  for (int i = 16; i; i >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, i));
  if (lane == 0) sh.ref[warp] = m;
  if constexpr (GROUPS) {
    float gm = ps.most;
#pragma unroll
    for (int i = 1; i < LANES; i <<= 1) gm = fmaxf(gm, __shfl_xor_sync(~0u, gm, i));
    if (t % LANES == 0) sh.group[t / LANES] = gm;
  }
  __syncthreads();                        // (all threads are done with the row before)
  if (t == 0) sh.count = sh.again = 0;
  m = sh.ref[lane % WARPS];
#pragma unroll
  for (int i = WARPS / 2; i; i >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, i));
  if constexpr (CS > 1) {
    cg::cluster_group cl = cg::this_cluster();
    if (t == 0) sh.cta_ref = m;
    cl.sync();
    for (int c = 0; c < CS; ++c) m = fmaxf(m, cl.map_shared_rank(&sh, c)->cta_ref);
  }
  o.ref.set(a, m);
  su.move_to(a, o.ref);
#pragma unroll
  for (int i = 16; i; i >>= 1) {
    su.s += __shfl_xor_sync(~0u, su.s, i);
    su.t += __shfl_xor_sync(~0u, su.t, i);
  }
  if (lane == 0) sh.warp[warp] = make_float2(su.s, su.t);
  __syncthreads();
  float2 x = sh.warp[lane % WARPS];
#pragma unroll
  for (int i = WARPS / 2; i; i >>= 1) {
    x.x += __shfl_xor_sync(~0u, x.x, i);
    x.y += __shfl_xor_sync(~0u, x.y, i);
  }
  if constexpr (CS > 1) {
    cg::cluster_group cl = cg::this_cluster();
    if (t == 0) sh.cta = x;
    cl.sync();
    x = make_float2(0.f, 0.f);
    for (int c = 0; c < CS; ++c) {
      const float2 y = cl.map_shared_rank(&sh, c)->cta;
      x.x += y.x;
      x.y += y.y;
    }
    float g = 0.f;
    const bool take = GROUPS && t < kGroups;
    if (take) g = cl.map_shared_rank(&sh, t / (kGroups / CS))->group[t % (kGroups / CS)];
    cl.sync();                            // the other CTAs have read this one's part
    if (take) sh.group[t] = g;
    __syncthreads();
  }
  o.none = !o.ref.open(a) && x.x == 0.f;
  o.bad = !(x.x > 0.f) && !o.none;
  o.logs = log2f(x.x);
  o.lse = o.none ? -INFINITY : o.bad ? NAN : o.ref.raw * a.inv_tau + o.logs * kLn2;
  o.H = o.none ? 0.f : o.bad ? NAN : (o.logs - x.y / x.x) * kLn2;
  return o;
}
__device__ __forceinline__ void write_numbers(const Args& a, int64_t r, const Scores& o, int64_t token, float at_logit) {
  if (a.lse) a.lse[r] = o.lse;
  if (a.entropy) a.entropy[r] = o.H;
  if (token >= a.V) atomicOr(a.err, KF_DEV_BAD_TOKEN);
  if (a.logp) a.logp[r] = token < 0 ? 0.f : token >= a.V || o.bad ? NAN : o.none ? -INFINITY : o.lp(a, at_logit);
}
// what a row's threads hold beside their vectors: elements outside of them (fewer than 16), the
// token and its logit (read before the barriers: the gradient may overwrite the logits)
template <typename T>
struct Extra {
  int64_t token;
  float at_logit, edge_logit;
  int edge_id;
  bool edge;
  __device__ __forceinline__ Extra(const Args& a, const Row<T>& row, int64_t r, bool first_cta) {
    const int t = threadIdx.x;
    token = a.tokens[r];
    at_logit = t == 0 && token >= 0 && token < a.V ? to_f(row.p[token]) : 0.f;
    edge = first_cta && t < row.edge();
    edge_id = edge ? row.edge_id(t) : 0;
    edge_logit = edge ? to_f(row.p[edge_id]) : -INFINITY;
  }
};
template <typename T>
__device__ __forceinline__ Row<T> row_at(const Args& a, int64_t r) {
  return Row<T>(static_cast<const T*>(a.logits) + r * a.stride, a.V);
}
// The row's CTAs take consecutive stretches of per_cta * THREADS vectors: vector k of a thread is
// first + k * THREADS, if it has k < have(row)
template <int THREADS>
struct Mine {
  int per_cta, first;
  __device__ __forceinline__ Mine(int vectors, int cs, int rank) {
    per_cta = (vectors + cs * THREADS - 1) / (cs * THREADS);
    first = rank * per_cta * THREADS + threadIdx.x;
  }
  template <typename T> __device__ __forceinline__ int have(const Row<T>& w) const {
    return min(per_cta, (w.nvec - first + THREADS - 1) / THREADS);
  }
};

// ------------------------------------------------------------------ scores
// More candidates than the list holds (ties at the bound, as of a mask of the type's lowest value): those
// above the bound, then above the top-th largest of the listed, until they fit (each pass after the
// first drops all but top of the listed at least); ones at that bound follow by id.  Returns
// how many are listed.  A call, so that the kernel's registers stay its own (inline: 106 us for 99 at
// 4096 x 50257); 8 rows of 50257 with five open ones take 21 us
template <typename T, int THREADS>
__device__ __noinline__ int raise_bound(Shared<THREADS>& sh, const T* p, int V, int top, float inv_tau, float bound) {
  constexpr int N = Vec16<T>::N, WARPS = THREADS / 32;
  const Row<T> row(p, V);
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  int found = kList<THREADS> + 1;
#pragma unroll 1
  for (bool first = true; found > kList<THREADS>; first = false) {      // (uniform)
    if (!first) {
      for (int i = t; i < kList<THREADS>; i += THREADS) {
        const Cand c = sh.list[i];
        int rk = 0;
        for (int j = 0; j < kList<THREADS>; ++j) rk += before(sh.list[j], c);
        if (rk == top - 1) sh.bound = c.x;
      }
      __syncthreads();
      bound = sh.bound;
    }
    __syncthreads();
    if (t == 0) sh.count = 0;
    __syncthreads();
    auto above = [&](int id, float v) {
      const float x = v * inv_tau;
      if (x > bound) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < kList<THREADS>) sh.list[at] = Cand{x, id};
      }
    };
    if (t < row.edge()) above(row.edge_id(t), to_f(p[row.edge_id(t)]));
    for (int i = t; i < row.nvec; i += THREADS) {
      float v[N];
      Vec16<T>::unpack(*reinterpret_cast<const uint4*>(row.vec(i)), v);
#pragma unroll
      for (int e = 0; e < N; ++e) above(row.head + i * N + e, v[e]);
    }
    __syncthreads();
    found = sh.count;
  }
  if (found >= top) return found;
  for (int id0 = 0; found < top && id0 < V; id0 += THREADS) {            // (uniform)
    const int id = id0 + t;
    const bool tie = id < V && to_f(p[id]) * inv_tau == bound;
    const uint32_t same = __ballot_sync(~0u, tie);
    if (lane == 0) sh.tied[warp] = __popc(same);
    __syncthreads();
    int at = found + __popc(same & ((1u << lane) - 1));
    for (int w = 0; w < WARPS; ++w) {
      found += sh.tied[w];
      at += w < warp ? sh.tied[w] : 0;
    }
    if (tie && at < top) sh.list[at] = Cand{bound, id};
    __syncthreads();
  }
  return min(found, top);
}

template <typename T, int THREADS, int CS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_scores(const Args a) {
  extern __shared__ __align__(16) uint4 slots[];         // [batch of the ring][vector][thread]
  __shared__ Shared<THREADS> sh;
  constexpr int N = Vec16<T>::N, WARPS = THREADS / 32;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, rank = blockIdx.x % CS;
  const Mine<THREADS> mine(a.V / N, CS, rank);
  const int batches = (mine.per_cta + kBatch - 1) / kBatch;      // of a row
  const int step = gridDim.x / CS, R = (int)a.R;         // (up to 2^28 rows)
  const uint32_t slot0 = mma::smem_addr(slots + t);

  // the copies run kRing<THREADS> - 1 batches ahead, into the rows that follow
  int fr = blockIdx.x / CS, fb = 0, fslot = 0, fn = 0;
  const T* fp = nullptr;
  auto look = [&] {
    if (fr >= R) return;
    const Row<T> w = row_at<T>(a, fr);
    fn = mine.have(w);
    fp = w.vec(mine.first);
  };
  auto fill = [&] {                       // one group of copies, empty past the last row
    if (fr < R) {
      const T* p = fp + (size_t)fb * kBatch * THREADS * N;
      const uint32_t d = slot0 + fslot * kBatch * THREADS * 16;
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (fb * kBatch + j < fn) mma::cp_async16(d + j * THREADS * 16, p + j * THREADS * N, 16);
      if (++fb == batches) {
        fb = 0;
        fr += step;
        look();
      }
      fslot = fslot + 1 == kRing<THREADS> ? 0 : fslot + 1;
    }
    mma::cp_commit();
  };
  look();
#pragma unroll
  for (int i = 0; i < kRing<THREADS> - 1; ++i) fill();
  int slot = 0;
#pragma unroll 1
  for (int r = blockIdx.x / CS; r < R; r += step) {
    const Row<T> row = row_at<T>(a, r);
    const Extra<T> ex(a, row, r, rank == 0);
    const int n = mine.have(row);
    Pass ps;
#pragma unroll 1
    for (int b = 0; b < batches; ++b) {
      mma::cp_wait<kRing<THREADS> - 2>();          // this batch has landed
      fill();                             // into the slots of the batch before
      const uint4* s = slots + slot * kBatch * THREADS + t;
      if ((b + 1) * kBatch <= n) {
        float v[kBatch * N];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) Vec16<T>::unpack(s[j * THREADS], v + j * N);
        ps.add<kBatch * N>(a, v);
      } else {
        for (int j = 0; b * kBatch + j < n; ++j) {
          float v[N];
          Vec16<T>::unpack(s[j * THREADS], v);
          ps.add<N>(a, v);
        }
      }
      slot = slot + 1 == kRing<THREADS> ? 0 : slot + 1;
    }
    const float vec_max = ps.most;
    if (ex.edge) ps.add_one(a, ex.edge_logit);
    const Scores o = reduce_row<THREADS, CS, true>(a, sh, ps);
    if (rank == 0 && t == 0) write_numbers(a, r, o, ex.token, ex.at_logit);

    if (a.top == 0) continue;             // (uniform)
    int32_t* ids = a.top_ids + (int64_t)r * a.top;
    float* lps = a.top_logp + (int64_t)r * a.top;
    if (o.bad) {                          // (uniform over the row's CTAs)
      if (rank == 0)
        for (int i = t; i < a.top; i += THREADS) {
          ids[i] = -1;
          lps[i] = NAN;
        }
      continue;
    }
    // the bound: the top-th largest of the groups' maxima
    if (t < kGroups) {
      const float g = sh.group[t];
      int rk = 0;
#pragma unroll 16
      for (int j = 0; j < kGroups; ++j) rk += sh.group[j] > g || (sh.group[j] == g && j < t);
      if (rk == a.top - 1) sh.bound = g * a.inv_tau;
    }
    __syncthreads();
    float bound = sh.bound;
    // (uniform over the row's CTAs) masks, or many alternatives: this CTA's threads' own maxima
    if (bound == -INFINITY || (CS == 1 && THREADS > kGroups && a.top > kFew)) {
      float* own = reinterpret_cast<float*>(sh.list);
      own[t] = vec_max;
      __syncthreads();
      int rk = 0;
      for (int j = 0; j < THREADS; ++j) rk += own[j] > vec_max || (own[j] == vec_max && j < t);
      if (rk == min(a.top, THREADS) - 1) sh.bound = a.top <= THREADS ? vec_max * a.inv_tau : -INFINITY;
      __syncthreads();
      bound = sh.bound;
      if constexpr (CS > 1) {
        // the best of the CTAs' bounds: top elements of that one are at or above it
        cg::cluster_group cl = cg::this_cluster();
        cl.sync();
        for (int c = 0; c < CS; ++c) bound = fmaxf(bound, cl.map_shared_rank(&sh, c)->bound);
        cl.sync();
      }
    }
    Shared<THREADS>* lead = &sh;
    if constexpr (CS > 1) lead = cg::this_cluster().map_shared_rank(&sh, 0);
    // (a bound of -inf: the open tokens are listed, the closed ones follow by id)
    auto listed = [&](float x) { return x >= bound && x > -INFINITY; };
    auto list = [&](int id, float v) {
      const float x = v * a.inv_tau;
      if (listed(x)) {
        const int at = atomicAdd(&lead->count, 1);
        if (at < kList<THREADS>) lead->list[at] = Cand{x, id};
      }
    };
    if (listed(vec_max * a.inv_tau)) sh.thread[atomicAdd(&sh.again, 1)] = (uint16_t)t;
    if (ex.edge) list(ex.edge_id, ex.edge_logit);
    __syncthreads();
    auto list_vector = [&](int i) {
      float v[N];
      Vec16<T>::unpack(*reinterpret_cast<const uint4*>(row.vec(i)), v);
      const int id0 = row.head + i * N;
#pragma unroll
      for (int e = 0; e < N; ++e) list(id0 + e, v[e]);
    };
    // a warp per such thread, or each by itself, whichever has fewer vectors in turn
    if (sh.again * ((mine.per_cta + 31) / 32) <= WARPS * mine.per_cta) {
      for (int j = warp; j < sh.again; j += WARPS)
        for (int k = lane; k < mine.per_cta; k += 32) {
          const int i = mine.first - t + sh.thread[j] + k * THREADS;
          if (i >= row.nvec) break;
          list_vector(i);
        }
    } else if (listed(vec_max * a.inv_tau)) {
#pragma unroll 4
      for (int k = 0; k < n; ++k) list_vector(mine.first + k * THREADS);
    }
    if constexpr (CS > 1) cg::this_cluster().sync();
    else __syncthreads();
    if (rank != 0) continue;
    int found = sh.count;
    if (found > kList<THREADS>) found = raise_bound(sh, row.p, a.V, a.top, a.inv_tau, bound);      // (uniform)
    auto put = [&](int place, Cand c) {
      ids[place] = c.id;
      lps[place] = o.lp(a, to_f(row.p[c.id]));
    };
    for (int i = t; i < found; i += THREADS) {
      const Cand c = sh.list[i];
      int rk = 0;
      for (int j = 0; j < found; ++j) rk += before(sh.list[j], c);
      if (rk < a.top) put(rk, c);
    }
    // fewer open tokens than asked for: closed ones by id
    if (found < a.top && t == 0) {
      int k = found;
      for (int id = 0; k < a.top && id < a.V; ++id) {
        if (to_f(row.p[id]) * a.inv_tau > -INFINITY) continue;
        ids[k] = id;
        lps[k++] = -INFINITY;
      }
    }
  }
  mma::cp_wait<0>();
}

// ---------------------------------------------------------------- gradient
static_assert(2 * (kPairBytes + sizeof(Shared<512>) + 1024) <= 233472, "two CTAs on an SM");
template <typename T, int THREADS, int CS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_scores_grad(const Args a) {
  extern __shared__ __align__(16) uint4 slots[];         // [vector][thread]
  __shared__ Shared<THREADS> sh;
  constexpr int N = Vec16<T>::N;
  const int t = threadIdx.x, rank = blockIdx.x % CS;
  const Mine<THREADS> mine(a.V / N, CS, rank);
  const int64_t step = gridDim.x / CS;
  const uint32_t slot0 = mma::smem_addr(slots + t);
  auto fill = [&](const Row<T>& w, int n, int g) {       // batch g of a row: one group of copies, always
    const T* p = w.vec(mine.first);
#pragma unroll
    for (int j = g * kBatch; j < (g + 1) * kBatch; ++j)
      if (j < n) mma::cp_async16(slot0 + j * THREADS * 16, p + (size_t)j * THREADS * N, 16);
    mma::cp_commit();
  };
  {
    const Row<T> w = row_at<T>(a, blockIdx.x / CS);
#pragma unroll
    for (int g = 0; g < kResident; ++g) fill(w, mine.have(w), g);
  }
#pragma unroll 1
  for (int64_t r = blockIdx.x / CS; r < a.R; r += step) {
    const Row<T> row = row_at<T>(a, r);
    const bool more = r + step < a.R;
    const Row<T> next = row_at<T>(a, more ? r + step : r);
    const Extra<T> ex(a, row, r, rank == 0);
    const int n = mine.have(row), n_next = mine.have(next);
    Pass ps;
#pragma unroll
    for (int g = 0; g < kResident; ++g) {
      // this batch's copies are done, later ones may not be
      if (g == 0) mma::cp_wait<kResident - 1>();
      else if (g == 1) mma::cp_wait<kResident - 2>();
      else if (g == 2) mma::cp_wait<kResident - 3>();
      else mma::cp_wait<0>();
      const uint4* s = slots + g * kBatch * THREADS + t;
      if ((g + 1) * kBatch <= n) {
        float v[kBatch * N];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) Vec16<T>::unpack(s[j * THREADS], v + j * N);
        ps.add<kBatch * N>(a, v);
      } else {
        for (int j = 0; g * kBatch + j < n; ++j) {
          float v[N];
          Vec16<T>::unpack(s[j * THREADS], v);
          ps.add<N>(a, v);
        }
      }
    }
    if (ex.edge) ps.add_one(a, ex.edge_logit);
    const Scores o = reduce_row<THREADS, CS, false>(a, sh, ps);
    if (rank == 0 && t == 0) write_numbers(a, r, o, ex.token, ex.at_logit);

    const bool has = ex.token >= 0 && ex.token < a.V;
    const float gl = has && a.g_logp ? a.g_logp[r] : 0.f, gh = a.g_entropy ? a.g_entropy[r] : 0.f;
    // grad = p (A + B log2 p) + (v == token) gl / tau.  A row with a NaN has A = NaN; one
    // without open tokens p = 0
    const float A = (-gl - gh * o.H) * a.inv_tau, B = -gh * a.inv_tau * kLn2;
    const float at_token = o.none ? 0.f : gl * a.inv_tau;
    T* out = static_cast<T*>(a.grad) + r * a.grad_stride;
    const uint64_t c2 = f2(a.c2, a.c2), nm = f2(o.ref.nm, o.ref.nm), nlogs = f2(-o.logs, -o.logs), A2 = f2(A, A), B2 = f2(B, B);
    auto pair = [&](float& x, float& y) {
      float2 d;
      if (!o.ref.big) d = f2_split(add_f2(fma_f2(f2(x, y), c2, nm), nlogs));      // (one constant for both would lose log S)
      else d = f2_split(add_f2(mul_f2(add_f2(f2(x, y), nm), c2), nlogs));
      d.x = fmaxf(d.x, kLeast);
      d.y = fmaxf(d.y, kLeast);
      const float2 g = f2_split(mul_f2(f2(ex2(d.x), ex2(d.y)), fma_f2(B2, f2(d.x, d.y), A2)));
      x = g.x;
      y = g.y;
    };
    const bool same = (reinterpret_cast<uintptr_t>(out) & 15) == (reinterpret_cast<uintptr_t>(row.p) & 15);
    if (ex.edge) {
      float x = ex.edge_logit, y = -INFINITY;
      pair(x, y);
      out[ex.edge_id] = from_f<T>(ex.edge_id == ex.token ? x + at_token : x);
    }
#pragma unroll
    for (int g = 0; g < kResident; ++g) {
#pragma unroll
      for (int j = g * kBatch; j < (g + 1) * kBatch; ++j) {
        if (j >= n) break;
        float v[N];
        Vec16<T>::unpack(slots[j * THREADS + t], v);
        const int id0 = row.head + (mine.first + j * THREADS) * N;
#pragma unroll
        for (int e = 0; e < N; e += 2) pair(v[e], v[e + 1]);
        if (ex.token >= id0 && ex.token < id0 + N) {
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (id0 + e == ex.token) v[e] += at_token;
        }
        if (same) {
          *reinterpret_cast<uint4*>(out + id0) = Vec16<T>::pack(v);
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) out[id0 + e] = from_f<T>(v[e]);
        }
      }
      if (more) fill(next, n_next, g);
    }
  }
}

// ------------------------------------------------------------------ host
// a grid of as many clusters as fit the SMs at once, for the rows that there are
template <int THREADS, int CS, typename K>
void launch_rows(K* kernel, PerDevice& attr, const Args& a, size_t bytes, cudaStream_t s) {
  set_smem_attr(attr, kernel, bytes);
  const int64_t per_sm = std::max<int64_t>(1, std::min<int64_t>(1024 / THREADS, 233472 / (bytes + sizeof(Shared<THREADS>) + 1024)));
  const int64_t rows = std::min<int64_t>(a.R, std::max<int64_t>(1, per_sm * device_sms() / CS));
  launch_cluster(kernel, dim3((unsigned)(rows * CS)), dim3(THREADS), bytes, CS, false, s, a);
}
template <typename T, int THREADS, int CS>
void launch_scores(const Args& a, cudaStream_t s) {
  static PerDevice attr;
  launch_rows<THREADS, CS>(k_scores<T, THREADS, CS>, attr, a, (size_t)kRing<THREADS> * kBatch * THREADS * 16, s);
}
template <typename T, int THREADS, int CS>
void launch_grad(const Args& a, cudaStream_t s) {
  static PerDevice attr;
  const int k = (a.V / Vec16<T>::N + CS * THREADS - 1) / (CS * THREADS);
  launch_rows<THREADS, CS>(k_scores_grad<T, THREADS, CS>, attr, a, (size_t)k * THREADS * 16, s);
}
template <typename T, bool GRAD>
int launch(const Args& a, cudaStream_t s) {
  // Many rows that are not wide take CTAs of two warps, sixteen a SM (the gradient's ten): less of
  // a row's time goes to its joins (up to kFew alternatives, see there).  Measured on bf16 with two warps against wide CTAs, us:
  //   scores, five alternatives   6000 of 304 rows  7.2  5.3, of 608  7.8  7.2, of 4096  23.2  37.7;
  //                               18000 of 4096  43.6  52.9, 30000  67.2  67.0, 50257  113  92
  //   without alternatives        50257 of 608  14.4  13.5, of 4096  71.5  76.0
  //   gradient                    6000 of 304  7.2  5.5, of 608  7.4  9.4, of 4096  29.7  54.1
  // Few rows are split over a cluster while half the SMs would idle and each thread keeps two
  // vectors (50257, one CTA a row against the cluster: 8 rows 8.1  7.0, 32 rows 8.0  7.6, 64 rows 8.2
  // 8.8, 128 rows 8.2  9.6; the gradient 8.4  6.1, 8.6  6.5, 8.5  8.1, 8.7  11.1); the gradient's
  // also until they fit the slots
  const int64_t bytes = (int64_t)a.V * sizeof(T), sms = device_sms();
  int cs = 1;
  if constexpr (GRAD) {
    while (cs < 8 && (bytes > (int64_t)cs * kPairBytes || (a.R * cs * 2 <= sms && bytes >= cs * 2 * 2 * 512 * 16))) cs *= 2;
    if (bytes <= 12288 && a.R > 2 * sms) launch_grad<T, 64, 1>(a, s);
    else if (cs == 1) launch_grad<T, 512, 1>(a, s);
    else if (cs == 2) launch_grad<T, 512, 2>(a, s);
    else if (cs == 4) launch_grad<T, 512, 4>(a, s);
    else launch_grad<T, 512, 8>(a, s);
  } else {
    while (cs < 8 && a.R * cs * 2 <= sms && bytes >= cs * 2 * 2 * 256 * 16) cs *= 2;
    if (a.R > 4 * sms && a.top <= kFew && bytes <= (a.top ? 49152 : 114688)) launch_scores<T, 64, 1>(a, s);
    else if (cs == 1) launch_scores<T, 256, 1>(a, s);
    else if (cs == 2) launch_scores<T, 256, 2>(a, s);
    else if (cs == 4) launch_scores<T, 256, 4>(a, s);
    else launch_scores<T, 256, 8>(a, s);
  }
  return launched(GRAD ? "kf_op_token_scores_grad" : "kf_op_token_scores");
}

template <bool GRAD>
int scores(const char* what, int32_t type, int64_t R, Args a, float tau, cudaStream_t s) {
  const int size = type == KF_TYPE_FP32 ? 4 : 2;
  if (type != KF_TYPE_FP32 && type != KF_TYPE_BF16 && type != KF_TYPE_FP16)
    return refuse(what, "the logits' type is fp32, bf16 or fp16");
  if (R < 0 || R > (1 << 28)) return refuse(what, "rows out of range");
  if (a.V < 1 || a.V > kMostRow / size || a.stride < a.V) return refuse(what, "vocabulary (a row is at most 1 MiB) or row stride out of range");
  if (!(tau > 0.f) || !(1.f / tau > 0.f) || std::isinf(1.f / tau * kLog2e)) return refuse(what, "tau is a positive number, and log2(e) / tau one of fp32's");
  if (a.top < 0 || a.top > kMaxTop || a.top > a.V) return refuse(what, "top is 0 to 64 and at most the vocabulary");
  if (R == 0) return KF_OK;
  if (!a.logits || !a.tokens || (a.top && (!a.top_ids || !a.top_logp))) return refuse(what, "a null array");
  if (!aligned(a.logits, size) || !aligned(a.tokens, 8)) return refuse(what, "an array is not aligned to its elements");
  if (GRAD && (!a.grad || !aligned(a.grad, size) || a.grad_stride < a.V)) return refuse(what, "grad: null, misaligned or rows too near");
  if (GRAD && a.grad == a.logits && a.grad_stride != a.stride) return refuse(what, "grad over the logits has their row stride");
  a.inv_tau = 1.f / tau;
  a.c2 = a.inv_tau * kLog2e;
  a.margin = kRaise / a.c2;
  if (!(a.err = serving_error_word())) return refuse(what, "no error word", KF_E_CUDA);
  if (type == KF_TYPE_FP32) return launch<float, GRAD>(a, s);
  if (type == KF_TYPE_BF16) return launch<__nv_bfloat16, GRAD>(a, s);
  return launch<__half, GRAD>(a, s);
}

}  // namespace
}  // namespace kf

using namespace kf;

extern "C" int kf_op_token_scores(int32_t type, int64_t R, int32_t V, const void* logits, int64_t stride,
                                  const int64_t* tokens, float tau, int32_t top, float* logp, float* entropy,
                                  float* lse, int32_t* top_ids, float* top_logp, void* stream) {
  Args a{logits, stride, tokens, nullptr, nullptr, logp, entropy, lse, top_logp, top_ids, nullptr, 0, R, V, top, 1.f, 1.f, 1.f, nullptr};
  return scores<false>("kf_op_token_scores", type, R, a, tau, (cudaStream_t)stream);
}

extern "C" int kf_op_token_scores_grad(int32_t type, int64_t R, int32_t V, const void* logits, int64_t stride,
                                       const int64_t* tokens, float tau, const float* g_logp,
                                       const float* g_entropy, float* logp, float* entropy, float* lse,
                                       void* grad, int64_t grad_stride, void* stream) {
  Args a{logits, stride, tokens, g_logp, g_entropy, logp, entropy, lse, nullptr, nullptr, grad, grad_stride, R, V, 0, 1.f, 1.f, 1.f, nullptr};
  return scores<true>("kf_op_token_scores_grad", type, R, a, tau, (cudaStream_t)stream);
}
