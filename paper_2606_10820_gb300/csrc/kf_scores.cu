// Scores of tokens under rows of logits (kf_op_token_scores), their
// gradient (kf_op_token_scores_grad), and the clipped policy loss with its gradient
// (kf_op_policy_loss).
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
// Policy loss: the gradient's two passes, with a row's loss and its two derivatives between them (every thread
// computes them: a broadcast would cost a barrier).
//
// Measured: 4096 bf16 rows of 50257 in 96 us with eight alternatives (4.3 TB/s), 72 without (5.7); 8 fp32
// rows 7.5; the gradient of 2048 bf16 rows 86 us (4.8 TB/s); the policy loss of 4096 in 177 us (4.7 TB/s), of 61 fp32 rows in
// 10 us.  The gradient's passes take 20 instructions an element, 62 % of the issue slots: two rows fill an SM's shared
// memory, so two CTAs take turns at loads, barriers and arithmetic.  Measured and not kept: the
// arithmetic on single numbers instead of pairs (fewer moves, more of the fma pipe: 194 us for 179).
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

// the policy loss: its inputs and outputs of a row, its constants
struct Policy {
  const float *old_logp, *advantage, *ref_logp, *weight;
  float *loss, *ratio, *kl;
  float low, high;                 // the ratio's ends
  float kl_weight, entropy_weight, c2_low;      // c2_low: what c2 lost in rounding
};
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
  Policy pol;
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
// so there the logits' difference is formed first and scaled after.
// WHOLE (the policy loss, not where big): references are whole numbers in base-2 units, so that a move from one to another multiplies by a
// power of two and loses nothing
struct Ref {
  float raw, nm;                   // nm: minus the reference, base-2 units (a logit where big)
  float limit;                     // a logit past this raises the reference
  bool big;
  static __device__ __forceinline__ bool large(const Args& a, float r) {
    const float m = fabsf(r * a.inv_tau);
    return m >= kLarge && m < INFINITY;
  }
  template <bool WHOLE>
  static __device__ __forceinline__ float units(const Args& a, float r) {
    return WHOLE ? rintf(__fmul_rn(r, a.c2)) : __fmul_rn(r, a.c2);
  }
  template <bool WHOLE>
  __device__ __forceinline__ void set(const Args& a, float r) {
    const float m = r * a.inv_tau;
    raw = r;
    limit = r == -INFINITY ? r : r + a.margin;
    big = large(a, r);
    nm = m == -INFINITY ? 0.f : big ? -r : -units<WHOLE>(a, r);
  }
  __device__ __forceinline__ bool open(const Args& a) const { return raw * a.inv_tau != -INFINITY; }
  // log2 of exp(x - m)
  __device__ __forceinline__ float less(const Args& a, float v) const {
    return big ? (v + nm) * a.c2 : fmaf(v, a.c2, nm);
  }
  // log2 of exp(m' - m) for an open reference m' of the logit `from`, both as they were rounded
  template <bool WHOLE>
  __device__ __forceinline__ float less_ref(const Args& a, float from) const {
    if (large(a, from)) return less(a, from);
    const float was = units<WHOLE>(a, from);
    return big ? fmaf(nm, a.c2, was) : __fadd_rn(was, nm);      // (no fused multiply-add)
  }
};

// S and T (base-2 units) of some elements against the reference `raw`; without an open element
// they are 0 (or NaN)
struct Sums {
  float raw, s, t;
  // against the reference r (at or above this one)
  template <bool WHOLE>
  __device__ __forceinline__ void move_to(const Args& a, const Ref& r) {
    const float d = raw * a.inv_tau == -INFINITY ? 0.f : fmaxf(r.less_ref<WHOLE>(a, raw), kLeast), f = ex2(d);
    t = f * fmaf(d, s, t);
    s *= f;
    raw = r.raw;
  }
};

__device__ __forceinline__ float min3f(float x, float y, float z) {
  float r;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}
// the largest of a warp's numbers (all 32 lanes call it)
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// One thread's pass over its elements.  LOW, the policy loss: it keeps the smallest too, and batches without a closed token go
// without the clamps (179 -> 173 us; the scores and their gradient, whose registers it costs, are 1.5 % slower so).  What its S may
// lose, log p and the ratio do, and kl = e^u - 1 - u twice that over u.  So the references are whole numbers and at first the warp's largest (exponents round at
// their size), and S is added up a batch at a time: an addition to a sum that holds the row's largest term (a quarter of S, where
// the logits deviate by four) rounds at that term's size, and one chain of fifty of them lost most.  4096 x 50257 bf16, log p off by
// (root of the mean) and us: 1.2e-7 and 174.8 with none of it, 9.0e-8 by batches, 7.5e-8 and 176.0 with whole references,
// 6.6e-8 and 177.7 with the warp's (not kept: with joins in two parts instead 6.1e-8 and 182)
template <bool LOW>
struct Pass {
  Ref r;
  float most = -INFINITY;          // the largest logit
  float least = INFINITY;          // and the smallest
  uint64_t s = 0ull, t = 0ull;     // S and T, in two lanes each
  __device__ __forceinline__ Pass() : r{-INFINITY, 0.f, -INFINITY, false} {}
  __device__ __forceinline__ void raise(const Args& a, float to) {
    const Ref was = r;
    r.template set<LOW>(a, to);
    if (was.open(a)) {
      const float d = fmaxf(r.template less_ref<LOW>(a, was.raw), kLeast), f = ex2(d);
      t = mul_f2(f2(f, f), fma_f2(f2(d, d), s, t));
      s = mul_f2(f2(f, f), s);
    }
  }
  // (to: the sum that S's part goes to)
  __device__ __forceinline__ void pair(float2 d, uint64_t& to) {
    const uint64_t e = f2(ex2(d.x), ex2(d.y));
    to = add_f2(to, e);
    t = fma_f2(e, f2(fmaxf(d.x, kLeast), fmaxf(d.y, kLeast)), t);
  }
  // (differences above kLeast)
  __device__ __forceinline__ void pair_of_open(uint64_t d, uint64_t& to) {
    const float2 x = f2_split(d);
    const uint64_t e = f2(ex2(x.x), ex2(x.y));
    to = add_f2(to, e);
    t = fma_f2(e, d, t);
  }
  // first (uniform over the warp, LOW): the reference is the whole warp's largest
  template <int N>
  __device__ __forceinline__ void add(const Args& a, const float* v, bool first = false) {
    float top = fmaxf(v[0], v[1]), low = LOW ? fminf(v[0], v[1]) : 0.f;
#pragma unroll
    for (int i = 2; i < N; i += 2) {
      top = max3f(top, v[i], v[i + 1]);
      if (LOW) low = min3f(low, v[i], v[i + 1]);
    }
    most = fmaxf(most, top);
    if (LOW) least = fminf(least, low);
    if (LOW && first) raise(a, warp_max(top));
    else if (top > r.limit) raise(a, top);
    const uint64_t c = f2(a.c2, a.c2), nm = f2(r.nm, r.nm);
    uint64_t batch = 0ull, &to = LOW ? batch : s;
    if (LOW && !r.big && fmaf(low, a.c2, r.nm) > kLeast) {
#pragma unroll
      for (int i = 0; i < N; i += 2) pair_of_open(fma_f2(f2(v[i], v[i + 1]), c, nm), to);
    } else if (!r.big) {
#pragma unroll
      for (int i = 0; i < N; i += 2) pair(f2_split(fma_f2(f2(v[i], v[i + 1]), c, nm)), to);
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2) pair(f2_split(mul_f2(add_f2(f2(v[i], v[i + 1]), nm), c)), to);
    }
    if (LOW) s = add_f2(s, batch);
  }
  __device__ __forceinline__ void add_one(const Args& a, float v) {
    most = fmaxf(most, v);
    if (v > r.limit) raise(a, v);
    pair(make_float2(r.less(a, v), -INFINITY), s);
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
  float s, logs, lse, H;           // S, log2 S; H: the entropy
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
template <int THREADS, int CS, bool GROUPS, bool LOW>
__device__ __forceinline__ Scores reduce_row(const Args& a, Shared<THREADS>& sh, const Pass<LOW>& ps) {
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
  o.ref.template set<LOW>(a, m);
  su.template move_to<LOW>(a, o.ref);
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
  o.s = x.x;
  o.logs = log2f(x.x);
  o.lse = o.none ? -INFINITY : o.bad ? NAN : o.ref.raw * a.inv_tau + o.logs * kLn2;
  o.H = o.none ? 0.f : o.bad ? NAN : (o.logs - x.y / x.x) * kLn2;
  return o;
}
// Sum of two numbers, and what its rounding lost
__device__ __forceinline__ float2 two_sum(float x, float y) {
  const float s = __fadd_rn(x, y), z = __fsub_rn(s, x);
  return make_float2(s, __fadd_rn(__fsub_rn(x, __fsub_rn(s, z)), __fsub_rn(y, z)));
}
// The policy loss of a row: ratio = exp(lp - old), u = ref - lp,
//   loss = w (kl_weight (e^u - 1 - u) - min(ratio A, clip(ratio) A) - entropy_weight H),
// and its derivatives by lp and H.  The exponents are small differences of numbers of size ten and more, so
// lp is kept in two parts: in one it would carry 5e-7 of rounding into ratio, and ten times as
// much of its own size into the KL term.
// (its inputs: read before the pass over the row)
struct PolicyIn {
  float w, old, A, ref;
  __device__ __forceinline__ PolicyIn(const Policy& p, int64_t r)
      : w(p.weight ? __ldg(p.weight + r) : 1.f), old(__ldg(p.old_logp + r)), A(__ldg(p.advantage + r)), ref(p.ref_logp ? __ldg(p.ref_logp + r) : 0.f) {}
};
struct PolicyRow {
  float logp, ratio, kl, loss, gl, gh;
  bool left_out;                   // no part in the loss: padding, a weight of 0 (or a token outside the vocabulary)
  __device__ __forceinline__ PolicyRow(const Args& a, const Scores& o, const PolicyIn& in, int64_t token, float at_logit) {
    const Policy& p = a.pol;
    const float w = in.w;
    const bool has = token >= 0 && token < a.V;
    left_out = !has || w == 0.f;
    logp = kl = gl = gh = loss = 0.f;
    ratio = 1.f;
    if (token >= a.V) logp = ratio = kl = loss = NAN;
    if (!has) return;
    // log2 p = (v - m) c - log2 S; S = 2^e f, 1 <= f < 2
    float2 x;
    if (o.bad) x = make_float2(NAN, 0.f);
    else if (o.none) x = make_float2(-INFINITY, 0.f);
    else {
      const int bits = __float_as_int(o.s);       // (S is above a half: the reference is an element to half a unit)
      const float e = (float)((bits >> 23) - 127), f = __int_as_float((bits & 0x7fffff) | 0x3f800000);
      float lo;
      if (!o.ref.big) {
        const float v = __fmul_rn(at_logit, a.c2);
        x = two_sum(v, o.ref.nm);
        lo = fmaf(at_logit, a.c2, -v);
      } else {
        const float d = at_logit + o.ref.nm;
        x = make_float2(__fmul_rn(d, a.c2), 0.f);
        lo = fmaf(d, a.c2, -x.x);
      }
      // (what c2 lost in rounding, of the token's difference and of S: d log2 S / d c = sum p (v - m), with m the reference as it was rounded)
      const float mean = o.logs - o.H * kLog2e;
      lo += x.y + fmaf((x.x - mean) / a.c2, p.c2_low, -log2f(f));
      x = two_sum(x.x, -e);
      x = two_sum(x.x, x.y + lo);
      if (!(fabsf(x.x) < INFINITY)) x = make_float2(o.lp(a, at_logit) * kLog2e, 0.f);
      // in natural units
      constexpr float kLn2Low = -1.9046543e-9f;   // what kLn2 lost in rounding
      const float h = __fmul_rn(x.x, kLn2);
      if (fabsf(h) < INFINITY) x = make_float2(h, fmaf(x.x, kLn2, -h) + fmaf(x.y, kLn2, x.x * kLn2Low));
      else x = make_float2(h, 0.f);
    }
    logp = x.x + x.y;
    const float A = in.A;
    ratio = expf((x.x - in.old) + x.y);
    float em1 = 0.f;               // e^u - 1
    if (p.ref_logp) {
      const float u = (in.ref - x.x) - x.y;
      if (fabsf(u) < 0.25f) {
        // u^2 / 2 + u^3 / 6 + ... to u^8
        kl = u * u * fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, 1.f / 40320, 1.f / 5040), 1.f / 720), 1.f / 120), 1.f / 24), 1.f / 6), 0.5f);
        em1 = u + kl;
      } else {
        em1 = expm1f(u);
        kl = em1 == INFINITY ? em1 : em1 - u;
      }
    }
    if (w == 0.f) return;
    // whether the clip decides (comparisons, false of a NaN: fminf and fmaxf would drop it, and the loss be a number)
    const bool clipped = A > 0.f ? ratio > p.high : A < 0.f && ratio < p.low;
    const float gain = (!clipped ? ratio : A > 0.f ? p.high : p.low) * A;
    const float k = p.kl_weight == 0.f ? 0.f : p.kl_weight * kl, gk = p.kl_weight == 0.f ? 0.f : p.kl_weight * em1;
    const float c = p.entropy_weight == 0.f ? 0.f : p.entropy_weight * o.H;
    loss = w * (k - gain - c);
    gl = w * (-gk - (clipped ? 0.f : ratio * A));
    gh = -w * p.entropy_weight;
  }
};
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
  __device__ __forceinline__ Extra(const Args& a, const Row<T>& row, int64_t r, bool first_cta, bool all = false) {
    const int t = threadIdx.x;
    token = a.tokens[r];
    at_logit = (all || t == 0) && token >= 0 && token < a.V ? to_f(row.p[token]) : 0.f;
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
    Pass<false> ps;
#pragma unroll 1
    for (int b = 0; b < batches; ++b) {
      mma::cp_wait<kRing<THREADS> - 2>();          // this batch has landed
      fill();                             // into the slots of the batch before
      const uint4* s = slots + slot * kBatch * THREADS + t;
      if ((b + 1) * kBatch <= n) {
        float v[kBatch * N];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) Vec16<T>::unpack(s[j * THREADS], v + j * N);
        ps.template add<kBatch * N>(a, v);
      } else {
        for (int j = 0; b * kBatch + j < n; ++j) {
          float v[N];
          Vec16<T>::unpack(s[j * THREADS], v);
          ps.template add<N>(a, v);
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
template <typename T, int THREADS, int CS, bool POLICY>
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
    const Extra<T> ex(a, row, r, rank == 0, POLICY);
    const int n = mine.have(row), n_next = mine.have(next);
    std::conditional_t<POLICY, PolicyIn, int> input = [&] {
      if constexpr (POLICY) return PolicyIn(a.pol, r);
      else return 0;
    }();
    Pass<POLICY> ps;
    const bool together = POLICY && __all_sync(~0u, kBatch <= n);      // all lanes have a first batch
#pragma unroll (POLICY ? 1 : kResident)
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
        ps.template add<kBatch * N>(a, v, together && g == 0);
      } else {
        for (int j = 0; g * kBatch + j < n; ++j) {
          float v[N];
          Vec16<T>::unpack(s[j * THREADS], v);
          ps.template add<N>(a, v);
        }
      }
    }
    if (ex.edge) ps.add_one(a, ex.edge_logit);
    const Scores o = reduce_row<THREADS, CS, false>(a, sh, ps);
    float gl, gh;
    bool zeros = false;                   // (uniform) a row that the loss leaves out, whatever it holds
    if constexpr (POLICY) {
      const PolicyRow p(a, o, input, ex.token, ex.at_logit);
      gl = p.gl;
      gh = p.gh;
      zeros = p.left_out || o.none;
      if (rank == 0 && t == 0) {
        if (ex.token >= a.V) atomicOr(a.err, KF_DEV_BAD_TOKEN);
        a.logp[r] = p.logp;
        a.entropy[r] = o.H;
        a.pol.loss[r] = p.loss;
        a.pol.ratio[r] = p.ratio;
        if (a.pol.kl) a.pol.kl[r] = p.kl;
      }
    } else {
      if (rank == 0 && t == 0) write_numbers(a, r, o, ex.token, ex.at_logit);
      const bool has = ex.token >= 0 && ex.token < a.V;
      gl = has && a.g_logp ? a.g_logp[r] : 0.f;
      gh = a.g_entropy ? a.g_entropy[r] : 0.f;
    }
    // grad = p (A + B log2 p) + (v == token) gl / tau.  A row with a NaN has A = NaN; one
    // without open tokens p = 0
    const float A = (-gl - gh * o.H) * a.inv_tau, B = -gh * a.inv_tau * kLn2;
    const float at_token = o.none ? 0.f : gl * a.inv_tau;
    T* out = static_cast<T*>(a.grad) + r * a.grad_stride;
    // log2 p of a logit (one constant for both would lose log S); `value`: its gradient but for the token's part
    auto log_p = [&](float v) {
      return __fadd_rn(o.ref.big ? __fmul_rn(__fadd_rn(v, o.ref.nm), a.c2) : fmaf(v, a.c2, o.ref.nm), -o.logs);
    };
    auto value = [&](float d) { return __fmul_rn(ex2(d), fmaf(B, d, A)); };
    // The policy loss takes one constant all the same, and what that loses, the same of all of the row's elements, into A and B:
    // p (A + B log2 p) = 2^d f (A + B lo + B d), d = log2 p - lo, f = 2^lo
    const float2 nml = two_sum(o.ref.nm, -o.logs);
    const float f = ex2(nml.y), B1 = B * f, A1 = fmaf(B, nml.y, A) * f;
    // (no clamp where none of this thread's elements needs it)
    const uint64_t c2 = f2(a.c2, a.c2), nm = f2(o.ref.nm, o.ref.nm), nlogs = f2(-o.logs, -o.logs), A2 = f2(A, A), B2 = f2(B, B);
    const uint64_t nml2 = f2(nml.x, nml.x), A12 = f2(A1, A1), B12 = f2(B1, B1);
    const bool plain = !o.none && !o.ref.big && fmaf(ps.least, a.c2, nml.x) > kLeast + 1.f;
    const int token = ex.token >= 0 && ex.token < a.V ? (int)ex.token : -1;
    const bool same = (reinterpret_cast<uintptr_t>(out) & 15) == (reinterpret_cast<uintptr_t>(row.p) & 15);
    if (ex.edge) {
      float x = value(fmaxf(log_p(ex.edge_logit), kLeast));
      if (POLICY && zeros) x = 0.f;
      out[ex.edge_id] = from_f<T>(ex.edge_id == token ? x + at_token : x);
    }
#pragma unroll (POLICY ? 1 : kResident)
    for (int g = 0; g < kResident; ++g) {
#pragma unroll
      for (int jj = 0; jj < kBatch; ++jj) {
        const int j = g * kBatch + jj;
        if (j >= n) break;
        float v[N];
        Vec16<T>::unpack(slots[j * THREADS + t], v);
        const int id0 = row.head + (mine.first + j * THREADS) * N;
        if constexpr (!POLICY) {
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            const uint64_t x = f2(v[e], v[e + 1]);
            float2 d;
            if (!o.ref.big) d = f2_split(add_f2(fma_f2(x, c2, nm), nlogs));
            else d = f2_split(add_f2(mul_f2(add_f2(x, nm), c2), nlogs));
            d.x = fmaxf(d.x, kLeast);
            d.y = fmaxf(d.y, kLeast);
            const float2 y = f2_split(mul_f2(f2(ex2(d.x), ex2(d.y)), fma_f2(B2, f2(d.x, d.y), A2)));
            v[e] = y.x;
            v[e + 1] = y.y;
          }
        } else if (plain && !zeros) {
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            const uint64_t d = fma_f2(f2(v[e], v[e + 1]), c2, nml2);
            const float2 ds = f2_split(d);
            const float2 y = f2_split(mul_f2(f2(ex2(ds.x), ex2(ds.y)), fma_f2(B12, d, A12)));
            v[e] = y.x;
            v[e + 1] = y.y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) v[e] = zeros ? 0.f : value(fmaxf(log_p(v[e]), kLeast));
        }
        if ((unsigned)(token - id0) < (unsigned)N) {
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (id0 + e == token) v[e] += at_token;
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
template <typename T, int THREADS, int CS, bool POLICY>
void launch_grad(const Args& a, cudaStream_t s) {
  static PerDevice attr;
  const int k = (a.V / Vec16<T>::N + CS * THREADS - 1) / (CS * THREADS);
  launch_rows<THREADS, CS>(k_scores_grad<T, THREADS, CS, POLICY>, attr, a, (size_t)k * THREADS * 16, s);
}
enum Kind { SCORES, GRAD, POLICY };
constexpr const char* kNames[] = {"kf_op_token_scores", "kf_op_token_scores_grad", "kf_op_policy_loss"};
template <typename T, Kind K>
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
  if constexpr (K != SCORES) {
    while (cs < 8 && (bytes > (int64_t)cs * kPairBytes || (a.R * cs * 2 <= sms && bytes >= cs * 2 * 2 * 512 * 16))) cs *= 2;
    if (bytes <= 12288 && a.R > 2 * sms) launch_grad<T, 64, 1, K == POLICY>(a, s);
    else if (cs == 1) launch_grad<T, 512, 1, K == POLICY>(a, s);
    else if (cs == 2) launch_grad<T, 512, 2, K == POLICY>(a, s);
    else if (cs == 4) launch_grad<T, 512, 4, K == POLICY>(a, s);
    else launch_grad<T, 512, 8, K == POLICY>(a, s);
  } else {
    while (cs < 8 && a.R * cs * 2 <= sms && bytes >= cs * 2 * 2 * 256 * 16) cs *= 2;
    if (a.R > 4 * sms && a.top <= kFew && bytes <= (a.top ? 49152 : 114688)) launch_scores<T, 64, 1>(a, s);
    else if (cs == 1) launch_scores<T, 256, 1>(a, s);
    else if (cs == 2) launch_scores<T, 256, 2>(a, s);
    else if (cs == 4) launch_scores<T, 256, 4>(a, s);
    else launch_scores<T, 256, 8>(a, s);
  }
  return launched(kNames[K]);
}

template <Kind K>
int scores(int32_t type, int64_t R, Args a, float tau, cudaStream_t s) {
  const char* what = kNames[K];
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
  if (K != SCORES && (!a.grad || !aligned(a.grad, size) || a.grad_stride < a.V)) return refuse(what, "grad: null, misaligned or rows too near");
  if (K != SCORES && a.grad == a.logits && a.grad_stride != a.stride) return refuse(what, "grad over the logits has their row stride");
  a.inv_tau = 1.f / tau;
  a.c2 = a.inv_tau * kLog2e;
  a.margin = kRaise / a.c2;
  if (!(a.err = serving_error_word())) return refuse(what, "no error word", KF_E_CUDA);
  if (type == KF_TYPE_FP32) return launch<float, K>(a, s);
  if (type == KF_TYPE_BF16) return launch<__nv_bfloat16, K>(a, s);
  return launch<__half, K>(a, s);
}

}  // namespace
}  // namespace kf

using namespace kf;

extern "C" int kf_op_token_scores(int32_t type, int64_t R, int32_t V, const void* logits, int64_t stride,
                                  const int64_t* tokens, float tau, int32_t top, float* logp, float* entropy,
                                  float* lse, int32_t* top_ids, float* top_logp, void* stream) {
  Args a{logits, stride, tokens, nullptr, nullptr, logp, entropy, lse, top_logp, top_ids, nullptr, 0, R, V, top, 1.f, 1.f, 1.f, nullptr, {}};
  return scores<SCORES>(type, R, a, tau, (cudaStream_t)stream);
}

extern "C" int kf_op_token_scores_grad(int32_t type, int64_t R, int32_t V, const void* logits, int64_t stride,
                                       const int64_t* tokens, float tau, const float* g_logp,
                                       const float* g_entropy, float* logp, float* entropy, float* lse,
                                       void* grad, int64_t grad_stride, void* stream) {
  Args a{logits, stride, tokens, g_logp, g_entropy, logp, entropy, lse, nullptr, nullptr, grad, grad_stride, R, V, 0, 1.f, 1.f, 1.f, nullptr, {}};
  return scores<GRAD>(type, R, a, tau, (cudaStream_t)stream);
}

extern "C" int kf_op_policy_loss(int32_t type, int64_t R, int32_t V, const void* logits, int64_t stride, const int64_t* tokens,
                                 double tau, const float* old_logp, const float* advantage, const float* ref_logp,
                                 const float* weight, float clip_low, float clip_high, float kl_weight, float entropy_weight,
                                 float* loss, float* logp, float* entropy, float* ratio, float* kl, void* grad, int64_t grad_stride,
                                 void* stream) {
  const char* what = "kf_op_policy_loss";
  if (!(clip_low >= 0.f) || !(clip_low <= 1.f) || !(clip_high >= 0.f)) return refuse(what, "clip: 0 to 1 below, 0 or more above");
  if (!(std::fabs(kl_weight) < INFINITY) || !(std::fabs(entropy_weight) < INFINITY)) return refuse(what, "the terms' weights are finite");
  if (kl_weight != 0.f && !ref_logp) return refuse(what, "the KL term wants ref_logp");
  if (R > 0 && (!old_logp || !advantage || !loss || !logp || !entropy || !ratio || (ref_logp && !kl))) return refuse(what, "a null array");
  for (const void* p : {(const void*)old_logp, (const void*)advantage, (const void*)ref_logp, (const void*)weight, (const void*)loss,
                        (const void*)logp, (const void*)entropy, (const void*)ratio, (const void*)kl})
    if (!aligned(p, 4)) return refuse(what, "an array is not aligned to its elements");
  const double c = 1.4426950408889634074 / tau;
  Args a{logits, stride, tokens, nullptr, nullptr, logp, entropy, nullptr, nullptr, nullptr, grad, grad_stride, R, V, 0, 1.f, 1.f, 1.f, nullptr,
         Policy{old_logp, advantage, ref_logp, weight, loss, ratio, ref_logp ? kl : nullptr, 1.f - clip_low, 1.f + clip_high, kl_weight,
                entropy_weight, 0.f}};
  const float t32 = (float)tau;
  if (t32 > 0.f) a.pol.c2_low = (float)(c - (double)(float)((1.f / t32) * kLog2e));
  return scores<POLICY>(type, R, a, t32, (cudaStream_t)stream);
}
