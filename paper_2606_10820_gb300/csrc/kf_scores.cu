// Scores of tokens under rows of logits (kf_op_token_scores) and their
// gradient (kf_op_token_scores_grad).
//
// With x = logits / tau and a reference m near max x, one pass over a row gives
//   S = sum exp(x - m),  T = sum (x - m) exp(x - m),
//   lse = m + log S,     entropy = log S - T / S
// (against a near reference no term cancels against a much larger one).
// A thread keeps (m, S, T) of the 16-byte vectors it reads; two such triples
// join as S = S1 f1 + S2 f2, T = f1 (T1 + d1 S1) + f2 (T2 + d2 S2) with d = m_i - m
// and f = exp(d).  All of it is fp32, in base-2 units: 2^d with d = x log2(e) - m log2(e).
//
// Top alternatives: the 256 threads of a row's CTA (CTAs) form 64 groups, and the
// n-th largest of the 64 groups' maxima is at or below the n-th largest logit (n
// groups have an element at or above it).  So only the vectors of threads whose own
// maximum reaches that bound are read again (from L2, a warp per such thread), and their
// elements at or above it listed, a few dozen of a vocabulary; each one's rank among
// them is its place.  Rows where that list would not fit (ties in the hundreds) choose round by round.
//
// What bounds it: the logits' bytes, read once (scores) or read and written once (gradient:
// the second reading comes from L2), and close behind them the instructions: five an
// element and pass, most of them on pairs (fma.rn.f32x2).
#include <algorithm>
#include <cooperative_groups.h>

#include "kf_serving.cuh"
#include "kf_tc.cuh"

namespace cg = cooperative_groups;

namespace kf {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kGroups = 64;        // groups whose maxima bound the n-th largest logit
constexpr int kMaxTop = kGroups;
constexpr int kLanes = kThreads / kGroups;   // lanes of a group (times the CTAs of the row)
constexpr int kList = 1024;        // listed candidates of a row
constexpr int kRanked = 256;       // up to so many are ranked against each other, more are chosen in rounds
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -300.f;   // 2^-300 is 0 in fp32: stands for -inf where it multiplies that 0
constexpr float kRaise = 8.f;
constexpr float kBig = 1e38f;      // references past it would overflow in base-2 units

struct Args {
  const void* logits;
  int64_t stride;
  const int64_t* tokens;
  const float *g_logp, *g_entropy;
  float *logp, *entropy, *lse, *top_logp;
  int32_t* top_ids;
  void* grad;
  int64_t grad_stride;
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
__device__ __forceinline__ uint4 ld_stream(const void* p) {
  uint4 u;
  asm("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
  return u;
}

// What scores are taken against: a logit `raw` that no element exceeds by more than
// 2^kRaise.  (The maximum itself would change for some lane of a warp at almost every
// vector: with a kRaise of 0 the changes were half of all instructions, 123 against
// 81 us at 4096 x 50257.)  A reference past kBig (a row at the type's lowest value) keeps its
// differences in natural units until they are formed
struct Ref {
  float raw, nm;                   // nm: minus the reference, base-2 units (natural where big)
  float limit;                     // a logit past this raises the reference
  bool big;
  __device__ __forceinline__ void set(const Args& a, float r) {
    const float m = r * a.inv_tau;
    raw = r;
    limit = r == -INFINITY ? r : r + a.margin;
    big = fabsf(m) > kBig && fabsf(m) < INFINITY;
    nm = m == -INFINITY ? 0.f : big ? -m : -__fmul_rn(r, a.c2);
  }
  __device__ __forceinline__ bool open(const Args& a) const { return raw * a.inv_tau != -INFINITY; }
  // log2 of exp(x - m)
  __device__ __forceinline__ float less(const Args& a, float v) const {
    return big ? fmaf(v, a.inv_tau, nm) * kLog2e : fmaf(v, a.c2, nm);
  }
};

// S and T (base-2 units) of some elements against their Ref; without an open element they are 0 (or NaN)
struct Sums {
  float raw, s, t;
};
__device__ __forceinline__ Sums join(const Args& a, Sums x, Sums y) {
  Ref r;
  r.set(a, fmaxf(x.raw, y.raw));
  Sums o{r.raw, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const Sums c = i ? y : x;
    // (the difference of the two references as they were rounded: no fused multiply-add)
    const float by = r.big ? r.less(a, c.raw) : __fadd_rn(__fmul_rn(c.raw, a.c2), r.nm);
    const float d = c.raw * a.inv_tau == -INFINITY ? 0.f : fmaxf(by, kLeast), f = ex2(d);
    o.s += f * c.s;
    o.t += f * fmaf(d, c.s, c.t);
  }
  return o;
}

// one thread's pass over its elements
struct Pass {
  Ref r;
  float most = -INFINITY;          // the largest logit
  uint64_t s = 0ull, t = 0ull;     // S and T, each in two lanes
  __device__ __forceinline__ Pass() : r{-INFINITY, 0.f, -INFINITY, false} {}
  __device__ __forceinline__ void raise(const Args& a, float to) {
    const Ref was = r;
    r.set(a, to);
    if (was.open(a)) {
      const float by = r.big ? r.less(a, was.raw) : was.big ? -INFINITY : __fsub_rn(r.nm, was.nm);
      const float d = fmaxf(by, kLeast), f = ex2(d);
      t = mul_f2(f2(f, f), fma_f2(f2(d, d), s, t));
      s = mul_f2(f2(f, f), s);
    }
  }
  __device__ __forceinline__ void pair(float dx, float dy) {
    const uint64_t e = f2(ex2(dx), ex2(dy));
    s = add_f2(s, e);
    t = fma_f2(e, f2(fmaxf(dx, kLeast), fmaxf(dy, kLeast)), t);
  }
  template <int N>
  __device__ __forceinline__ void add(const Args& a, const float* v) {
    float top = fmaxf(v[0], v[1]);
#pragma unroll
    for (int i = 2; i < N; i += 2) top = max3f(top, v[i], v[i + 1]);
    most = fmaxf(most, top);
    if (top > r.limit) raise(a, top);
    if (!r.big) {
      const uint64_t c = f2(a.c2, a.c2), nm = f2(r.nm, r.nm);
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const float2 d = f2_split(fma_f2(f2(v[i], v[i + 1]), c, nm));
        pair(d.x, d.y);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2) pair(r.less(a, v[i]), r.less(a, v[i + 1]));
    }
  }
  __device__ __forceinline__ void add_one(const Args& a, float v) {
    most = fmaxf(most, v);
    if (v > r.limit) raise(a, v);
    pair(r.less(a, v), -INFINITY);
  }
  __device__ __forceinline__ Sums sums() const {
    const float2 a = f2_split(s), b = f2_split(t);
    return Sums{r.raw, a.x + a.y, b.x + b.y};
  }
};

// A row's elements in 16-byte vectors: `head` elements lie before the first
// aligned one, then nvec vectors, then the rest
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

// f(id, logit) for the elements of vector i
template <typename T, typename F>
__device__ __forceinline__ void each_of_vector(const Row<T>& row, int i, F f) {
  float v[Vec16<T>::N];
  Vec16<T>::unpack(*reinterpret_cast<const uint4*>(row.vec(i)), v);
  const int id0 = row.head + i * Vec16<T>::N;
#pragma unroll
  for (int e = 0; e < Vec16<T>::N; ++e) f(id0 + e, v[e]);
}

struct Cand {
  float x;
  int id;
};
__device__ __forceinline__ bool before(Cand a, Cand b) { return a.x > b.x || (a.x == b.x && a.id < b.id); }
// the first of the block's candidates in that order (every thread gets it)
__device__ __forceinline__ Cand block_first(Cand c, Cand* buf) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const Cand d{__shfl_xor_sync(~0u, c.x, o), __shfl_xor_sync(~0u, c.id, o)};
    if (before(d, c)) c = d;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = c;
  __syncthreads();
  c = buf[0];
  for (int i = 1; i < kWarps; ++i)
    if (before(buf[i], c)) c = buf[i];
  return c;
}

struct Shared {
  Sums warp[kWarps];
  Sums cta;
  float group[kGroups];
  float bound;
  int count, again;
  int thread[kThreads];            // threads whose vectors are read again
  Cand first[kWarps];
  Cand list[kList];
};

// Clusters of CS CTAs share a row (CS = 1: no cluster).  GRAD: the gradient's
// second pass instead of the alternatives.
template <typename T, int CS, bool GRAD>
__global__ void __launch_bounds__(kThreads, 4) k_scores(const Args a) {
  __shared__ Shared sh;
  constexpr int N = Vec16<T>::N;
  constexpr int kAll = CS * kThreads;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int64_t r = blockIdx.x / CS;
  const int rank = blockIdx.x % CS, me = rank * kThreads + t;
  const Row<T> row(static_cast<const T*>(a.logits) + r * a.stride, a.V);
  // (read before the barriers: the gradient may overwrite the logits)
  const int64_t token = a.tokens[r];
  const float at_logit = t == 0 && token >= 0 && token < a.V ? to_f(row.p[token]) : 0.f;

  Pass ps;
  {
    int i = me;
    for (; i + 3 * kAll < row.nvec; i += 4 * kAll) {
      uint4 u[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = ld_stream(row.vec(i + j * kAll));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float v[N];
        Vec16<T>::unpack(u[j], v);
        ps.add<N>(a, v);
      }
    }
    for (; i < row.nvec; i += kAll) {
      float v[N];
      Vec16<T>::unpack(ld_stream(row.vec(i)), v);
      ps.add<N>(a, v);
    }
  }
  const float vec_max = ps.most;
  if (me < row.edge()) ps.add_one(a, to_f(row.p[row.edge_id(me)]));      // (fewer than 256 of them)
  // the row's sums, in one fixed order
  Sums su = ps.sums();
  auto join_lanes = [&](int o) {
    const Sums other{__shfl_xor_sync(~0u, su.raw, o), __shfl_xor_sync(~0u, su.s, o), __shfl_xor_sync(~0u, su.t, o)};
    su = (lane & o) ? join(a, other, su) : join(a, su, other);
  };
#pragma unroll
  for (int o = 16; o; o >>= 1) join_lanes(o);
  if (lane == 0) sh.warp[warp] = su;
  if (!GRAD && a.top) {
    // the groups' maxima
    float gm = ps.most;
#pragma unroll
    for (int o = 1; o < kLanes * CS; o <<= 1) gm = fmaxf(gm, __shfl_xor_sync(~0u, gm, o));
    if (t % (kLanes * CS) == 0) sh.group[t / (kLanes * CS)] = gm;
    if (t == 0) sh.count = sh.again = 0;
  }
  __syncthreads();
  su = sh.warp[lane % kWarps];
#pragma unroll
  for (int o = kWarps / 2; o; o >>= 1) join_lanes(o);
  Shared* lead = &sh;
  if constexpr (CS > 1) {
    cg::cluster_group cl = cg::this_cluster();
    if (t == 0) sh.cta = su;
    cl.sync();
    su = cl.map_shared_rank(&sh, 0)->cta;
    for (int c = 1; c < CS; ++c) su = join(a, su, cl.map_shared_rank(&sh, c)->cta);
    lead = cl.map_shared_rank(&sh, 0);
    // every CTA has all groups' maxima
    const bool take = !GRAD && a.top && t < kGroups;
    float g = 0.f;
    if (take) g = cl.map_shared_rank(&sh, t / (kGroups / CS))->group[t % (kGroups / CS)];
    cl.sync();          // the other CTAs have read this one's part
    if (take) sh.group[t] = g;
    __syncthreads();
  }
  Ref ref;
  ref.set(a, su.raw);
  const bool none = !ref.open(a) && su.s == 0.f;          // every token closed
  const bool bad = !(su.s > 0.f) && !none;                // NaN or +inf in the row
  const float logs = log2f(su.s);                         // (base-2 units)
  const float lse = none ? -INFINITY : bad ? NAN : su.raw * a.inv_tau + logs * kLn2;
  const float H = none ? 0.f : bad ? NAN : (logs - su.t / su.s) * kLn2;
  // log p of a logit: from the difference to the reference, not from lse, which loses log S where the
  // reference is the type's lowest value (and in natural units where base-2 ones overflow)
  auto lp_of = [&](float v) {
    const float x = v * a.inv_tau;
    return fabsf(x) > kBig ? (x - ref.raw * a.inv_tau) - logs * kLn2 : (ref.less(a, v) - logs) * kLn2;
  };
  if (rank == 0 && t == 0) {
    if (a.lse) a.lse[r] = lse;
    if (a.entropy) a.entropy[r] = H;
    if (token >= a.V) atomicOr(a.err, KF_DEV_BAD_TOKEN);
    if (a.logp) a.logp[r] = token < 0 ? 0.f : token >= a.V || bad ? NAN : none ? -INFINITY : lp_of(at_logit);
  }

  if constexpr (GRAD) {
    const bool has = token >= 0 && token < a.V;
    const float gl = has && a.g_logp ? a.g_logp[r] : 0.f, gh = a.g_entropy ? a.g_entropy[r] : 0.f;
    // grad = p (A + B log2 p) + (v == token) gl / tau.  A row with a NaN has A = NaN; one
    // without open tokens p = 0
    const float A = (-gl - gh * H) * a.inv_tau, B = -gh * a.inv_tau * kLn2;
    const float at_token = none ? 0.f : gl * a.inv_tau;
    T* out = static_cast<T*>(a.grad) + r * a.grad_stride;
    const uint64_t c2 = f2(a.c2, a.c2), nm = f2(ref.nm, ref.nm), nlogs = f2(-logs, -logs), A2 = f2(A, A), B2 = f2(B, B);
    auto pair = [&](float& x, float& y) {
      float2 d;
      if (!ref.big) d = f2_split(add_f2(fma_f2(f2(x, y), c2, nm), nlogs));      // (one constant for both would lose log S)
      else d = make_float2(ref.less(a, x) - logs, ref.less(a, y) - logs);
      d.x = fmaxf(d.x, kLeast);
      d.y = fmaxf(d.y, kLeast);
      const float2 g = f2_split(mul_f2(f2(ex2(d.x), ex2(d.y)), fma_f2(B2, f2(d.x, d.y), A2)));
      x = g.x;
      y = g.y;
    };
    const bool same = (reinterpret_cast<uintptr_t>(out) & 15) == (reinterpret_cast<uintptr_t>(row.p) & 15);
    if (me < row.edge()) {
      const int id = row.edge_id(me);
      float x = to_f(row.p[id]), y = -INFINITY;
      pair(x, y);
      out[id] = from_f<T>(id == token ? x + at_token : x);
    }
    auto store = [&](int i, uint4 u) {
      float v[N];
      Vec16<T>::unpack(u, v);
      const int id0 = row.head + i * N;
#pragma unroll
      for (int e = 0; e < N; e += 2) pair(v[e], v[e + 1]);
      if (token >= id0 && token < id0 + N) {
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
    };
    int i = me;
    for (; i + 3 * kAll < row.nvec; i += 4 * kAll) {
      uint4 u[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = *reinterpret_cast<const uint4*>(row.vec(i + j * kAll));
#pragma unroll
      for (int j = 0; j < 4; ++j) store(i + j * kAll, u[j]);
    }
    for (; i < row.nvec; i += kAll) store(i, *reinterpret_cast<const uint4*>(row.vec(i)));
    return;
  }

  if (a.top == 0) return;                 // (uniform)
  int32_t* ids = a.top_ids + r * a.top;
  float* lps = a.top_logp + r * a.top;
  if (bad) {                              // (uniform over the row's CTAs)
    if (rank == 0 && t < a.top) {
      ids[t] = -1;
      lps[t] = NAN;
    }
    return;
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
  const float bound = sh.bound;
  // (a bound of -inf: the open tokens are listed, the closed ones follow by id)
  auto listed = [&](float x) { return x >= bound && x > -INFINITY; };
  auto list = [&](int id, float v) {
    const float x = v * a.inv_tau;
    if (listed(x)) {
      const int at = atomicAdd(&lead->count, 1);
      if (at < kList) lead->list[at] = Cand{x, id};
    }
  };
  if (listed(vec_max * a.inv_tau)) sh.thread[atomicAdd(&sh.again, 1)] = t;
  if (me < row.edge()) list(row.edge_id(me), to_f(row.p[row.edge_id(me)]));
  __syncthreads();
  for (int k = warp; k < sh.again; k += kWarps)
    for (int i = rank * kThreads + sh.thread[k] + lane * kAll; i < row.nvec; i += 32 * kAll) each_of_vector(row, i, list);
  if constexpr (CS > 1) cg::this_cluster().sync();
  else __syncthreads();
  if (rank != 0) return;
  const int n = sh.count;
  auto put = [&](int place, Cand c) {
    ids[place] = c.id;
    lps[place] = lp_of(to_f(row.p[c.id]));
  };
  if (n <= kRanked) {
    if (t < n) {
      const Cand c = sh.list[t];
      int rk = 0;
      for (int j = 0; j < n; ++j) rk += before(sh.list[j], c);
      if (rk < a.top) put(rk, c);
    }
  } else {
    // round by round: the first candidate after the last one chosen, of the list or
    // (where that overflowed) of the row
    Cand last{INFINITY, -1};
    for (int k = 0; k < min(n, a.top); ++k) {
      Cand c{-INFINITY, 0x7fffffff};
      auto look = [&](Cand d) {
        if (before(last, d) && before(d, c)) c = d;
      };
      auto look_at = [&](int id, float v) {
        const float x = v * a.inv_tau;
        if (listed(x)) look(Cand{x, id});
      };
      if (n <= kList) {
        for (int j = t; j < n; j += kThreads) look(sh.list[j]);
      } else {
        if (t < row.edge()) look_at(row.edge_id(t), to_f(row.p[row.edge_id(t)]));
        for (int i = t; i < row.nvec; i += kThreads) each_of_vector(row, i, look_at);
      }
      last = block_first(c, sh.first);
      if (t == 0) put(k, last);
    }
  }
  // fewer open tokens than asked for: closed ones by id
  if (n < a.top && t == 0) {
    int k = n;
    for (int id = 0; k < a.top; ++id) {
      if (to_f(row.p[id]) * a.inv_tau > -INFINITY) continue;
      ids[k] = id;
      lps[k++] = -INFINITY;
    }
  }
}

template <typename T, bool GRAD>
int launch(const Args& a, int64_t R, cudaStream_t s) {
  // Few rows: a row is split over a cluster while the CTAs fit the SMs, and each
  // thread keeps two vectors
  const int64_t sms = device_sms(), vecs = a.V / Vec16<T>::N;
  const int cs = R * 8 <= sms && vecs >= 8 * 2 * kThreads ? 8 : R * 4 <= 2 * sms && vecs >= 4 * 2 * kThreads ? 4
                 : R * 2 <= 3 * sms && vecs >= 2 * 2 * kThreads ? 2 : 1;
  const dim3 grid((unsigned)(R * cs));
  if (cs == 8) launch_cluster(k_scores<T, 8, GRAD>, grid, dim3(kThreads), 0, 8, false, s, a);
  else if (cs == 4) launch_cluster(k_scores<T, 4, GRAD>, grid, dim3(kThreads), 0, 4, false, s, a);
  else if (cs == 2) launch_cluster(k_scores<T, 2, GRAD>, grid, dim3(kThreads), 0, 2, false, s, a);
  else launch_cluster(k_scores<T, 1, GRAD>, grid, dim3(kThreads), 0, 1, false, s, a);
  return launched(GRAD ? "kf_op_token_scores_grad" : "kf_op_token_scores");
}

template <bool GRAD>
int scores(const char* what, int32_t type, int64_t R, Args a, float tau, cudaStream_t s) {
  const int size = type == KF_TYPE_FP32 ? 4 : 2;
  if (type != KF_TYPE_FP32 && type != KF_TYPE_BF16 && type != KF_TYPE_FP16)
    return refuse(what, "the logits' type is fp32, bf16 or fp16");
  if (R < 0 || R > (1 << 28)) return refuse(what, "rows out of range");
  if (a.V < 1 || a.V > (1 << 30) || a.stride < a.V) return refuse(what, "vocabulary or row stride out of range");
  if (!(tau > 0.f) || !(1.f / tau > 0.f) || std::isinf(1.f / tau)) return refuse(what, "tau is a positive number");
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
  if (type == KF_TYPE_FP32) return launch<float, GRAD>(a, R, s);
  if (type == KF_TYPE_BF16) return launch<__nv_bfloat16, GRAD>(a, R, s);
  return launch<__half, GRAD>(a, R, s);
}

}  // namespace
}  // namespace kf

using namespace kf;

extern "C" int kf_op_token_scores(int32_t type, int64_t R, int32_t V, const void* logits, int64_t stride,
                                  const int64_t* tokens, float tau, int32_t top, float* logp, float* entropy,
                                  float* lse, int32_t* top_ids, float* top_logp, void* stream) {
  Args a{logits, stride, tokens, nullptr, nullptr, logp, entropy, lse, top_logp, top_ids, nullptr, 0, V, top, 1.f, 1.f, 1.f, nullptr};
  return scores<false>("kf_op_token_scores", type, R, a, tau, (cudaStream_t)stream);
}

extern "C" int kf_op_token_scores_grad(int32_t type, int64_t R, int32_t V, const void* logits, int64_t stride,
                                       const int64_t* tokens, float tau, const float* g_logp,
                                       const float* g_entropy, float* logp, float* entropy, float* lse,
                                       void* grad, int64_t grad_stride, void* stream) {
  Args a{logits, stride, tokens, g_logp, g_entropy, logp, entropy, lse, nullptr, nullptr, grad, grad_stride, V, 0, 1.f, 1.f, 1.f, nullptr};
  return scores<true>("kf_op_token_scores_grad", type, R, a, tau, (cudaStream_t)stream);
}
