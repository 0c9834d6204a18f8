// Scores of tokens under rows of logits (kf_op_token_scores) and their
// gradient (kf_op_token_scores_grad).
//
// With x = logits / tau and m = max x, one pass over a row gives
//   S = sum exp(x - m),  T = sum (x - m) exp(x - m),
//   lse = m + log S,     entropy = log S - T / S
// (the sums against the maximum: no term cancels against another of its size).
// A thread keeps (m, S, T) of the 16-byte vectors it reads; two such triples
// join as S = S1 f1 + S2 f2, T = f1 (T1 + d1 S1) + f2 (T2 + d2 S2) with d = m_i - m
// and f = exp(d).  All of it is fp32.
//
// Top alternatives: the 512 threads of a row's CTA (CTAs) form 64 groups, and the
// n-th largest of the 64 groups' maxima is at or below the n-th largest logit (n
// groups have an element at or above it).  So only the threads whose own maximum
// reaches that bound read their vectors again (from L2) and list the elements at or
// above it, a few dozen of a vocabulary; each one's rank among them is its place.
// Rows where that list would not fit (ties in the hundreds) choose round by round.
//
// What bounds it: the logits' bytes, read once (scores) or read and written once (gradient:
// the second reading comes from L2).
#include <algorithm>
#include <cooperative_groups.h>

#include "kf_serving.cuh"

namespace cg = cooperative_groups;

namespace kf {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kGroups = 64;        // groups whose maxima bound the n-th largest logit
constexpr int kMaxTop = kGroups;
constexpr int kList = 1024;        // listed candidates of a row
constexpr int kRanked = 256;       // up to so many are ranked against each other, more are chosen in rounds
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLeast = -200.f;   // exp of it is 0 in fp32: stands for -inf where it multiplies that 0

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
  float inv_tau;
  int* err;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// exp with 2^x of the special-function unit: relative error about 2^-22 plus the
// rounding of the argument
__device__ __forceinline__ float exp_fast(float x) { return ex2(x * kLog2e); }
__device__ __forceinline__ uint4 ld_stream(const void* p) {
  uint4 u;
  asm("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
  return u;
}

// (m, S, T) of some elements; m = -inf: none of them is open (S and T are 0, or NaN)
struct Sums {
  float m, s, t;
};
__device__ __forceinline__ Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  Sums r{m, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const Sums c = i ? b : a;
    const float d = c.m == -INFINITY ? 0.f : fmaxf(c.m - m, kLeast), f = exp_fast(d);
    r.s += f * c.s;
    r.t += f * fmaf(d, c.s, c.t);
  }
  return r;
}

// one thread's pass over its elements
struct Pass {
  float raw = -INFINITY;   // the largest logit so far
  float nm = 0.f;          // minus the reference: -raw / tau (0 while that is infinite)
  float s = 0.f, t = 0.f;
  __device__ __forceinline__ float m(float inv_tau) const { return raw * inv_tau; }
  __device__ __forceinline__ void raise(float to, float inv_tau) {
    const float was = raw * inv_tau, m = to * inv_tau;
    if (was != -INFINITY) {
      const float d = fmaxf(was - m, kLeast), f = exp_fast(d);
      t = f * fmaf(d, s, t);
      s *= f;
    }
    raw = to;
    nm = m == -INFINITY ? 0.f : -m;
  }
  template <int N>
  __device__ __forceinline__ void add(const float* v, float inv_tau) {
    float top = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, v[i]);
    if (top > raw) raise(top, inv_tau);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = fmaf(v[i], inv_tau, nm), e = exp_fast(d);
      s += e;
      t = fmaf(e, fmaxf(d, kLeast), t);
    }
  }
};

// A row's elements in 16-byte vectors: `head` elements lie before the first
// aligned one, then nvec vectors, then `tail` elements
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

// f(id, x) for each element of thread `me` of `all` threads
template <typename T, typename F>
__device__ __forceinline__ void each_element(const Row<T>& row, int me, int all, F f) {
  for (int j = me; j < row.edge(); j += all) {
    const int id = row.edge_id(j);
    f(id, to_f(row.p[id]));
  }
  for (int i = me; i < row.nvec; i += all) {
    float v[Vec16<T>::N];
    Vec16<T>::unpack(*reinterpret_cast<const uint4*>(row.vec(i)), v);
    const int id0 = row.head + i * Vec16<T>::N;
#pragma unroll
    for (int e = 0; e < Vec16<T>::N; ++e) f(id0 + e, v[e]);
  }
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
  int count;
  Cand first[kWarps];
  Cand list[kList];
};

// Clusters of CS CTAs share a row (CS = 1: no cluster).  GRAD: the gradient's
// second pass instead of the alternatives.
template <typename T, int CS, bool GRAD>
__global__ void __launch_bounds__(kThreads, 2) k_scores(const Args a) {
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
        ps.add<N>(v, a.inv_tau);
      }
    }
    for (; i < row.nvec; i += kAll) {
      float v[N];
      Vec16<T>::unpack(ld_stream(row.vec(i)), v);
      ps.add<N>(v, a.inv_tau);
    }
    for (int j = me; j < row.edge(); j += kAll) {
      const float v = to_f(row.p[row.edge_id(j)]);
      ps.add<1>(&v, a.inv_tau);
    }
  }
  // the row's sums, in one fixed order
  Sums su{ps.m(a.inv_tau), ps.s, ps.t};
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const Sums other{__shfl_xor_sync(~0u, su.m, o), __shfl_xor_sync(~0u, su.s, o), __shfl_xor_sync(~0u, su.t, o)};
    su = (lane & o) ? join(other, su) : join(su, other);
  }
  if (lane == 0) sh.warp[warp] = su;
  if (!GRAD && a.top) {
    // the groups' maxima: 8 CS lanes each
    float gm = ps.raw;
#pragma unroll
    for (int o = 1; o < 8 * CS; o <<= 1) gm = fmaxf(gm, __shfl_xor_sync(~0u, gm, o));
    if (t % (8 * CS) == 0) sh.group[t / (8 * CS)] = gm;
    if (t == 0) sh.count = 0;
  }
  __syncthreads();
  su = sh.warp[lane % kWarps];
#pragma unroll
  for (int o = kWarps / 2; o; o >>= 1) {
    const Sums other{__shfl_xor_sync(~0u, su.m, o), __shfl_xor_sync(~0u, su.s, o), __shfl_xor_sync(~0u, su.t, o)};
    su = (lane & o) ? join(other, su) : join(su, other);
  }
  Shared* lead = &sh;
  if constexpr (CS > 1) {
    cg::cluster_group cl = cg::this_cluster();
    if (t == 0) sh.cta = su;
    cl.sync();
    su = cl.map_shared_rank(&sh, 0)->cta;
    for (int c = 1; c < CS; ++c) su = join(su, cl.map_shared_rank(&sh, c)->cta);
    lead = cl.map_shared_rank(&sh, 0);
    // every CTA has all groups' maxima
    const bool take = !GRAD && a.top && t < kGroups;
    float g = 0.f;
    if (take) g = cl.map_shared_rank(&sh, t / (kGroups / CS))->group[t % (kGroups / CS)];
    cl.sync();          // the other CTAs have read this one's part
    if (take) sh.group[t] = g;
    __syncthreads();
  }
  const bool none = su.m == -INFINITY && su.s == 0.f;     // every token closed
  const bool bad = !(su.s > 0.f) && !none;                // NaN or +inf in the row
  const float logs = logf(su.s);
  const float lse = none ? -INFINITY : bad ? NAN : su.m + logs;
  const float H = none ? 0.f : bad ? NAN : logs - su.t / su.s;
  if (rank == 0 && t == 0) {
    if (a.lse) a.lse[r] = lse;
    if (a.entropy) a.entropy[r] = H;
    if (token >= a.V) atomicOr(a.err, KF_DEV_BAD_TOKEN);
    if (a.logp)
      a.logp[r] = token < 0 ? 0.f : token >= a.V || bad ? NAN : none ? -INFINITY : (at_logit * a.inv_tau - su.m) - logs;
  }

  if constexpr (GRAD) {
    const bool has = token >= 0 && token < a.V;
    const float gl = has && a.g_logp ? a.g_logp[r] : 0.f, gh = a.g_entropy ? a.g_entropy[r] : 0.f;
    // grad = p (A + B lp) + (v == token) gl, over tau
    const float A = (-gl - gh * H) * a.inv_tau, B = -gh * a.inv_tau;
    const float at_token = gl * a.inv_tau;
    T* out = static_cast<T*>(a.grad) + r * a.grad_stride;
    auto one = [&](int id, float v) {
      const float lp = fmaxf(fmaf(v, a.inv_tau, -su.m) - logs, kLeast);
      float g = exp_fast(lp) * fmaf(B, lp, A);
      if (id == token) g += at_token;
      return none ? 0.f : bad ? NAN : g;
    };
    const bool same = (reinterpret_cast<uintptr_t>(out) & 15) == (reinterpret_cast<uintptr_t>(row.p) & 15);
    for (int j = me; j < row.edge(); j += kAll) {
      const int id = row.edge_id(j);
      out[id] = from_f<T>(one(id, to_f(row.p[id])));
    }
    int i = me;
    auto store = [&](int i, uint4 u) {
      float v[N];
      Vec16<T>::unpack(u, v);
      const int id0 = row.head + i * N;
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = one(id0 + e, v[e]);
      if (same) {
        *reinterpret_cast<uint4*>(out + id0) = Vec16<T>::pack(v);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) out[id0 + e] = from_f<T>(v[e]);
      }
    };
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
    for (int j = 0; j < kGroups; ++j) rk += sh.group[j] > g || (sh.group[j] == g && j < t);
    if (rk == a.top - 1) sh.bound = g * a.inv_tau;
  }
  __syncthreads();
  const float bound = sh.bound;
  // (a bound of -inf: the open tokens are listed, the closed ones follow by id)
  auto listed = [&](float x) { return x >= bound && x > -INFINITY; };
  if (listed(ps.raw * a.inv_tau))
    each_element(row, me, kAll, [&](int id, float v) {
      const float x = v * a.inv_tau;
      if (listed(x)) {
        const int at = atomicAdd(&lead->count, 1);
        if (at < kList) lead->list[at] = Cand{x, id};
      }
    });
  if constexpr (CS > 1) cg::this_cluster().sync();
  else __syncthreads();
  if (rank != 0) return;
  const int n = sh.count;
  auto put = [&](int place, Cand c) {
    ids[place] = c.id;
    lps[place] = (c.x - su.m) - logs;      // (lse itself loses log S where m is the type's lowest value)
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
      if (n <= kList)
        for (int j = t; j < n; j += kThreads) look(sh.list[j]);
      else
        each_element(row, t, kThreads, [&](int id, float v) {
          const float x = v * a.inv_tau;
          if (listed(x)) look(Cand{x, id});
        });
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
  const int cs = R * 4 <= sms && vecs >= 4 * 2 * kThreads ? 4 : R * 2 <= sms && vecs >= 2 * 2 * kThreads ? 2 : 1;
  const dim3 grid((unsigned)(R * cs));
  if (cs == 4) launch_cluster(k_scores<T, 4, GRAD>, grid, dim3(kThreads), 0, 4, false, s, a);
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
  Args a{logits, stride, tokens, nullptr, nullptr, logp, entropy, lse, top_logp, top_ids, nullptr, 0, V, top, 1.f, nullptr};
  return scores<false>("kf_op_token_scores", type, R, a, tau, (cudaStream_t)stream);
}

extern "C" int kf_op_token_scores_grad(int32_t type, int64_t R, int32_t V, const void* logits, int64_t stride,
                                       const int64_t* tokens, float tau, const float* g_logp,
                                       const float* g_entropy, float* logp, float* entropy, float* lse,
                                       void* grad, int64_t grad_stride, void* stream) {
  Args a{logits, stride, tokens, g_logp, g_entropy, logp, entropy, lse, nullptr, nullptr, grad, grad_stride, V, 0, 1.f, nullptr};
  return scores<true>("kf_op_token_scores_grad", type, R, a, tau, (cudaStream_t)stream);
}
