// Norms of query and key heads and their rotary positions (kf_op_rotate_heads), the same
// with K and V rows to the pages of a cache (kf_op_rotate_append), and the
// gradients (kf_op_rotate_heads_grad).
//
// A head x of hd elements: r = (mean x^2 + eps)^-1/2, y = x r w, and the pairs (y_i, y_i+n) (or
// (y_2i, y_2i+1)), i < n, turned by t = pos freq_i: (a cos t - b sin t, b cos t + a sin t).  Back: g = R^T dy,
//   dw = sum g xh,  dx = r (g w - xh mean(g w xh)),  xh = x r.
//
// Angles: freq_i / 2 pi turns as a fraction of 64 bits; times the position (mod 2^64) it leaves the
// fraction of a turn with an error of at most |pos| 2^-64 (2^-33 of a turn), where a product in fp32 would have lost the angle
// from positions of a few thousand on.  The nearest quarter turn comes off in whole numbers, so the
// sine and cosine are taken of |t| <= pi / 4.
//
// What bounds it: the heads, read and written once.  A warp's pass takes 4 or 8 heads of a token: hd / 16 lanes a head, two
// 16-byte vectors a lane, so that both elements of a pair are in one lane.  The passes of all tokens form one list that
// the warps share evenly.  Each lane streams its vectors through slots of shared memory that are its own (cp.async, a few
// passes ahead, across tokens; no thread waits for another's), so the loads under way do not
// cost registers; a token's angles are computed once by the warp's lanes and passed on through shared memory.
// Measured (GPU time, bf16): 16,411 tokens, 32 + 8 heads of 128, norms, in 58 us (5.8 TB/s; with the loads in registers, four
// passes ahead, 73); 24,361 tokens and V to pages, fp16, in 105 us (5.7 TB/s); eight rows of 256 sequences, 12 + 4 heads of 64, in 6.1 us
// (the chain of starts, slot, length and page: 7.5 a token at a time); the gradients of 16,384 tokens in 88 us (5.7 TB/s; 127 with the loads
// in registers, 92 with the weights read a pass); 8 tokens in 2.0 us.  Not kept: the weights multiplied into the turns (57 -> 61), tokens dealt out
// in turn instead of in stretches (57 -> 59, the gradients 85 -> 95).
#include <algorithm>
#include <climits>
#include <cstdlib>

#include "kf_mma.cuh"
#include "kf_serving.cuh"

namespace kf {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;      // of a CTA
// Slots of a warp: one in use, the others' loads under way (to pages, whose rows are written in no order, eight: 111 -> 104 us at
// the prompts above; rotation alone 57 with five, 60 with eight)
template <bool APPEND> constexpr int kAhead = APPEND ? 8 : 5;
constexpr int kBackAhead = 4;
constexpr int kJoinThreads = 256;

struct Rows {
  const void* p;
  int64_t row, head;
};
struct Out {
  void* p;
  int64_t row, head;
};
struct Book {
  const int32_t *which, *starts, *table, *lens;
  void* pool;
  int64_t n_pages;
  int n, page, slots, width;
  Div by_page;
};
struct Args {
  Rows q, k, v, dq, dk;          // v: append; dq, dk: gradient
  Out oq, ok;
  const void *wq, *wk;
  const int32_t* pos;
  const double* freq;
  float* part;                   // [CTAs][2][hd]: the weights' gradients
  Book book;
  int* err;
  int64_t T;
  int64_t each, more;            // passes of a warp; the first `more` warps have one more
  Div by_passes;                 // (below 2^31 passes; else divided in 64 bits)
  int Hq, Hkv, n, passes, warps; // n: pairs; passes: of a token; warps: that have passes
  float eps, sign;               // eps < 0: no norms; sign: -1 turns back
};

// freq / 2 pi mod 1 as a fraction of 64 bits: the mantissa times 2^130 / 2 pi (two words; of one alone a far position of a large frequency
// would keep little: 1.1e-2 at 2^31 and 4e9), shifted; at most 1 of its last place too small.  NaN, infinities and |freq| >= 2^32: *bad
__device__ __forceinline__ uint64_t turns_of(double freq, bool* bad) {
  constexpr uint64_t k = 11743562013128004905ull, k_low = 18169587780923219392ull;      // 2^130 / 2 pi
  const uint64_t u = (uint64_t)__double_as_longlong(freq);
  const int e = (int)(u >> 52) & 0x7ff;
  const uint64_t m = (u & 0xfffffffffffffull) | (e ? 1ull << 52 : 0ull);
  *bad = e >= 1023 + 32;
  // m 2^(e - 1075) / 2 pi 2^64 = (m k) 2^(e - 1077): to the right by 23 and more
  const uint64_t lo = m * k + __umul64hi(m, k_low), hi = __umul64hi(m, k) + (lo < m * k);
  const int s = *bad ? 127 : 1077 - max(e, 1);
  uint64_t t;
  if (s < 64) t = (hi << (64 - s)) | (lo >> s);
  else t = s < 128 ? hi >> (s - 64) : 0ull;
  return (u >> 63) ? 0ull - t : t;
}
// (cos, sin) of pos times these turns
__device__ __forceinline__ float2 turn(int pos, uint64_t turns, bool bad) {
  const uint64_t a = (uint64_t)(int64_t)pos * turns;
  const int q = (int)(((a >> 61) + 1) >> 1);                     // the nearest quarter turn (0 .. 4)
  const int64_t rest = (int64_t)(a - ((uint64_t)q << 62));       // at most 2^61 away
  float s, c;
  sincospif((float)rest * 0x1p-63f, &s, &c);
  if (q & 1) {
    const float x = c;
    c = -s;
    s = x;
  }
  if (q & 2) {
    c = -c;
    s = -s;
  }
  return bad ? make_float2(NAN, NAN) : make_float2(c, s);
}

// Where a lane's two vectors lie in a head, the first of its angles, and which of its pairs are turned at all (an angle of 0 would
// not leave the others as they are: 0 times an infinity is no number)
template <int HD, bool NB>
struct Place {
  static constexpr int LANES = HD / 16, PER = 32 / LANES;
  int c0, c1, a0;                // vectors; angle (NB: of the first vector, the second's are HD / 4 on)
  bool on[2];                    // the first and the last four of its pairs
  __device__ __forceinline__ Place(int lane, int n) {
    const int l = lane % LANES, n8 = n / 8;
    if (NB) {
      c0 = l;
      c1 = l + LANES;
      a0 = 4 * l;
      on[0] = a0 < n;
      on[1] = HD / 4 + a0 < n;
    } else {
      on[0] = on[1] = l < n8;
      c0 = on[0] ? l : 2 * n8 + (l - n8);
      c1 = c0 + (on[0] ? n8 : (HD - 16 * n8) / 16);
      a0 = on[0] ? 8 * l : 0;
    }
  }
};

// A token's angles to the warp's table: cosine and sine of each pair that is turned
template <int HD>
__device__ __forceinline__ void fill_table(const Args& a, float2* tab, int pos, int lane) {
  __syncwarp();                  // (the token before is through with it)
#pragma unroll
  for (int i = lane; i < HD / 2; i += 32)
    if (i < a.n) {
      bool bad;
      const uint64_t t = turns_of(__ldg(a.freq + i), &bad);
      float2 v = turn(pos, t, bad);
      v.y *= a.sign;
      tab[i] = v;
    }
  __syncwarp();
}
// The 8 pairs of a lane
template <int HD, bool NB>
struct Angles {
  float c[8], s[8];
  __device__ __forceinline__ void take(const float2* tab, const Place<HD, NB>& pl) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const int i = NB ? pl.a0 + (e < 4 ? e : HD / 4 + e - 4) : pl.a0 + e;
      const float4 v = *reinterpret_cast<const float4*>(tab + i);      // (of a pair that is not turned: anything)
      c[e] = v.x;
      s[e] = v.y;
      c[e + 1] = v.z;
      s[e + 1] = v.w;
    }
  }
  // x: the lane's 16 elements of a head
  static constexpr __device__ __forceinline__ int first(int e) { return NB ? 2 * e : e; }
  static constexpr __device__ __forceinline__ int second(int e) { return NB ? 2 * e + 1 : e + 8; }
  __device__ __forceinline__ void turn_pairs(float* x, int from, int to) const {
#pragma unroll
    for (int e = from; e < to; ++e) {
      float &a = x[first(e)], &b = x[second(e)];
      const float y = fmaf(a, c[e], -b * s[e]);
      b = fmaf(b, c[e], a * s[e]);
      a = y;
    }
  }
  __device__ __forceinline__ void turn_head(float* x, const Place<HD, NB>& pl) const {
    if constexpr (NB) {
      if (pl.on[0]) turn_pairs(x, 0, 4);
      if (pl.on[1]) turn_pairs(x, 4, 8);
    } else {
      if (pl.on[0]) turn_pairs(x, 0, 8);
    }
  }
};
template <int LANES> __device__ __forceinline__ float sum_head(float v) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}
template <typename T> __device__ __forceinline__ void unpack16(const uint4* u, float* x) {
  Vec16<T>::unpack(u[0], x);
  Vec16<T>::unpack(u[1], x + 8);
}

// The places of a warp's tokens in their sequences' caches, looked up 32 at a time: lane i holds that of token base + i, so the
// chain of loads (starts, slot, length, page) is waited for once
struct Places {
  int64_t base;
  int pos;                       // -1: not known
  int64_t row;                   // K's row of head 0 in the pool, in rows of hd; -1: not to be written
  // tokens t .. t + n - 1 (n <= 32); `flags`: the first of them is this warp's to report
  __device__ __forceinline__ void look(const Book& k, int Hkv, int64_t t, int n, bool flags, int lane, int* err) {
    base = t;
    pos = -1;
    row = -1;
    // the last sequence that starts at or before a lane's token
    int lo = 0;
    if (k.n <= 256) {
      int start[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) start[i] = 32 * i + lane < k.n ? __ldg(k.starts + 32 * i + lane) : INT_MAX;
#pragma unroll 1
      for (int x = 0; x < n; ++x) {
        int below = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) below += start[i] <= t + x;
        below = __reduce_add_sync(~0u, below);
        if (x == lane) lo = max(0, below - 1);
      }
    } else if (lane < n) {
      for (int hi = k.n - 1; lo < hi;) {
        const int mid = (lo + hi + 1) >> 1;
        if (__ldg(k.starts + mid) <= t + lane) lo = mid;
        else hi = mid - 1;
      }
    }
    if (lane >= n) return;
    const int first = __ldg(k.starts + lo), end = __ldg(k.starts + lo + 1), s = __ldg(k.which + lo);
    int bad = 0;
    if (t + lane < first || t + lane >= end || s < 0 || s >= k.slots) bad = KF_DEV_BAD_ROW;
    else {
      const int64_t p = (int64_t)k.lens[s] - end + t + lane;
      if (p < 0 || p >= (int64_t)k.width * k.page) bad = KF_DEV_BAD_ROW;
      else {
        pos = (int)p;
        const int col = k.by_page.of(pos), id = k.table[(int64_t)s * k.width + col];
        if (id < 0 || id >= k.n_pages) bad = KF_DEV_BAD_PAGE;
        else row = (int64_t)id * 2 * Hkv * k.page + (pos - col * k.page);
      }
    }
    if (bad && (flags || lane > 0)) atomicOr(err, bad);
  }
};

// A warp's passes, first .. last - 1 of the list; pass x is pass x % passes of token x / passes
struct Range {
  int64_t t;
  int p, left;                   // the token and pass that come next; how many are left
  __device__ __forceinline__ Range(const Args& a, int w) {
    const int64_t first = w * a.each + min((int64_t)w, a.more);
    left = w < a.warps ? (int)(a.each + (w < a.more)) : 0;
    t = first < 0x7fffffff ? a.by_passes.of((int)first) : first / a.passes;
    p = (int)(first - t * a.passes);
  }
  __device__ __forceinline__ void next(const Args& a) {
    --left;
    if (++p == a.passes) {
      p = 0;
      ++t;
    }
  }
};

template <typename T, int HD, bool NB, bool APPEND>
__global__ void __launch_bounds__(kThreads, 6) k_rotate(const __grid_constant__ Args a) {
  __shared__ __align__(16) float2 tab[kWarps][HD / 2];
  constexpr int AHEAD = kAhead<APPEND>;
  __shared__ uint4 slots[kWarps][AHEAD][2][32];
  constexpr int LANES = HD / 16, PER = 32 / LANES;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = lane / LANES;
  Range now(a, blockIdx.x * kWarps + warp), ahead = now;
  if (now.left == 0) return;
  const int heads = a.Hq + a.Hkv * (APPEND ? 2 : 1);
  const Place<HD, NB> pl(lane, a.n);
  const uint32_t slot0 = mma::smem_addr(&slots[warp][0][0][lane]);
  int fslot = 0;
  auto fill = [&] {              // one group of copies, empty past the last pass
    const int j = ahead.p * PER + grp;
    if (ahead.left > 0 && j < heads) {
      const bool is_q = j < a.Hq, is_v = APPEND && j >= a.Hq + a.Hkv;
      const Rows& r = is_q ? a.q : is_v ? a.v : a.k;
      const T* x = static_cast<const T*>(r.p) + ahead.t * r.row + (j - (is_q ? 0 : is_v ? a.Hq + a.Hkv : a.Hq)) * r.head;
      mma::cp_async16(slot0 + fslot * 1024, x + 8 * pl.c0, 16);
      mma::cp_async16(slot0 + fslot * 1024 + 512, x + 8 * pl.c1, 16);
    }
    mma::cp_commit();
    if (ahead.left > 0) ahead.next(a);
    fslot = fslot + 1 == AHEAD ? 0 : fslot + 1;
  };
#pragma unroll 1
  for (int i = 0; i < AHEAD - 1; ++i) fill();
  Angles<HD, NB> an;
  Places places;
  places.base = -32;
  int pos = 0;
  int64_t row = -1, token = -1;
  int slot = 0;
#pragma unroll 1
  for (; now.left > 0; now.next(a)) {
    const int64_t t = now.t;
    const int j = now.p * PER + grp;
    const bool is_q = j < a.Hq, is_v = APPEND && j >= a.Hq + a.Hkv;
    if (t != token) {            // (uniform)
      token = t;
      if constexpr (APPEND) {
        if (t >= places.base + 32) {
          const int tokens = a.by_passes.of(min(now.p + now.left - 1, INT_MAX - 1)) + 1;      // of this warp, from t on
          places.look(a.book, a.Hkv, t, min(tokens, 32), now.p == 0, lane, a.err);
        }
        pos = __shfl_sync(~0u, places.pos, (int)(t - places.base));
        row = __shfl_sync(~0u, places.row, (int)(t - places.base));
      } else {
        pos = __ldg(a.pos + t);
      }
      fill_table<HD>(a, tab[warp], pos, lane);
      an.take(tab[warp], pl);
    }
    mma::cp_wait<AHEAD - 2>();
    fill();                      // into the slot of the pass before
    uint4 o[2] = {slots[warp][slot][0][lane], slots[warp][slot][1][lane]};
    slot = slot + 1 == AHEAD ? 0 : slot + 1;
    float x[16];
    unpack16<T>(o, x);
    if (a.eps >= 0.f) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
      const float r = rsqrtf(fmaf(sum_head<LANES>(ss), 1.f / HD, a.eps));
      const uint4* w = static_cast<const uint4*>(is_q ? a.wq : a.wk);
      if (w) {
        float g[16];
        const uint4 gw[2] = {__ldg(w + pl.c0), __ldg(w + pl.c1)};
        unpack16<T>(gw, g);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] *= r * g[e];
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] *= r;
      }
    }
    an.turn_head(x, pl);
    if (!is_v) {
      o[0] = Vec16<T>::pack(x);
      o[1] = Vec16<T>::pack(x + 8);
    }
    if (j >= heads) continue;
    T* to;
    if (is_q) {
      to = static_cast<T*>(a.oq.p) + t * a.oq.row + j * a.oq.head;
      if (APPEND && pos < 0) o[0] = o[1] = make_uint4(0u, 0u, 0u, 0u);
    } else if (APPEND) {
      // (V's heads follow K's in a page)
      if (row < 0) continue;
      to = static_cast<T*>(a.book.pool) + (row + (int64_t)(j - a.Hq) * a.book.page) * HD;
    } else {
      to = static_cast<T*>(a.ok.p) + t * a.ok.row + (j - a.Hq) * a.ok.head;
    }
    *reinterpret_cast<uint4*>(to + 8 * pl.c0) = o[0];
    *reinterpret_cast<uint4*>(to + 8 * pl.c1) = o[1];
  }
  mma::cp_wait<0>();
}

// Gradients: a token's passes over its query heads, then over its key heads; a warp keeps the
// weights' sums in registers, each CTA leaves its own, which k_join adds in one fixed order.
template <typename T, int HD, bool NB>
__global__ void __launch_bounds__(kThreads, 3) k_back(const __grid_constant__ Args a) {
  __shared__ __align__(16) float2 tab[kWarps][HD / 2];
  __shared__ float sums[kWarps][2][HD];
  __shared__ uint4 slots[kWarps][kBackAhead][4][32];
  constexpr int LANES = HD / 16, PER = 32 / LANES;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = lane / LANES, q_passes = (a.Hq + PER - 1) / PER;
  const Place<HD, NB> pl(lane, a.n);
  float acc[2][16];
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[0][e] = acc[1][e] = 0.f;
  Range now(a, blockIdx.x * kWarps + warp), ahead = now;
  const uint32_t slot0 = mma::smem_addr(&slots[warp][0][0][lane]);
  int fslot = 0;
  auto fill = [&] {
    const bool k = ahead.p >= q_passes;
    const int j = (k ? ahead.p - q_passes : ahead.p) * PER + grp;
    if (ahead.left > 0 && j < (k ? a.Hkv : a.Hq)) {
      const Rows &rx = k ? a.k : a.q, &rd = k ? a.dk : a.dq;
      const T* x = static_cast<const T*>(rx.p) + ahead.t * rx.row + j * rx.head;
      const T* d = static_cast<const T*>(rd.p) + ahead.t * rd.row + j * rd.head;
      mma::cp_async16(slot0 + fslot * 2048, x + 8 * pl.c0, 16);
      mma::cp_async16(slot0 + fslot * 2048 + 512, x + 8 * pl.c1, 16);
      mma::cp_async16(slot0 + fslot * 2048 + 1024, d + 8 * pl.c0, 16);
      mma::cp_async16(slot0 + fslot * 2048 + 1536, d + 8 * pl.c1, 16);
    }
    mma::cp_commit();
    if (ahead.left > 0) ahead.next(a);
    fslot = fslot + 1 == kBackAhead ? 0 : fslot + 1;
  };
#pragma unroll 1
  for (int i = 0; i < kBackAhead - 1; ++i) fill();
  Angles<HD, NB> an;
  float g[16];                   // the weights, of the query or the key heads (`held`)
  int64_t token = -1;
  int slot = 0, held = -1;
#pragma unroll 1
  for (; now.left > 0; now.next(a)) {
    const int64_t t = now.t;
    const bool k = now.p >= q_passes;
    const int j = (k ? now.p - q_passes : now.p) * PER + grp;
    const bool has = j < (k ? a.Hkv : a.Hq);
    if (t != token) {            // (uniform)
      token = t;
      fill_table<HD>(a, tab[warp], __ldg(a.pos + t), lane);
      an.take(tab[warp], pl);
    }
    if (held != (int)k) {        // (uniform)
      held = k;
#pragma unroll
      for (int e = 0; e < 16; ++e) g[e] = 1.f;
      if (const uint4* w = static_cast<const uint4*>(k ? a.wk : a.wq)) {
        const uint4 gw[2] = {__ldg(w + pl.c0), __ldg(w + pl.c1)};
        unpack16<T>(gw, g);
      }
    }
    mma::cp_wait<kBackAhead - 2>();
    fill();                      // into the slot of the pass before
    const uint4 ux[2] = {slots[warp][slot][0][lane], slots[warp][slot][1][lane]}, ud[2] = {slots[warp][slot][2][lane], slots[warp][slot][3][lane]};
    slot = slot + 1 == kBackAhead ? 0 : slot + 1;
    float x[16], d[16];
    unpack16<T>(ux, x);
    unpack16<T>(ud, d);
    an.turn_head(d, pl);
    float ss = 0.f, sg = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      ss = fmaf(x[e], x[e], ss);
      sg = fmaf(d[e] * g[e], x[e], sg);
    }
    const float r = rsqrtf(fmaf(sum_head<LANES>(ss), 1.f / HD, a.eps));
    const float m = sum_head<LANES>(sg) * (1.f / HD) * r * r;
    if (!has) continue;          // (lanes of heads that are not there hold anything)
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] *= r;
    if (a.part && !k) {          // (uniform)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[0][e] = fmaf(d[e], x[e], acc[0][e]);
    } else if (a.part) {
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[1][e] = fmaf(d[e], x[e], acc[1][e]);
    }
    // r g w - xh r mean(g w xh)
#pragma unroll
    for (int e = 0; e < 16; ++e) d[e] = fmaf(r * g[e], d[e], -m * x[e]);
    const Out& O = k ? a.ok : a.oq;
    T* to = static_cast<T*>(O.p) + t * O.row + j * O.head;
    *reinterpret_cast<uint4*>(to + 8 * pl.c0) = Vec16<T>::pack(d);
    *reinterpret_cast<uint4*>(to + 8 * pl.c1) = Vec16<T>::pack(d + 8);
  }
  mma::cp_wait<0>();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (!a.part) return;
#pragma unroll
  for (int part = 0; part < 2; ++part)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float v = acc[part][e];
#pragma unroll
      for (int o = LANES; o < 32; o <<= 1) v += __shfl_xor_sync(~0u, v, o);
      if (grp == 0) sums[warp][part][8 * (e < 8 ? pl.c0 : pl.c1) + (e & 7)] = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * HD; i += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int x = 0; x < kWarps; ++x) v += sums[x][i / HD][i % HD];
    a.part[(int64_t)blockIdx.x * 2 * HD + i] = v;
  }
}
// Block b: columns 8 b .. 8 b + 7 of the weights' gradients, the CTAs' parts added in fixed order
template <int HD>
__global__ void __launch_bounds__(kJoinThreads) k_join(const float* part, int ctas, float* dwq, float* dwk) {
  __shared__ float s[kJoinThreads / 8][8];
  const int c = threadIdx.x % 8, y = threadIdx.x / 8, col = blockIdx.x * 8 + c;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float v = 0.f;
#pragma unroll 8
  for (int i = y; i < ctas; i += kJoinThreads / 8) v += __ldcg(part + (int64_t)i * 2 * HD + col);
  s[y][c] = v;
  __syncthreads();
#pragma unroll
  for (int o = kJoinThreads / 16; o; o >>= 1) {
    if (y < o) s[y][c] += s[y + o][c];
    __syncthreads();
  }
  float* to = col < HD ? dwq : dwk;
  if (y == 0 && to) to[col % HD] = s[0][c];
}

// ------------------------------------------------------------------ host
// The list of T tokens' passes over as many warps as the SMs hold at once
void share(Args& a, int passes, int ctas_per_sm) {
  const int64_t total = a.T * passes;
  a.passes = passes;
  a.by_passes = Div(passes);
  a.warps = (int)std::min<int64_t>(total, (int64_t)device_sms() * ctas_per_sm * kWarps);
  a.each = total / a.warps;
  a.more = total % a.warps;
}
template <typename T, int HD, bool NB, bool APPEND>
void launch_rotate(Args a, cudaStream_t s) {
  share(a, ceil_div(a.Hq + a.Hkv * (APPEND ? 2 : 1), 32 / (HD / 16)), 6);
  launch_cluster(k_rotate<T, HD, NB, APPEND>, dim3(ceil_div(a.warps, kWarps)), dim3(kThreads), 0, 1, false, s, a);
}
void share_back(Args& a, int hd) {
  const int per = 32 / (hd / 16);
  share(a, ceil_div(a.Hq, per) + ceil_div(a.Hkv, per), 3);
}
template <typename T, int HD, bool NB>
void launch_back(Args a, float* dwq, float* dwk, cudaStream_t s) {
  share_back(a, HD);
  const int grid = ceil_div(a.warps, kWarps);
  launch_cluster(k_back<T, HD, NB>, dim3(grid), dim3(kThreads), 0, 1, false, s, a);
  if (a.part) launch_cluster(k_join<HD>, dim3(2 * HD / 8), dim3(kJoinThreads), 0, 1, true, s, (const float*)a.part, grid, dwq, dwk);
}
template <bool APPEND>
void rotate_any(int type, int hd, bool nb, const Args& a, cudaStream_t s) {
  auto by_type = [&](auto x) {
    using T = decltype(x);
    if (hd == 64) nb ? launch_rotate<T, 64, true, APPEND>(a, s) : launch_rotate<T, 64, false, APPEND>(a, s);
    else nb ? launch_rotate<T, 128, true, APPEND>(a, s) : launch_rotate<T, 128, false, APPEND>(a, s);
  };
  if (type == KF_TYPE_BF16) by_type(__nv_bfloat16{});
  else by_type(__half{});
}
void back_any(int type, int hd, bool nb, const Args& a, float* dwq, float* dwk, cudaStream_t s) {
  auto by_type = [&](auto x) {
    using T = decltype(x);
    if (hd == 64) nb ? launch_back<T, 64, true>(a, dwq, dwk, s) : launch_back<T, 64, false>(a, dwq, dwk, s);
    else nb ? launch_back<T, 128, true>(a, dwq, dwk, s) : launch_back<T, 128, false>(a, dwq, dwk, s);
  };
  if (type == KF_TYPE_BF16) by_type(__nv_bfloat16{});
  else by_type(__half{});
}

// what all three entries ask for; nullptr if it is fine
const char* fault(int32_t type, int64_t T, int32_t Hq, int32_t Hkv, int32_t hd, const double* freq, int32_t n_freq, float eps,
                  const void* wq, const void* wk) {
  if (type != KF_TYPE_BF16 && type != KF_TYPE_FP16) return "the type is bf16 or fp16";
  if (hd != 64 && hd != 128) return "head_dim is 64 or 128";
  if (T < 0 || T > 0x7fffffffll || Hq < 1 || Hkv < 1 || Hq > 4096 || Hkv > 4096) return "tokens or heads out of range";
  if (n_freq < 0 || n_freq % 8 || 2 * n_freq > hd) return "frequencies: a multiple of 8, at most head_dim / 2";
  if (!(eps < 0.f) && !(eps >= 0.f && !std::isinf(eps))) return "eps is a finite number (negative: no norms)";
  if (eps < 0.f && (wq || wk)) return "weights belong to norms (eps is negative)";
  if (n_freq && (!freq || !aligned(freq, 8))) return "frequencies: null or misaligned";
  if (!aligned(wq, 16) || !aligned(wk, 16)) return "weights are 16-byte aligned";
  return nullptr;
}
// one array of heads
const char* rows_fault(const void* p, int64_t row, int64_t head) {
  if (!p) return "a null array";
  if (!aligned(p, 16)) return "arrays of heads are 16-byte aligned";
  for (const int64_t s : {row, head})
    if (s % 8 || s < 0 || s > (1ll << 37)) return "strides are multiples of 8 elements";
  return nullptr;
}
// whether two of an output's heads share an element: |x row - y head| < hd for some x < T and y < H that are not both 0
bool heads_meet(int64_t T, int64_t H, int64_t row, int64_t head, int64_t hd) {
  if ((T > 1 && row < hd) || (H > 1 && head < hd)) return true;
  if (T == 1 || row >= (H - 1) * head + hd) return false;
  for (int64_t y = 1; y < H; ++y)
    for (const int64_t x : {y * head / row, y * head / row + 1})
      if (x < T && std::abs(x * row - y * head) < hd) return true;
  return false;
}

}  // namespace
}  // namespace kf

using namespace kf;

extern "C" int kf_op_rotate_heads(int32_t type, int64_t T, int32_t Hq, int32_t Hkv, int32_t hd, const void* q, int64_t q_row,
                                  int64_t q_head, const void* k, int64_t k_row, int64_t k_head, const int32_t* pos,
                                  const double* freq, int32_t n_freq, int32_t neighbours, float eps, const void* q_weight,
                                  const void* k_weight, void* q_out, int64_t q_out_row, int64_t q_out_head, void* k_out,
                                  int64_t k_out_row, int64_t k_out_head, void* stream) {
  const char* what = "kf_op_rotate_heads";
  if (const char* f = fault(type, T, Hq, Hkv, hd, freq, n_freq, eps, q_weight, k_weight)) return refuse(what, f);
  if (T == 0) return KF_OK;
  if (const char* f = rows_fault(q, q_row, q_head)) return refuse(what, f);
  if (const char* f = rows_fault(k, k_row, k_head)) return refuse(what, f);
  if (const char* f = rows_fault(q_out, q_out_row, q_out_head)) return refuse(what, f);
  if (const char* f = rows_fault(k_out, k_out_row, k_out_head)) return refuse(what, f);
  if (!pos || !aligned(pos, 4)) return refuse(what, "positions: null or misaligned");
  if (heads_meet(T, Hq, q_out_row, q_out_head, hd) || heads_meet(T, Hkv, k_out_row, k_out_head, hd))
    return refuse(what, "an output's heads lie over each other");
  if (q_out == k_out && !(q_out == q && k_out == k)) return refuse(what, "q_out and k_out are one array");
  if ((q_out == q && (q_out_row != q_row || q_out_head != q_head)) || (k_out == k && (k_out_row != k_row || k_out_head != k_head)))
    return refuse(what, "an output over its input has its strides");
  Args a{};
  a.q = Rows{q, q_row, q_head};
  a.k = Rows{k, k_row, k_head};
  a.oq = Out{q_out, q_out_row, q_out_head};
  a.ok = Out{k_out, k_out_row, k_out_head};
  a.wq = q_weight;
  a.wk = k_weight;
  a.pos = pos;
  a.freq = freq;
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.n = n_freq;
  a.eps = eps;
  a.sign = 1.f;
  rotate_any<false>(type, hd, neighbours != 0, a, (cudaStream_t)stream);
  return launched(what);
}

extern "C" int kf_op_rotate_append(int32_t type, int32_t n, const int32_t* which, const int32_t* starts, int64_t T, int32_t Hq,
                                   int32_t Hkv, int32_t hd, const void* q, int64_t q_row, int64_t q_head, const void* k,
                                   int64_t k_row, int64_t k_head, const void* v, int64_t v_row, int64_t v_head,
                                   const double* freq, int32_t n_freq, int32_t neighbours, float eps, const void* q_weight,
                                   const void* k_weight, void* q_out, void* pool, int32_t n_pages, int32_t page,
                                   const int32_t* table, int32_t slots, int32_t width, const int32_t* lens, void* stream) {
  const char* what = "kf_op_rotate_append";
  if (const char* f = fault(type, T, Hq, Hkv, hd, freq, n_freq, eps, q_weight, k_weight)) return refuse(what, f);
  if (n < 0 || n_pages < 1 || slots < 1 || width < 0) return refuse(what, "sequences, pages, slots or width out of range");
  if (page < 1 || page > (1 << 20) || (int64_t)width * page > 0x7fffffffll) return refuse(what, "page, or width * page, out of range");
  if (T == 0) return KF_OK;
  if (n == 0) return refuse(what, "tokens of no sequence");
  if (!which || !starts || !pool || !lens || (width && !table)) return refuse(what, "a null array");
  if (const char* f = rows_fault(q, q_row, q_head)) return refuse(what, f);
  if (const char* f = rows_fault(k, k_row, k_head)) return refuse(what, f);
  if (const char* f = rows_fault(v, v_row, v_head)) return refuse(what, f);
  if (const char* f = rows_fault(q_out, (int64_t)Hq * hd, hd)) return refuse(what, f);
  if (!aligned(pool, 16) || !aligned(which, 4) || !aligned(starts, 4) || !aligned(table, 4) || !aligned(lens, 4))
    return refuse(what, "the pool is 16-byte aligned, the book's lists 4-byte");
  Args a{};
  a.q = Rows{q, q_row, q_head};
  a.k = Rows{k, k_row, k_head};
  a.v = Rows{v, v_row, v_head};
  a.oq = Out{q_out, (int64_t)Hq * hd, hd};
  a.wq = q_weight;
  a.wk = k_weight;
  a.freq = freq;
  a.book = Book{which, starts, table, lens, pool, n_pages, n, page, slots, width, Div(page)};
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.n = n_freq;
  a.eps = eps;
  a.sign = 1.f;
  if (!(a.err = serving_error_word())) return refuse(what, "no error word", KF_E_CUDA);
  rotate_any<true>(type, hd, neighbours != 0, a, (cudaStream_t)stream);
  return launched(what);
}

extern "C" int64_t kf_op_rotate_heads_grad_work(int64_t T, int32_t Hq, int32_t Hkv, int32_t hd) {
  if (T < 1 || Hq < 1 || Hkv < 1 || (hd != 64 && hd != 128)) return 0;
  Args a{};
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  share_back(a, hd);
  return (int64_t)ceil_div(a.warps, kWarps) * 2 * hd * (int64_t)sizeof(float);
}

extern "C" int kf_op_rotate_heads_grad(int32_t type, int64_t T, int32_t Hq, int32_t Hkv, int32_t hd, const void* dq, int64_t dq_row,
                                       int64_t dq_head, const void* dk, int64_t dk_row, int64_t dk_head, const void* q,
                                       int64_t q_row, int64_t q_head, const void* k, int64_t k_row, int64_t k_head,
                                       const int32_t* pos, const double* freq, int32_t n_freq, int32_t neighbours, float eps,
                                       const void* q_weight, const void* k_weight, void* q_grad, void* k_grad,
                                       float* q_weight_grad, float* k_weight_grad, void* work, void* stream) {
  const char* what = "kf_op_rotate_heads_grad";
  if (const char* f = fault(type, T, Hq, Hkv, hd, freq, n_freq, eps, q_weight, k_weight)) return refuse(what, f);
  const bool norm = !(eps < 0.f);
  if ((q_weight_grad && !q_weight) || (k_weight_grad && !k_weight)) return refuse(what, "a weight's gradient wants the weight");
  if (!aligned(q_weight_grad, 4) || !aligned(k_weight_grad, 4)) return refuse(what, "a weight's gradient is misaligned");
  cudaStream_t s = (cudaStream_t)stream;
  if (T == 0) {
    for (float* g : {q_weight_grad, k_weight_grad})
      if (g && cudaMemsetAsync(g, 0, hd * sizeof(float), s) != cudaSuccess) return launched(what);
    return KF_OK;
  }
  if (const char* f = rows_fault(dq, dq_row, dq_head)) return refuse(what, f);
  if (const char* f = rows_fault(dk, dk_row, dk_head)) return refuse(what, f);
  if (norm)
    if (const char* f = rows_fault(q, q_row, q_head)) return refuse(what, f);
  if (norm)
    if (const char* f = rows_fault(k, k_row, k_head)) return refuse(what, f);
  if (const char* f = rows_fault(q_grad, (int64_t)Hq * hd, hd)) return refuse(what, f);
  if (const char* f = rows_fault(k_grad, (int64_t)Hkv * hd, hd)) return refuse(what, f);
  if (!pos || !aligned(pos, 4)) return refuse(what, "positions: null or misaligned");
  const bool weights = q_weight_grad || k_weight_grad;
  if (weights && (!work || !aligned(work, 256))) return refuse(what, "work is 256-byte aligned");
  Args a{};
  a.oq = Out{q_grad, (int64_t)Hq * hd, hd};
  a.ok = Out{k_grad, (int64_t)Hkv * hd, hd};
  a.pos = pos;
  a.freq = freq;
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.n = n_freq;
  a.eps = eps;
  a.sign = -1.f;
  if (!norm) {
    // the gradient of a rotation is the rotation back
    a.q = Rows{dq, dq_row, dq_head};
    a.k = Rows{dk, dk_row, dk_head};
    rotate_any<false>(type, hd, neighbours != 0, a, s);
    return launched(what);
  }
  a.q = Rows{q, q_row, q_head};
  a.k = Rows{k, k_row, k_head};
  a.dq = Rows{dq, dq_row, dq_head};
  a.dk = Rows{dk, dk_row, dk_head};
  a.wq = q_weight;
  a.wk = k_weight;
  a.part = weights ? static_cast<float*>(work) : nullptr;
  back_any(type, hd, neighbours != 0, a, q_weight_grad, k_weight_grad, s);
  return launched(what);
}
