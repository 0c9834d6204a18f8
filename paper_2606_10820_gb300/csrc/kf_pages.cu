// The pages of a paged cache: room, fork, free, compact, copy and append
// (kf_op_pages_*).
//
// The book (references of each page, page table, lengths) lives on the device, so
// that a scheduler's calls need no readback and can be captured.  One team of 1024 threads,
// or of a cluster of 8 x 1024 where the book is large, does a call's whole bookkeeping in one
// launch: it checks everything first and writes only when all of it can be
// done.  Free pages are found by counting: each warp holds its stretch of the
// references as ballots, the counts before it give the rank of its first one, so
// the i-th lowest free page goes to the i-th request whatever the team's size.  What
// bounds a call is its barriers and the loads between them (two or three of each).
// Page contents are moved by a second, dependent launch over all SMs that
// reads the list of moves (its bound: HBM, each moved byte read and written once).
// Measured: k_move 1.05 GB (read and written) in 159 us (6.6 TB/s); the bookkeeping of a compact of 16,384
// pages and 32,768 entries 16 us, of 1,024 pages 6; grow of 64 prompts of 1,000 tokens 8 us, of 512 sequences by a
// token 14; k_append 0.53 GB in 84 us (6.3 TB/s).
#include <algorithm>
#include <cooperative_groups.h>

#include "kf_serving.cuh"

namespace cg = cooperative_groups;

namespace kf {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kTeam = 8;                  // CTAs of a large book's team
constexpr int kCopyThreads = 256, kCopyUnit = kCopyThreads * 4 * 16;   // bytes that a CTA copies at a time

struct Book {
  int32_t *ref, *table, *lens;
  int n_pages, slots, width, page;
};
// the scratch of a call: a stamp per slot, an offset per request, lists of
// pages, and where a moved page went
struct Work {
  int32_t *count, *mark, *off, *src, *dst, *to;
};

constexpr int kCached = 8;                // ballots of 32 pages that a warp keeps

// What the team's warps tell each other at a barrier; two of them in turn, so that one
// is not written before everybody has read it
struct Exchange {
  int flag[kWarps], a[kWarps], b[kWarps];
};
struct Shared {
  Exchange x[2];
  int scan[kWarps], total;
};

template <int C>
struct Team {
  Shared& sh;
  int t, lane, warp, rank, id, turn;
  uint32_t live[kCached], none[kCached];   // this warp's pages with references, and without
  int lo, hi;                              // its stretch
  bool cached;
  __device__ __forceinline__ explicit Team(Shared& s) : sh(s) {
    t = threadIdx.x;
    lane = t & 31;
    warp = t >> 5;
    rank = C > 1 ? blockIdx.x : 0;
    id = rank * kThreads + t;
    turn = 0;
  }
  static constexpr int size = C * kThreads;
  __device__ __forceinline__ void sync() const {
    if constexpr (C > 1) cg::this_cluster().sync();
    else __syncthreads();
  }
  // before a CTA leaves: the others may still read its shared memory
  __device__ __forceinline__ void leave() const {
    if constexpr (C > 1) cg::this_cluster().sync();
  }
  __device__ __forceinline__ const Shared* of(int c) const {
    if constexpr (C > 1) return cg::this_cluster().map_shared_rank(&sh, c);
    else return &sh;
  }
  // the pages' references as ballots (a negative one is in neither)
  __device__ __forceinline__ void look(const Book& k) {
    const int per = round_up(ceil_div(k.n_pages, C * kWarps), 32);
    lo = (int)min((int64_t)k.n_pages, (int64_t)(rank * kWarps + warp) * per);
    hi = min(k.n_pages, lo + per);
    cached = per <= 32 * kCached;
    if (!cached) return;
    int r[kCached];
#pragma unroll
    for (int j = 0; j < kCached; ++j) r[j] = lo + 32 * j + lane < hi ? __ldcg(k.ref + lo + 32 * j + lane) : -1;
#pragma unroll
    for (int j = 0; j < kCached; ++j) {
      live[j] = __ballot_sync(~0u, r[j] > 0);
      none[j] = __ballot_sync(~0u, r[j] == 0);
    }
  }
  // f(first page, ballot of live ones, of free ones) over the stretch
  template <typename F>
  __device__ __forceinline__ void each(const Book& k, F f) const {
    if (cached) {
#pragma unroll
      for (int j = 0; j < kCached; ++j)
        if (lo + 32 * j < hi) f(lo + 32 * j, live[j], none[j]);
    } else {
#pragma unroll 4
      for (int p = lo; p < hi; p += 32) {
        const int r = p + lane < hi ? __ldcg(k.ref + p + lane) : -1;
        f(p, __ballot_sync(~0u, r > 0), __ballot_sync(~0u, r == 0));
      }
    }
  }
  // A barrier of the team that also orders its memory accesses: all threads' bits; of the warps'
  // counts a and b those before this warp and all of them
  __device__ __forceinline__ int exchange(int bits, int a, int b, int2* before, int2* all) {
    Exchange& x = sh.x[turn];
    bits = __reduce_or_sync(~0u, bits);
    if (lane == 0) {
      x.flag[warp] = bits;
      x.a[warp] = a;
      x.b[warp] = b;
    }
    sync();
    int flag = 0;
    int2 pre = make_int2(0, 0), tot = make_int2(0, 0);
    for (int c = 0; c < C; ++c) {
      const Exchange& y = of(c)->x[turn];
      const int ya = y.a[lane], yb = y.b[lane];
      flag |= y.flag[lane];
      tot.x += ya;
      tot.y += yb;
      if (c < rank || (c == rank && lane < warp)) {
        pre.x += ya;
        pre.y += yb;
      }
    }
    turn ^= 1;
    before->x = __reduce_add_sync(~0u, pre.x);
    before->y = __reduce_add_sync(~0u, pre.y);
    all->x = __reduce_add_sync(~0u, tot.x);
    all->y = __reduce_add_sync(~0u, tot.y);
    return __reduce_or_sync(~0u, flag);
  }
  __device__ __forceinline__ int exchange(int bits) {
    int2 x, y;
    return exchange(bits, 0, 0, &x, &y);
  }
  __device__ __forceinline__ int count_free(const Book& k) const {
    int n = 0;
    each(k, [&](int, uint32_t, uint32_t z) { n += __popc(z); });
    return n;
  }
  // the n lowest free pages to list (there are as many); base: the free ones before this warp's
  __device__ __forceinline__ void list_free(const Book& k, int n, int base, int32_t* list) const {
    each(k, [&](int p, uint32_t, uint32_t z) {
      const int rk = base + __popc(z & ((1u << lane) - 1));
      if (((z >> lane) & 1u) && rk < n) list[rk] = p + lane;
      base += __popc(z);
    });
  }
  // off[i] = sum of f(0 .. i-1) for i < n and sh.total all of them, by the first CTA (ordered by the next exchange)
  template <typename F>
  __device__ __forceinline__ void offsets(int n, int32_t* off, F f) const {
    if (rank != 0) return;
    int run = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
      const int i = i0 + t, v = i < n ? f(i) : 0;
      int incl = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(~0u, incl, o);
        if (lane >= o) incl += u;
      }
      if (lane == 31) sh.scan[warp] = incl;
      __syncthreads();
      const int w = sh.scan[lane];
      const int before = __reduce_add_sync(~0u, lane < warp ? w : 0), all = __reduce_add_sync(~0u, w);
      if (i < n) off[i] = run + before + incl - v;
      run += all;
      __syncthreads();
    }
    if (t == 0) sh.total = run;
  }
};

// (len + page - 1 may pass 32 bits)
__device__ __forceinline__ int pages_of(int len, int page) { return len / page + (len % page != 0); }
// Slot which[i] in range, and stamped with i.  (A slot listed twice holds the stamp of one of the two, so
// after a barrier the other's check fails; the stamps need no clearing)
template <int C>
__device__ __forceinline__ int stamp(const Team<C>& team, const Book& k, const int32_t* which, int n, int32_t* mark) {
  int bad = 0;
  for (int i = team.id; i < n; i += team.size) {
    const int s = which[i];
    if (s < 0 || s >= k.slots) bad = KF_DEV_BAD_ROW;
    else mark[s] = i;
  }
  return bad;
}
template <int C>
__device__ __forceinline__ int twice(const Team<C>& team, const int32_t* which, int n, const int32_t* mark) {
  int bad = 0;
  for (int i = team.id; i < n; i += team.size)
    if (__ldcg(mark + which[i]) != i) bad = KF_DEV_BAD_ROW;
  return bad;
}
template <int C>
__device__ __forceinline__ bool refused(const Team<C>& team, int bad, int* err) {
  if (!bad) return false;
  if (bad & KF_DEV_BAD_ROW) bad = KF_DEV_BAD_ROW;      // (what a bad list makes of the pages is no fault of theirs)
  if (team.id == 0) atomicOr(err, bad);
  team.leave();
  return true;
}

template <int C>
__global__ void __launch_bounds__(kThreads, 1) k_grow(const Book k, int n, const int32_t* which, const int32_t* new_lens, const Work w, int* err) {
  __shared__ Shared sh;
  Team<C> team(sh);
  team.look(k);
  int bad = stamp(team, k, which, n, w.mark);
  // new pages of request i (0 for a bad one)
  auto more = [&](int i) {
    const int s = which[i], now = new_lens[i];
    if (s < 0 || s >= k.slots) return 0;
    const int was = k.lens[s];
    if (was < 0 || now < was || now > (int64_t)k.width * k.page) {
      bad |= KF_DEV_BAD_ROW;
      return 0;
    }
    return pages_of(now, k.page) - pages_of(was, k.page);
  };
  team.offsets(n, w.off, more);
  int2 before, all;
  bad = team.exchange(bad, team.count_free(k), 0, &before, &all);
  if (refused(team, bad, err)) return;
  const int total = team.of(0)->total, warps = team.size >> 5;
  team.list_free(k, min(total, all.x), before.x, w.src);
  bad = twice(team, which, n, w.mark);
  // f(place in the table, rank among the new pages) of every new column, then done(request): a warp's lanes hold a request
  // each and take its one column, or all of them the columns of one after the other
  auto columns = [&](auto f, auto done) {
    for (int i0 = team.id >> 5; i0 < n; i0 += 32 * warps) {
      const int i = i0 + warps * team.lane;
      int s = 0, have = 0, add = 0, off = 0;
      if (i < n) {
        s = which[i];
        have = pages_of(k.lens[s], k.page);
        add = pages_of(new_lens[i], k.page) - have;
        off = __ldcg(w.off + i);
      }
      if (add == 1) f((int64_t)s * k.width + have, off);
      for (uint32_t wide = __ballot_sync(~0u, add > 1); wide; wide &= wide - 1) {
        const int j = __ffs(wide) - 1, nj = __shfl_sync(~0u, add, j), oj = __shfl_sync(~0u, off, j);
        const int64_t at = (int64_t)__shfl_sync(~0u, s, j) * k.width + __shfl_sync(~0u, have, j);
        for (int c = team.lane; c < nj; c += 32) f(at + c, oj + c);
      }
      if (i < n) done(i);
    }
  };
  // (a page there, as after a length that was lowered by hand, would be lost)
  columns([&](int64_t at, int) { bad |= k.table[at] != -1 ? KF_DEV_BAD_PAGE : 0; }, [](int) {});
  bad = team.exchange(bad);
  if (!bad && total > all.x) bad = KF_DEV_NO_PAGES;
  if (refused(team, bad, err)) return;
  columns(
      [&](int64_t at, int rank) {
        const int p = __ldcg(w.src + rank);
        k.table[at] = p;
        k.ref[p] = 1;
      },
      [&](int i) { k.lens[which[i]] = new_lens[i]; });
  team.leave();
}

template <int C>
__global__ void __launch_bounds__(kThreads, 1) k_free(const Book k, int n, const int32_t* which, const Work w, int* err) {
  __shared__ Shared sh;
  Team<C> team(sh);
  int bad = team.exchange(stamp(team, k, which, n, w.mark));
  if (refused(team, bad, err)) return;
  const uint32_t all = (uint32_t)n * k.width, width = k.width;
  bad = twice(team, which, n, w.mark);
  for (uint32_t e = team.id; e < all; e += team.size) {
    const int p = k.table[(int64_t)which[e / width] * k.width + e % width];
    if (p == -1) continue;
    if (p < 0 || p >= k.n_pages || atomicSub(k.ref + p, 1) <= 0) bad |= KF_DEV_BAD_PAGE;
  }
  bad = team.exchange(bad);
  if (bad)
    // the references as they were
    for (uint32_t e = team.id; e < all; e += team.size) {
      const int p = k.table[(int64_t)which[e / width] * k.width + e % width];
      if (p >= 0 && p < k.n_pages) atomicAdd(k.ref + p, 1);
    }
  if (refused(team, bad, err)) return;
  for (uint32_t e = team.id; e < all; e += team.size) k.table[(int64_t)which[e / width] * k.width + e % width] = -1;
  for (int i = team.id; i < n; i += team.size) k.lens[which[i]] = 0;
  team.leave();
}

template <int C>
__global__ void __launch_bounds__(kThreads, 1) k_fork(const Book k, int n, const int32_t* src, const int32_t* dst, const Work w, int* err) {
  __shared__ Shared sh;
  Team<C> team(sh);
  if (team.id == 0) *w.count = 0;            // (a refused call copies nothing)
  team.look(k);
  int bad = stamp(team, k, dst, n, w.mark);
  for (int i = team.id; i < n; i += team.size) {
    const int s = src[i], d = dst[i];
    if (s < 0 || s >= k.slots || k.lens[s] < 0 || k.lens[s] > (int64_t)k.width * k.page) bad |= KF_DEV_BAD_ROW;
    if (d >= 0 && d < k.slots && k.lens[d] != 0) bad |= KF_DEV_BAD_ROW;
  }
  team.offsets(n, w.off, [&](int i) { return src[i] >= 0 && src[i] < k.slots && k.lens[src[i]] % k.page != 0 ? 1 : 0; });
  int2 before, free;
  bad = team.exchange(bad, team.count_free(k), 0, &before, &free);
  if (refused(team, bad, err)) return;
  const int total = team.of(0)->total;
  bad = twice(team, dst, n, w.mark);
  for (int i = team.id; i < n; i += team.size) {
    const int s = src[i], m = __ldcg(w.mark + s);
    if (m >= 0 && m < n && dst[m] == s) bad |= KF_DEV_BAD_ROW;      // a source that is a destination
  }
  const uint32_t all = (uint32_t)n * k.width, width = k.width;
  for (uint32_t e = team.id; e < all; e += team.size) {
    const int i = (int)(e / width), c = (int)(e % width);
    if (k.table[(int64_t)dst[i] * k.width + c] != -1) bad |= KF_DEV_BAD_PAGE;      // not empty
    if (c >= pages_of(k.lens[src[i]], k.page)) continue;
    const int p = k.table[(int64_t)src[i] * k.width + c];
    if (p < 0 || p >= k.n_pages || __ldcg(k.ref + p) <= 0) bad |= KF_DEV_BAD_PAGE;
  }
  team.list_free(k, min(total, free.x), before.x, w.dst);
  bad = team.exchange(bad);
  if (!bad && total > free.x) bad = KF_DEV_NO_PAGES;
  if (refused(team, bad, err)) return;
  for (uint32_t e = team.id; e < all; e += team.size) {
    const int i = (int)(e / width), c = (int)(e % width), len = k.lens[src[i]], full = len / k.page;
    int p = -1;
    if (c < full) {
      p = k.table[(int64_t)src[i] * k.width + c];
      atomicAdd(k.ref + p, 1);
    } else if (c == full && len % k.page) {
      const int off = __ldcg(w.off + i);
      w.src[off] = k.table[(int64_t)src[i] * k.width + c];
      p = __ldcg(w.dst + off);
      k.ref[p] = 1;
    }
    if (p != -1) k.table[(int64_t)dst[i] * k.width + c] = p;
    if (c == 0) k.lens[dst[i]] = len;
  }
  if (team.id == 0) *w.count = total;
  team.leave();
}

template <int C>
__global__ void __launch_bounds__(kThreads, 1) k_compact(const Book k, const Work w, int32_t* live, int* err) {
  __shared__ Shared sh;
  Team<C> team(sh);
  if (team.id == 0) *w.count = 0;
  team.look(k);
  int bad = 0, n = 0;
  team.each(k, [&](int p, uint32_t x, uint32_t z) {
    n += __popc(x);
    const uint32_t in = p + 32 <= team.hi ? ~0u : (1u << (team.hi - p)) - 1;
    if ((x | z) != in) bad |= KF_DEV_BAD_PAGE;             // a negative reference count
  });
  const uint32_t entries = (uint32_t)k.slots * k.width;
  for (uint32_t e = team.id; e < entries; e += team.size) {
    const int p = k.table[e];
    if (p != -1 && (p < 0 || p >= k.n_pages || __ldcg(k.ref + p) <= 0)) bad |= KF_DEV_BAD_PAGE;
  }
  int2 before, all;
  bad = team.exchange(bad, n, 0, &before, &all);
  if (refused(team, bad, err)) return;
  const int L = all.x;
  // the live pages at or above L, and as many free ones below
  auto high = [&](int p, uint32_t x) { return p >= L ? x : p + 32 <= L ? 0u : x & ~((1u << (L - p)) - 1); };
  auto hole = [&](int p, uint32_t z) { return p >= L ? 0u : p + 32 <= L ? z : z & ((1u << (L - p)) - 1); };
  int nh = 0, nz = 0;
  team.each(k, [&](int p, uint32_t x, uint32_t z) {
    nh += __popc(high(p, x));
    nz += __popc(hole(p, z));
  });
  team.exchange(0, nh, nz, &before, &all);
  team.each(k, [&](int p, uint32_t x, uint32_t z) {
    const uint32_t h = high(p, x), o = hole(p, z), below = (1u << team.lane) - 1;
    if ((h >> team.lane) & 1u) {
      const int rk = before.x + __popc(h & below);
      w.src[rk] = p + team.lane;
      w.to[p + team.lane] = rk;
    }
    if ((o >> team.lane) & 1u) w.dst[before.y + __popc(o & below)] = p + team.lane;
    before.x += __popc(h);
    before.y += __popc(o);
  });
  team.sync();
  for (int i = team.id; i < all.x; i += team.size) {
    const int s = __ldcg(w.src + i), d = __ldcg(w.dst + i);
    k.ref[d] = __ldcg(k.ref + s);
    k.ref[s] = 0;
  }
  for (uint32_t e = team.id; e < entries; e += team.size) {
    const int p = k.table[e];
    if (p >= L) k.table[e] = __ldcg(w.dst + __ldcg(w.to + p));
  }
  if (team.id == 0) {
    *w.count = all.x;
    if (live) *live = L;
  }
}

// page src[i] to dst[i] in every layer; the list's length is n, or *count
__global__ void __launch_bounds__(kCopyThreads) k_move(uint8_t* pool, int layers, int n_pages, int64_t page_bytes, const int32_t* src,
                                                     const int32_t* dst, int n, const int32_t* count, int* err) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (count) n = __ldcg(count);
  const int chunks = (int)((page_bytes + kCopyUnit - 1) / kCopyUnit);
  const int64_t units = (int64_t)n * layers * chunks;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t m = u / chunks;
    const int i = (int)(m / layers), layer = (int)(m % layers);
    const int s = __ldcg(src + i), d = __ldcg(dst + i);
    if (s < 0 || d < 0 || s >= n_pages || d >= n_pages) {
      if (threadIdx.x == 0) atomicOr(err, KF_DEV_BAD_PAGE);
      continue;
    }
    const int64_t at = (u - m * chunks) * kCopyUnit + threadIdx.x * 16;
    const uint8_t* from = pool + ((int64_t)layer * n_pages + s) * page_bytes + at;
    uint8_t* to = pool + ((int64_t)layer * n_pages + d) * page_bytes + at;
    uint4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at + j * kCopyThreads * 16 < page_bytes) v[j] = *reinterpret_cast<const uint4*>(from + j * kCopyThreads * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at + j * kCopyThreads * 16 < page_bytes) *reinterpret_cast<uint4*>(to + j * kCopyThreads * 16) = v[j];
  }
}

// K and V rows into their pages: a CTA takes kTokens tokens; a thread copies 16 bytes at a time
constexpr int kTokens = 16;
struct Append {
  const int32_t *which, *starts, *table, *lens;
  const uint8_t *k, *v;
  uint8_t* pool;
  int64_t T, k_row, k_head, v_row, v_head;       // strides in bytes
  int n, Hkv, chunks, n_pages, page, slots, width;   // chunks: 16-byte pieces of a head
};
__global__ void __launch_bounds__(kCopyThreads) k_append(const Append a, int* err) {
  __shared__ int64_t row[kTokens];               // K's first piece in the pool, or -1
  const int64_t t0 = (int64_t)blockIdx.x * kTokens;
  if (threadIdx.x < kTokens && t0 + threadIdx.x < a.T) {
    const int64_t t = t0 + threadIdx.x;
    int lo = 0, hi = a.n - 1;                    // the last sequence that starts at or before t
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (__ldg(a.starts + mid) <= t) lo = mid;
      else hi = mid - 1;
    }
    const int first = __ldg(a.starts + lo), end = __ldg(a.starts + lo + 1), s = __ldg(a.which + lo);
    int64_t at = -1;
    int bad = 0;
    if (t < first || t >= end || s < 0 || s >= a.slots) bad = KF_DEV_BAD_ROW;
    else {
      const int64_t pos = (int64_t)a.lens[s] - end + t;
      if (pos < 0 || pos >= (int64_t)a.width * a.page) bad = KF_DEV_BAD_ROW;
      else {
        const int p = a.table[(int64_t)s * a.width + pos / a.page];
        if (p < 0 || p >= a.n_pages) bad = KF_DEV_BAD_PAGE;
        else at = ((int64_t)p * 2 * a.Hkv * a.page + pos % a.page) * a.chunks;
      }
    }
    if (bad) atomicOr(err, bad);
    row[threadIdx.x] = at;
  }
  __syncthreads();
  const int per = 2 * a.Hkv * a.chunks, tokens = (int)min((int64_t)kTokens, a.T - t0);
  const int total = tokens * per;
#pragma unroll 4
  for (int i = threadIdx.x; i < total; i += kCopyThreads) {
    const int j = i / per, e = i - j * per, h2 = e / a.chunks, ch = e - h2 * a.chunks;     // h2: K heads, then V heads
    if (row[j] < 0) continue;
    const bool v = h2 >= a.Hkv;
    const uint8_t* from = v ? a.v + (t0 + j) * a.v_row + (h2 - a.Hkv) * a.v_head : a.k + (t0 + j) * a.k_row + h2 * a.k_head;
    const int64_t to = row[j] + (int64_t)h2 * a.page * a.chunks + ch;
    reinterpret_cast<uint4*>(a.pool)[to] = *reinterpret_cast<const uint4*>(from + ch * 16);
  }
}

// ------------------------------------------------------------------ host
Work layout(void* work, int n_pages, int slots, int n) {
  int32_t* p = static_cast<int32_t*>(work);
  Work w;
  w.count = p;
  w.mark = p + 64;
  w.off = w.mark + slots;
  w.src = w.off + n;
  w.dst = w.src + n_pages;
  w.to = w.dst + n_pages;
  return w;
}
const char* book_fault(const Book& k, const void* work) {
  if (k.n_pages < 1 || k.n_pages > (1 << 30) || k.slots < 1 || k.slots > (1 << 30) || k.width < 0 || k.width > (1 << 30)) return "pages, slots or width out of range";
  if ((int64_t)k.slots * k.width > 0x7fffffffll) return "slots * width out of range";      // (sums of pages stay in 32 bits)
  if (k.page < 1 || k.page > (1 << 20) || (int64_t)k.width * k.page > 0x7fffffffll) return "page, or width * page, out of range";
  if (!k.ref || (k.width && !k.table) || !work) return "a null array";
  if (!aligned(k.ref, 4) || !aligned(k.table, 4) || !aligned(k.lens, 4) || !aligned(work, 256)) return "an array is not aligned (work: 256 bytes)";
  return nullptr;
}
const char* pool_fault(const void* pool, int layers, int64_t page_bytes) {
  if (layers < 1 || layers > (1 << 20)) return "layers out of range";
  if (page_bytes < 16 || page_bytes % 16 || page_bytes > (1 << 30)) return "page_bytes is a multiple of 16";
  if (!pool || !aligned(pool, 16)) return "the pool is null or not 16-byte aligned";
  return nullptr;
}
// A cluster's barriers cost a few microseconds that a small book does not repay: one CTA up
// to 8 references (what its warps keep as ballots) and 8 table entries a thread.  Measured on
// compact's bookkeeping, one CTA and the cluster: 1,024 pages 6.3 and 13.7 us, 8,192 10.9 and
// 14.2, 16,384 21.1 and 15.0, 131,072 144 and 31
bool small_book(int64_t pages, int64_t entries) { return pages <= 8 * kThreads && entries <= 8 * kThreads; }

#define KF_TEAM(kernel, small, s, ...)                                                      \
  do {                                                                                      \
    if (small) launch_cluster(kernel<1>, dim3(1), dim3(kThreads), 0, 1, false, s, __VA_ARGS__); \
    else launch_cluster(kernel<kTeam>, dim3(kTeam), dim3(kThreads), 0, kTeam, false, s, __VA_ARGS__); \
  } while (0)

void launch_move(uint8_t* pool, int layers, int n_pages, int64_t page_bytes, const int32_t* src, const int32_t* dst, int n,
                 const int32_t* count, int* err, bool dependent, cudaStream_t s) {
  const int64_t units = (int64_t)n * layers * ((page_bytes + kCopyUnit - 1) / kCopyUnit);
  const int grid = (int)std::min<int64_t>(8ll * device_sms(), std::max<int64_t>(1, units));
  launch_cluster(k_move, dim3(grid), dim3(kCopyThreads), 0, 1, dependent, s, pool, layers, n_pages, page_bytes, src, dst, n, count, err);
}

}  // namespace
}  // namespace kf

using namespace kf;

extern "C" int64_t kf_op_pages_work(int32_t n_pages, int32_t slots, int32_t n) {
  if (n_pages < 0 || slots < 0 || n < 0) return 0;
  return 4 * (64 + (int64_t)slots + n + 3 * (int64_t)n_pages);
}

extern "C" int kf_op_pages_grow(int32_t n, const int32_t* which, const int32_t* new_lens, int32_t* ref, int32_t n_pages,
                                int32_t* table, int32_t slots, int32_t width, int32_t* lens, int32_t page, void* work,
                                void* stream) {
  const char* what = "kf_op_pages_grow";
  const Book k{ref, table, lens, n_pages, slots, width, page};
  if (const char* f = book_fault(k, work)) return refuse(what, f);
  if (n < 0 || n > slots) return refuse(what, "more slots listed than there are");
  if (n == 0) return KF_OK;
  if (!which || !new_lens || !lens || !aligned(which, 4) || !aligned(new_lens, 4)) return refuse(what, "a null or misaligned list");
  int* err = serving_error_word();
  if (!err) return refuse(what, "no error word", KF_E_CUDA);
  KF_TEAM(k_grow, small_book(n_pages, n), (cudaStream_t)stream, k, n, which, new_lens, layout(work, n_pages, slots, n), err);
  return launched(what);
}

extern "C" int kf_op_pages_free(int32_t n, const int32_t* which, int32_t* ref, int32_t n_pages, int32_t* table, int32_t slots,
                                int32_t width, int32_t* lens, int32_t page, void* work, void* stream) {
  const char* what = "kf_op_pages_free";
  const Book k{ref, table, lens, n_pages, slots, width, page};
  if (const char* f = book_fault(k, work)) return refuse(what, f);
  if (n < 0 || n > slots) return refuse(what, "more slots listed than there are");
  if (n == 0) return KF_OK;
  if (!which || !lens || !aligned(which, 4)) return refuse(what, "a null or misaligned list");
  int* err = serving_error_word();
  if (!err) return refuse(what, "no error word", KF_E_CUDA);
  KF_TEAM(k_free, small_book(0, (int64_t)n * width), (cudaStream_t)stream, k, n, which, layout(work, n_pages, slots, n), err);
  return launched(what);
}

extern "C" int kf_op_pages_fork(int32_t n, const int32_t* src, const int32_t* dst, int32_t* ref, int32_t n_pages, int32_t* table,
                                int32_t slots, int32_t width, int32_t* lens, int32_t page, void* pool, int32_t layers,
                                int64_t page_bytes, void* work, void* stream) {
  const char* what = "kf_op_pages_fork";
  const Book k{ref, table, lens, n_pages, slots, width, page};
  if (const char* f = book_fault(k, work)) return refuse(what, f);
  if (const char* f = pool_fault(pool, layers, page_bytes)) return refuse(what, f);
  if (n < 0 || n > slots) return refuse(what, "more slots listed than there are");
  if (n == 0) return KF_OK;
  if (!src || !dst || !lens || !aligned(src, 4) || !aligned(dst, 4)) return refuse(what, "a null or misaligned list");
  int* err = serving_error_word();
  if (!err) return refuse(what, "no error word", KF_E_CUDA);
  const Work w = layout(work, n_pages, slots, n);
  cudaStream_t s = (cudaStream_t)stream;
  KF_TEAM(k_fork, small_book(n_pages, (int64_t)n * width), s, k, n, src, dst, w, err);
  if (const int rc = launched(what)) return rc;
  launch_move(static_cast<uint8_t*>(pool), layers, n_pages, page_bytes, w.src, w.dst, n, w.count, err, true, s);
  return launched(what);
}

extern "C" int kf_op_pages_compact(int32_t* ref, int32_t n_pages, int32_t* table, int32_t slots, int32_t width, void* pool,
                                   int32_t layers, int64_t page_bytes, int32_t* live, void* work, void* stream) {
  const char* what = "kf_op_pages_compact";
  const Book k{ref, table, nullptr, n_pages, slots, width, 1};
  if (const char* f = book_fault(k, work)) return refuse(what, f);
  if (const char* f = pool_fault(pool, layers, page_bytes)) return refuse(what, f);
  if (!aligned(live, 4)) return refuse(what, "live is misaligned");
  int* err = serving_error_word();
  if (!err) return refuse(what, "no error word", KF_E_CUDA);
  const Work w = layout(work, n_pages, slots, 0);
  cudaStream_t s = (cudaStream_t)stream;
  KF_TEAM(k_compact, small_book(n_pages, (int64_t)slots * width), s, k, w, live, err);
  if (const int rc = launched(what)) return rc;
  launch_move(static_cast<uint8_t*>(pool), layers, n_pages, page_bytes, w.src, w.dst, n_pages, w.count, err, true, s);
  return launched(what);
}

extern "C" int kf_op_pages_copy(int32_t n, const int32_t* src, const int32_t* dst, void* pool, int32_t layers, int32_t n_pages,
                                int64_t page_bytes, void* stream) {
  const char* what = "kf_op_pages_copy";
  if (const char* f = pool_fault(pool, layers, page_bytes)) return refuse(what, f);
  if (n < 0 || n_pages < 1 || n > n_pages) return refuse(what, "more pages listed than there are");
  if (n == 0) return KF_OK;
  if (!src || !dst || !aligned(src, 4) || !aligned(dst, 4)) return refuse(what, "a null or misaligned list");
  int* err = serving_error_word();
  if (!err) return refuse(what, "no error word", KF_E_CUDA);
  launch_move(static_cast<uint8_t*>(pool), layers, n_pages, page_bytes, src, dst, n, nullptr, err, false, (cudaStream_t)stream);
  return launched(what);
}

extern "C" int kf_op_pages_append(int32_t n, const int32_t* which, const int32_t* starts, int64_t T, int32_t Hkv, int32_t hd,
                                  const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row, int64_t v_head,
                                  void* pool, int32_t n_pages, int32_t page, const int32_t* table, int32_t slots, int32_t width,
                                  const int32_t* lens, void* stream) {
  const char* what = "kf_op_pages_append";
  if (n < 0 || T < 0 || T > 0x7fffffffll || n_pages < 1 || slots < 1 || width < 0) return refuse(what, "sequences, tokens, pages, slots or width out of range");
  if (Hkv < 1 || Hkv > 4096 || hd < 8 || hd % 8 || hd > 4096) return refuse(what, "heads out of range, or hd no multiple of 8");
  if (page < 1 || page > (1 << 20) || (int64_t)width * page > 0x7fffffffll) return refuse(what, "page, or width * page, out of range");
  if (n == 0 || T == 0) return KF_OK;
  if (!which || !starts || !k || !v || !pool || !lens || (width && !table)) return refuse(what, "a null array");
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(pool, 16) || !aligned(which, 4) || !aligned(starts, 4) || !aligned(table, 4) || !aligned(lens, 4))
    return refuse(what, "k, v and the pool are 16-byte aligned");
  if (k_row % 8 || k_head % 8 || v_row % 8 || v_head % 8) return refuse(what, "strides are multiples of 8 elements");
  int* err = serving_error_word();
  if (!err) return refuse(what, "no error word", KF_E_CUDA);
  const Append a{which, starts, table, lens, static_cast<const uint8_t*>(k), static_cast<const uint8_t*>(v), static_cast<uint8_t*>(pool),
                 T, k_row * 2, k_head * 2, v_row * 2, v_head * 2, n, Hkv, hd / 8, n_pages, page, slots, width};
  launch_cluster(k_append, dim3((unsigned)((T + kTokens - 1) / kTokens)), dim3(kCopyThreads), 0, 1, false, (cudaStream_t)stream, a, err);
  return launched(what);
}
