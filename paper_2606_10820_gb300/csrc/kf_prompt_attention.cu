// Causal attention over packed prompts (kf_op_prompt_attention): grouped heads,
// head_dim 64 or 128, bf16 or fp16, on tcgen05.
//
// An item is two sub-tiles of 128 query rows that read the same K and V tiles: the same
// rows under two heads of a group where groups are even (both sub-tiles then end at
// the same key), else 256 consecutive rows of one head.  A CTA per SM of twelve warps:
//   warp 0      takes items, and copies Q, K and V tiles (TMA, 128-byte swizzle);
//   warp 1      issues S = Q K^T (128 x 128 x hd) and O += P V (128 x hd x 128), the two
//               sub-tiles in turn, so that one's softmax runs under the other's products;
//   warps 4-7, 8-11  the softmax of sub-tile 0 and 1, one thread per row (its TMEM
//               lane): no exchange between threads.  P goes back to TMEM in two halves, so
//               that its product begins under the second half's exponentials: to columns of
//               its own at head_dim 64, over the first half of its own S columns at 128 (the
//               products run in the order of their instructions, so the next S needs no other buffer).
// Scores are taken against a reference per row that follows its maximum only past a factor of
// 2^8, so O is rarely rescaled; sums are fp32, P is rounded to the inputs' type (the
// tensor cores' operand).
//
// The items come sorted by their key tiles, longest first.  Up to 128 sequences each CTA's load
// warp holds the lengths in registers and finds its items itself; for more a block before
// (k_plan) writes the list (a launch and about 5 us that a short call does not repay).  The grid has a
// CTA per item, and a CTA that is through takes over one that has not started (dealt out beforehand
// the items took 30.2 us against 26.6 at 16 prompts of 128 to 896, 12 heads over 4 of 64).  What bounds it: long prompts the tensor
// cores (2,048 clocks a key tile of hd 128 and 256 rows), short ones the chain of an item.
//
// Measured (bf16): prompts of 7,411 and 8,192, 16 heads over 4 of 128, in 317 us (1.57 PFLOP/s); 16
// of 128 to 896, 12 over 4 of 64, in 26 us; five of 1 to 77, 7 over 1 of 128, fp16, in 6.7 us.
#include <algorithm>
#include <climits>

#include "kf_attn_pair.cuh"
#include "kf_serving.cuh"

namespace kf {
namespace {
using namespace pair;

constexpr int kMaxTiles = 4096;                    // key tiles of a sequence: 524,288 tokens
constexpr int kPlanThreads = 1024;
constexpr int kDirect = 4;                          // sequences that a lane of the load warp holds: up to 128 without a plan

struct PlanItem { int start, len, tile, pad; };     // a sequence's first token, its tokens, its tile of rows
struct Plan {
  int* count;                                       // items (without heads)
  PlanItem* item;
};

// one sub-tile pair, as the load warp hands it to the others
struct Item {
  int start, len;
  int row[2], head[2], n[2];                        // first row, head, key tiles (0: no sub-tile)
};

struct Args {
  void* out;
  int64_t out_row, out_head;
  Plan plan;
  int* err;
  int Hq, G, heads, tiles;                          // of an item: heads x tiles of 128 rows (2 x 1, 1 x 2 or 1 x 1)
  int direct, steal, n, T, longest;                 // direct: the items are found from starts, without a plan; steal: a CTA per item, whose
                                                    // CTAs take over those that have not started
  const int32_t* starts;
  float scale2;
};
struct Maps { CUtensorMap q, k, v; };

// ------------------------------------------------------------------ plan
// Items of `rows` query rows, those with most keys first: with c tiles needed up to its
// last row, an item of class c comes after all items of higher classes, and each
// sequence of at least c tiles has one.  The order within a class is any.
__global__ void __launch_bounds__(kPlanThreads) k_plan(int n, int T, int longest, int rows, int classes, const int32_t* starts,
                                                        Plan plan, int* err) {
  extern __shared__ __align__(1024) uint8_t sm[];
  int* at_least = reinterpret_cast<int*>(sm);       // [classes + 2]: sequences of at least c tiles
  int* first = at_least + classes + 2;                    // [classes + 2]: the first item of class c
  __shared__ int warp_sum[32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  for (int c = t; c < 2 * (classes + 2); c += kPlanThreads) at_least[c] = 0;
  int bad = 0;
  for (int s = t; s < n; s += kPlanThreads) {
    const int a = starts[s], b = starts[s + 1];
    bad |= a < 0 || b < a || b > T || b - a > longest || (s == 0 && a != 0) || (s == n - 1 && b != T);
  }
  bad = __syncthreads_or(bad);
  if (bad) {
    if (t == 0) {
      atomicOr(err, KF_DEV_BAD_ROW);
      *plan.count = 0;
    }
    return;
  }
  for (int s = t; s < n; s += kPlanThreads) atomicAdd(&at_least[(starts[s + 1] - starts[s] + rows - 1) / rows], 1);
  __syncthreads();
  // suffix sums of the counts, then of those (each thread a run of classes, from the top)
  const int per = (classes + kPlanThreads - 1) / kPlanThreads;
  for (int round = 0; round < 2; ++round) {
    const int hi = classes - t * per, lo = max(0, hi - per);      // classes hi .. lo + 1
    int mine = 0;
    for (int c = hi; c > lo; --c) mine += at_least[c];
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(~0u, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    int run = __reduce_add_sync(~0u, lane < warp ? warp_sum[lane] : 0) + incl - mine;
    for (int c = hi; c > lo; --c) {
      if (round == 0) {
        run += at_least[c];
        at_least[c] = run;
      } else {
        first[c] = run;                             // the items of the classes above
        run += at_least[c];
      }
    }
    // (all items; before the barrier, behind which at_least counts down)
    if (round == 1 && hi > 0 && lo == 0) *plan.count = run;
    __syncthreads();
  }
  // A sequence's place among all, those with more tiles first: class c has the places
  // at_least[c + 1] .. at_least[c] - 1, taken from the end.  It holds in every class up to its own
  for (int s0 = 0; s0 < n; s0 += 32) {              // warps take 32 sequences at a time
    if ((s0 / 32) % 32 != warp) continue;
    const int s = s0 + lane;
    const int a = s < n ? starts[s] : 0, len = s < n ? starts[s + 1] - a : 0, c = (len + rows - 1) / rows;
    const int place = c > 0 ? atomicSub(&at_least[c], 1) - 1 : 0;
    for (int j = 0; j < 32; ++j) {
      const int cj = __shfl_sync(~0u, c, j), aj = __shfl_sync(~0u, a, j), lj = __shfl_sync(~0u, len, j), pj = __shfl_sync(~0u, place, j);
      for (int x = lane; x < cj; x += 32) plan.item[first[x + 1] + pj] = PlanItem{aj, lj, x, 0};
    }
  }
}

// ------------------------------------------------------------------ the products
// (themselves in kf_attn_pair.cuh; here, how a CTA takes the next ones)
// Cluster launch control: a running CTA cancels one that has not started and does its work (the
// hardware's queue instead of a counter in memory that a call would have to clear)
__device__ __forceinline__ void ask_for_cta(uint64_t* answer, uint64_t* bar) {
  mbar_expect_tx(smem_u32(bar), 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(answer)),
               "r"(smem_u32(bar))
               : "memory");
}
// its index, or -1: none is left
__device__ __forceinline__ int cta_taken(const uint64_t* answer) {
  uint64_t lo, hi;
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(lo), "=l"(hi) : "r"(smem_u32(answer)) : "memory");
  int x;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\t"
      "mov.b128 r, {%1, %2};\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
      "mov.s32 %0, -1;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, r;\n\t}"
      : "=&r"(x)
      : "l"(lo), "l"(hi));
  return x;
}

struct Bars : PairBars<Item> {
  uint64_t taken;                                        // a request to take over a CTA is answered
  alignas(16) uint64_t answer[2];
};
static_assert(sizeof(Bars) <= kBarBytes, "the barriers' part of the shared memory");

template <typename T, int HD>
__global__ void __launch_bounds__(kThreads, 1) k_prompt(const __grid_constant__ Maps maps, const Args a) {
  extern __shared__ __align__(1024) uint8_t sm[];
  constexpr int ST = kStages<HD>, AT = HD / 64;
  constexpr uint32_t TILE = kTile<HD>;
  Bars& b = *reinterpret_cast<Bars*>(sm + (2 + ST) * TILE);
  const uint32_t sQ = smem_u32(sm), sKV = sQ + 2 * TILE;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  if (sQ & 1023) {                              // (uniform) swizzle atoms need the alignment
    if (t == 0) atomicOr(a.err, kErrInternal);
    return;
  }
  if (t == 0) {
    auto init = [](uint64_t* p, uint32_t n) { mbar_init(smem_u32(p), n); };
    init(&b.q_full, 1);
    init(&b.q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      init(&b.item_full[i], 1);
      init(&b.item_empty[i], 9);                // the MMA warp and eight softmax warps
      init(&b.s_full[i], 1);
      init(&b.s_free[i], 4);
      init(&b.p_full[i][0], 4);
      init(&b.p_full[i][1], 4);
      init(&b.o_full[i], 1);
      init(&b.o_free[i], 4);
    }
    init(&b.tail, 1);
    init(&b.taken, 1);
    for (int i = 0; i < ST; ++i) {
      init(&b.kv_full[i], 1);
      init(&b.kv_empty[i], 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&b.tmem)), "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = b.tmem;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
    if (warp == 0) {
      // -------------------------------------------------------------- copies
      const int heads = a.Hq / a.heads, per = a.tiles;
      int first[kDirect], len[kDirect], tiles[kDirect], total = 0, most = 0;
      if (a.direct) {
        bool bad = false;
#pragma unroll
        for (int x = 0; x < kDirect; ++x) {
          const int s = lane + 32 * x;
          const int p = s < a.n ? __ldg(a.starts + s) : a.T, e = s < a.n ? __ldg(a.starts + s + 1) : a.T;
          bad |= p < 0 || e < p || e > a.T || e - p > a.longest || (s == 0 && p != 0) || (s == a.n - 1 && e != a.T);
          first[x] = p;
          len[x] = e - p;
          tiles[x] = (len[x] + per * kRows - 1) / (per * kRows);
        }
        bad = __any_sync(~0u, bad);
        if (bad && lane == 0 && blockIdx.x == 0) atomicOr(a.err, KF_DEV_BAD_ROW);
#pragma unroll
        for (int x = 0; x < kDirect; ++x) {
          if (bad) tiles[x] = 0;
          total += tiles[x];
          most = max(most, tiles[x]);
        }
        total = __reduce_add_sync(~0u, total);
        most = __reduce_max_sync(~0u, most);
      } else {
        total = __ldcg(a.plan.count);
      }
      const int items = total * heads;
      // the w-th item's {first token, tokens, tile of rows}, those of most key tiles first
      auto entry = [&](int w) -> int4 {
        if (w >= items) return make_int4(0, 0, 0, 0);
        const int u = w / heads;
        if (!a.direct) return __ldcg(reinterpret_cast<const int4*>(a.plan.item) + u);
        // tile c - 1 of the sequences of c tiles and more: after the items of higher tiles,
        // of which there are above(c); c is the least with above(c) <= u
        auto above = [&](int c) {
          int v = 0;
#pragma unroll
          for (int x = 0; x < kDirect; ++x) v += max(0, tiles[x] - c);
          return __reduce_add_sync(~0u, v);
        };
        int lo = 1, hi = most;
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (above(mid) <= u) hi = mid;
          else lo = mid + 1;
        }
        int rank = u - above(lo);
        int4 e = make_int4(0, 0, lo - 1, 0);
        bool found = false;
#pragma unroll
        for (int x = 0; x < kDirect; ++x) {
          const bool has = tiles[x] >= lo;
          const uint32_t m = __ballot_sync(~0u, has);
          const uint32_t at = __ballot_sync(~0u, !found && has && __popc(m & ((1u << lane) - 1)) == rank);
          if (at) {
            e.x = __shfl_sync(~0u, first[x], __ffs(at) - 1);
            e.y = __shfl_sync(~0u, len[x], __ffs(at) - 1);
            found = true;
          }
          rank -= __popc(m);
        }
        return e;
      };
      bool ok = true;
      int w = blockIdx.x, it = 0, q_issued = 0, g = 0, tails = 0, asks = 0, takes = 0;
      int4 e = entry(w);
      auto wait = [&](uint64_t* bar, uint32_t parity) -> bool { return __all_sync(~0u, mbar_wait(smem_u32(bar), parity, a.err)); };
      auto ask = [&] {
        __syncwarp();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (the answer before has been read)
        if (lane == 0) ask_for_cta(b.answer, &b.taken);
        ++asks;
        __syncwarp();
      };
      auto take = [&](int* cta) -> bool {
        if (!wait(&b.taken, takes++ & 1)) return false;
        *cta = cta_taken(b.answer);
        return true;
      };
      for (;; ++it) {
        Item im;
        im.start = e.x;
        im.len = e.y;
        const int hu = w % heads;
  #pragma unroll
        for (int i = 0; i < 2; ++i) {
          im.head[i] = a.heads * hu + (a.heads == 2 ? i : 0);
          const int rt = e.z * per + (a.heads == 2 ? 0 : i);
          im.row[i] = rt * kRows;
          im.n[i] = w < items && i < a.heads * a.tiles && im.row[i] < im.len ? rt + 1 : 0;
        }
        const int slot = it & 1;
        ok = wait(&b.item_empty[slot], ((it >> 1) & 1) ^ 1);
        if (!ok) break;
        if (lane == 0) {
          b.item[slot] = im;
          mbar_arrive(smem_u32(&b.item_full[slot]));
        }
        if (w >= items) {                         // (an item without sub-tiles ends the others)
          // (the grid is for the most items that the lengths could have: what is left of it need not start)
          for (int x = 0; a.steal && ok && w != INT_MAX && x >= 0;) {
            ask();
            ok = take(&x);
          }
          break;
        }
        if (a.steal) ask();
        if (it > 0) ok = wait(&b.q_empty, (it - 1) & 1);
        if (!ok) break;
        if (lane == 0) {
          mbar_expect_tx(smem_u32(&b.q_full), (im.n[1] > 0 ? 2 : 1) * TILE);
          for (int i = 0; i < 2; ++i)
            if (im.n[i] > 0)
              for (int x = 0; x < AT; ++x)
                tma_load_3d(sQ + i * TILE + x * kAtom, &maps.q, smem_u32(&b.q_full), 64 * x, im.head[i], im.start + im.row[i]);
        }
        q_issued = it + 1;
        const int n = max(im.n[0], im.n[1]), hk = im.head[0] / a.G;
        for (int j = 0; ok && j < n; ++j) {
          for (int kv = 0; kv < 2; ++kv, ++g) {
            const int st = g % ST;
            ok = wait(&b.kv_empty[st], ((g / ST) & 1) ^ 1);
            if (!ok) break;
            const uint32_t dst = sKV + st * TILE;
            // V rows past the sequence's end are another's, or nothing: their probabilities are 0,
            // and 0 times them has to be 0
            const int left = im.len - j * kKeys;
            const bool tail = kv == 1 && left < kKeys;
            uint64_t* bar = tail ? &b.tail : &b.kv_full[st];
            if (lane == 0) {
              mbar_expect_tx(smem_u32(bar), TILE);
              for (int x = 0; x < AT; ++x)
                tma_load_3d(dst + x * kAtom, kv ? &maps.v : &maps.k, smem_u32(bar), 64 * x, hk, im.start + j * kKeys);
            }
            __syncwarp();
            if (tail) {
              ok = wait(&b.tail, tails++ & 1);
              if (!ok) break;
              uint8_t* p = sm + (2 + st) * TILE;
              for (int x = 0; x < AT; ++x)
                for (int i = left * 128 + lane * 16; i < kKeys * 128; i += 32 * 16)
                  *reinterpret_cast<uint4*>(p + x * kAtom + i) = make_uint4(0u, 0u, 0u, 0u);
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) mbar_arrive(smem_u32(&b.kv_full[st]));
            }
          }
        }
        if (!ok) break;
        int next = -1;
        if (a.steal) ok = take(&next);
        if (!ok) break;
        w = next < 0 ? INT_MAX : next;
        e = entry(w);
      }
      if (!ok && lane == 0) {
        // let the copies still in flight land before the CTA ends (bounded)
        if (q_issued) mbar_wait(smem_u32(&b.q_full), (q_issued - 1) & 1, a.err);
        if (asks > takes) mbar_wait(smem_u32(&b.taken), takes & 1, a.err);
        for (int i = max(0, g - ST); i < g; ++i) mbar_wait(smem_u32(&b.kv_full[i % ST]), (i / ST) & 1, a.err);
      }
      __syncwarp();
    } else if (warp == 1) {
      product_warp<T, HD>(b, tmem, sQ, sKV, lane, a.err);
      __syncwarp();
    }
  } else {
    // ------------------------------------------------------------- softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    const int sub = warp >= 8, quarter = warp & 3, row = 32 * quarter + lane;
    const Softmax<T, HD> sx(tmem, sub, quarter, lane);
    const uint32_t tO = sx.tO;
    const float sc = a.scale2;
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool { return __all_sync(~0u, mbar_wait(smem_u32(bar), parity, a.err)); };
    auto arrive = [&](uint64_t* bar) {
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(bar));
    };
    int g = 0;                                  // this sub-tile's key tiles so far
    bool ok = true;
    for (int it = 0; ok; ++it) {
      const int slot = it & 1;
      if (!wait(&b.item_full[slot], (it >> 1) & 1)) break;
      const Item im = b.item[slot];
      arrive(&b.item_empty[slot]);
      if (im.n[0] == 0 && im.n[1] == 0) break;
      const int n = im.n[sub];
      if (n == 0) continue;
      float m = -INFINITY, l = 0.f;             // the reference (raw score), the sum
      for (int j = 0; j < n; ++j, ++g) {
        ok = sx.tile(b, sc, j == 0, g, m, l, a.err, [&](int c, uint32_t* s) {
          if (j == n - 1 && c >= quarter) {     // the diagonal tile: keys 0 .. row
            const int lim = c == quarter ? lane : -1;
#pragma unroll
            for (int e = 0; e < 32; ++e) s[e] = e <= lim ? s[e] : 0xff800000u;
          }
        });
        if (!ok) break;
      }
      if (!ok) break;
      if (!wait(&b.o_full[sub], (g - 1) & 1)) { ok = false; break; }
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const float inv = 1.f / l;
      const bool mine = im.row[sub] + row < im.len;
      T* dst = static_cast<T*>(a.out) + (int64_t)(im.start + im.row[sub] + row) * a.out_row + im.head[sub] * a.out_head;
      const bool wide = (reinterpret_cast<uintptr_t>(dst) & 31) == 0;
#pragma unroll
      for (int c = 0; c < HD / 32; ++c) {
        float o[32];
        tmem_ld32(tO + 32 * c, o);
        if (c == HD / 32 - 1) {
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          arrive(&b.o_free[sub]);
        }
        if (mine) {
          uint32_t pk[16];
#pragma unroll
          for (int d = 0; d < 16; ++d) pk[d] = pack2<T>(o[2 * d] * inv, o[2 * d + 1] * inv);
          if (wide) {
            st_32(dst + 32 * c, pk);
            st_32(dst + 32 * c + 16, pk + 8);
          } else {
#pragma unroll
            for (int d = 0; d < 16; d += 4)
              *reinterpret_cast<uint4*>(dst + 32 * c + 2 * d) = make_uint4(pk[d], pk[d + 1], pk[d + 2], pk[d + 3]);
          }
        }
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

// [T][heads][hd] as boxes of 128 tokens x 64 elements of one head
bool head_map(CUtensorMap* m, const void* p, int64_t T, int heads, int hd, int64_t row, int64_t head) {
  const uint64_t dims[3] = {(uint64_t)hd, (uint64_t)heads, (uint64_t)T};
  const uint64_t strides[2] = {(uint64_t)head * 2, (uint64_t)row * 2};
  const uint32_t box[3] = {64, 1, kRows};
  return encode_map_bf16(m, p, 3, dims, strides, box);      // (fp16 is copied the same way)
}

template <typename T, int HD>
int launch(const Maps& maps, const Args& a, int grid, cudaStream_t s) {
  static PerDevice attr;
  set_smem_attr(attr, k_prompt<T, HD>, kSmem<HD>);
  launch_cluster(k_prompt<T, HD>, dim3(grid), dim3(kThreads), kSmem<HD>, 1, !a.direct, s, maps, a);
  return launched("kf_op_prompt_attention");
}
int64_t plan_items(int n, int64_t T) { return T / kRows + n; }
bool without_plan(int n) { return n <= 32 * kDirect; }

}  // namespace
}  // namespace kf

using namespace kf;

extern "C" int64_t kf_op_prompt_attention_work(int32_t n, int64_t T) {
  return n < 0 || T < 0 || without_plan(n) ? 0 : 256 + plan_items(n, T) * (int64_t)sizeof(PlanItem);
}

extern "C" int kf_op_prompt_attention(int32_t type, int32_t n, int64_t T, int32_t longest, int32_t Hq, int32_t Hkv, int32_t hd,
                                      const void* q, int64_t q_row, int64_t q_head, const void* k, int64_t k_row, int64_t k_head,
                                      const void* v, int64_t v_row, int64_t v_head, void* out, int64_t out_row, int64_t out_head,
                                      const int32_t* starts, float scale, void* work, void* stream) {
  const char* what = "kf_op_prompt_attention";
  if (type != KF_TYPE_BF16 && type != KF_TYPE_FP16) return refuse(what, "the type is bf16 or fp16");
  if (hd != 64 && hd != 128) return refuse(what, "head_dim is 64 or 128");
  if (n < 0 || T < 0 || T > (1 << 30) || longest < 0 || longest > kMaxTiles * kRows) return refuse(what, "sequences or tokens out of range (a sequence has at most 524288)");
  if (Hkv < 1 || Hq < 1 || Hq % Hkv || Hq > 4096) return refuse(what, "heads out of range");
  if (!(scale > 0.f) || std::isinf(scale)) return refuse(what, "scale is a positive number");
  if (n == 0 || T == 0) return n == 0 && T > 0 ? refuse(what, "tokens of no sequence") : KF_OK;
  if (!q || !k || !v || !out || !starts || (!work && !without_plan(n))) return refuse(what, "a null array");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(starts, 4) || !aligned(work, 256))
    return refuse(what, "q, k, v and out are 16-byte aligned, work 256-byte");
  for (const int64_t st : {q_row, q_head, k_row, k_head, v_row, v_head, out_row, out_head})
    if (st % 8 || st < 0 || st > (1ll << 37)) return refuse(what, "strides are multiples of 8 elements");
  const int64_t cap = plan_items(n, T);
  if (cap * Hq > 0x7fffffff - 4096) return refuse(what, "too many rows and heads");
  Maps maps;
  if (!head_map(&maps.q, q, T, Hq, hd, q_row, q_head) || !head_map(&maps.k, k, T, Hkv, hd, k_row, k_head) ||
      !head_map(&maps.v, v, T, Hkv, hd, v_row, v_head))
    return refuse(what, "a tensor map is refused (strides)");
  int* err = serving_error_word();
  if (!err) return refuse(what, "no error word", KF_E_CUDA);
  const int G = Hq / Hkv;
  // One sub-tile an item where that ends sooner: a key tile then takes kAlone clocks, in pairs kPaired for both, and
  // an item kItem more.  Where few long items leave SMs idle the longest item's chain is what a call takes (one of 4096, 8
  // heads of 64: 41.4 us alone, 51.1 in pairs; one of 7074: 109.6 and 82.9).  (Lengths are on the device: the
  // estimate takes equal ones, and `longest` for the chain.  That is only a bound, so what the longer chain would
  // gain alone is set against what is lost if all sequences have the mean length: 64 of 512, 32 heads over 8 of 128, at
  // a bound of 131,072: 283 us alone, 184 in pairs; 1,606 and 3,063, 8 heads of 128: 52.1 and 42.9.)
  const double kAlone = hd == 64 ? 2050 : 2800, kPaired = hd == 64 ? 2600 : 2860, kItem = 2500;
  const double tiles = std::max<double>(1, (double)T / n / kRows);
  const double items = n * (double)Hq * tiles / device_sms();      // sub-tiles of an SM
  auto alone_by = [&](double chain) {                              // the time in pairs over that alone
    return std::max(chain * kPaired, items / 2 * ((tiles + 1) / 2 * kPaired + kItem)) / std::max(chain * kAlone, items * ((tiles + 1) / 2 * kAlone + kItem));
  };
  const double by_bound = alone_by(std::max<double>(1, (double)std::min<int64_t>(longest, T) / kRows)), by_mean = alone_by(tiles);
  const bool alone = by_bound > 1 && by_bound * by_mean >= 1;
  const int heads = !alone && G % 2 == 0 ? 2 : 1, rows = alone || heads == 2 ? kRows : 2 * kRows;
  const int classes = std::max(1, ceil_div(longest, rows));
  const int direct = without_plan(n);
  int* head = static_cast<int*>(work);
  const Plan plan{head, reinterpret_cast<PlanItem*>(head + 64)};
  const int64_t most = (T / rows + n) * (Hq / heads);      // items, by the lengths' sum
  const int steal = most > device_sms();
  const int grid = (int)(steal ? most : std::min<int64_t>(device_sms(), most));
  cudaStream_t s = (cudaStream_t)stream;
  if (!direct) launch_cluster(k_plan, dim3(1), dim3(kPlanThreads), 2 * (classes + 2) * sizeof(int), 1, false, s, n, (int)T, longest, rows, classes,
                 starts, plan, err);
  if (const int rc = launched(what)) return rc;
  const Args a{out, out_row, out_head, plan, err, Hq, G, heads, rows / kRows, direct, steal, n, (int)T, longest, starts, scale * 1.4426950408889634f};
  if (type == KF_TYPE_BF16) return hd == 64 ? launch<__nv_bfloat16, 64>(maps, a, grid, s) : launch<__nv_bfloat16, 128>(maps, a, grid, s);
  return hd == 64 ? launch<__half, 64>(maps, a, grid, s) : launch<__half, 128>(maps, a, grid, s);
}
