// Attention of groups of sequences that begin with the same tokens (kf_op_shared_attention): head_dim 64
// or 128, bf16 or fp16; the prefixes on tcgen05 (kf_attn_pair.cuh), the sum of all parts, and what reads which call's prefixes.
//
// The query rows that read a group's prefix under one KV head are its sequences' rows x group heads: a
// segment is up to 256 of them, two sub-tiles of 128, over all key tiles of 128 of the prefix.  So
// a prefix comes from memory once for all of a group's sequences.  The segments' tiles form one list which the
// CTAs (one a SM) share evenly, kExtra tiles more a segment for its start and end; what a part leaves
// unfinished the last kernel adds (kf_shared.cuh).  K and V come by TMA, in boxes of the 16 keys that a page is a multiple of
// (boxes of 128 rows were no faster); a page outside of the pool is a box outside of the map, which is zeros and closed by the
// softmax.  Each row sees keys up to its own position.
// What bounds it: long prefixes their bytes, beside 2,900 clocks of tensor cores and exponentials a tile of 256 rows (64 KB at
// head_dim 128, for which memory takes 2,800); short ones the first run through the code and the items' starts and ends: the first
// product starts 5 us after the launch, and an item more in a CTA costs what three tiles do.
// Measured (GPU time, floor of the bytes): 64 answers about 32,771 tokens, 32 heads over 8 of 128, in 69 us (40; all CTAs on the
// prefix first 75); 8 groups of 16 after 1,003 to 4,099 tokens 61 us (40; 66); joint steps of eight rows, 16 groups of 16 after 128 to 896, 12 heads over 4 of
// 64, 37 us (5); 8 candidates of one prompt of 517, by paged attention, 7.4 us.  Not kept: a single sub-tile's scores in both
// sub-tiles' columns in turn, so that the next S runs under the softmax (66 us both, the document 75 -> 78).
#include <algorithm>

#include "kf_attn_pair.cuh"
#include "kf_shared.cuh"

namespace kf {
namespace {
using namespace pair;

constexpr int kGran = 16, kGrans = kKeys / kGran;    // keys of a box; boxes of a tile
constexpr int kPrefixRows = 256;                     // query rows of a segment
constexpr int kExtra = 3;                            // a segment's start and end, in tiles
constexpr float kAhead = 1.3f;                       // see Walk::ctas
constexpr float kTileUnits = 9.f;                    // units of own keys (8 KB of K and V) that take as long as a tile of a prefix
// Sequences whose lengths are added up (by one warp of each CTA).  Of more there is work for all SMs on either side, and the
// adding costs more than the split wins: 80 groups of 16 after 1,003 to 4,099 tokens 475 us without and 482 with, 256 of 16 983 and 1,130, 8 of
// 256 after 4,000 to 16,000 449 and 505; joint steps of 80 groups of 16 134 and 142
constexpr int kMostCounted = 1024;
constexpr int kMinTiles = 2;                         // places of a CTA, at least

struct Item {
  int b0, first, rows;                               // the group's first sequence; the segment's first row, and its rows
  int hk, t0, len;                                   // KV head, first key tile, the prefix's tokens
  int n[2];                                          // key tiles (0: no sub-tile)
  int more;                                          // a later piece of its segment
};
// row r of an item: its sequence of the group, token of that and head of the KV head's
struct Row {
  int seq, tok, j;
  __device__ __forceinline__ Row(const SharedCall& a, const Item& im, int r) {
    const int R = im.first + r;
    seq = a.by_seq.of(R);
    const int x = R - seq * (int)a.by_seq.d;
    tok = a.by_group.of(x);
    j = x - tok * a.G;
  }
};
using Bars = PairBars<Item>;
static_assert(sizeof(Bars) <= kBarBytes, "the barriers' part of the shared memory");

// Places of a group: pairs of sub-tiles x KV heads x (tiles + kExtra)
struct Group {
  int b0, rows, len, tiles, pairs;
  int64_t before;                                    // rows a head before the group
  __device__ __forceinline__ Group(const SharedCall& a, int g) {
    const int2 m = members(a.sh, g, a.B);
    b0 = m.x;
    rows = (m.y - m.x) * a.rows * a.G;
    before = (int64_t)m.x * a.rows * a.G;
    len = prefix_of(a.sh, g, a.width * a.page);
    tiles = (len + kKeys - 1) / kKeys;
    pairs = tiles > 0 ? (rows + kPrefixRows - 1) / kPrefixRows : 0;
  }
  __device__ __forceinline__ int places(const SharedCall& a) const { return pairs * a.Hkv * (tiles + kExtra); }
};

// A CTA's pieces of segments, in order (by the load warp, uniform)
struct Walk {
  Parts parts;
  int x, x1, base, g;            // the next place, the part's end; the group that it lies in, whose places begin at base
  int at, pieces;                // of the piece: its segment's record, and the CTAs that have pieces of it
  // The CTAs that take parts; those of the kernel after this one, for each sequence's own keys, start on the SMs of the others.  This one
  // has kAhead of its share of all work, so that it ends before the other does (1.1, 1.3, 1.5: 62.6, 61.8, 66.4 us for the
  // groups above, 74.1, 69.9, 73.5 for the document)
  static __device__ __forceinline__ int ctas(const SharedCall& a, int lane, int total) {
    if (a.B > kMostCounted) return gridDim.x;
    float keys = 0.f;                           // of the sequences after their prefixes
#pragma unroll 4
    for (int b = lane; b < a.B; b += 32) keys += (float)min(max(__ldg(a.lens + b), 0), a.width * a.page);
    for (int i = lane; i < a.sh.n; i += 32) {
      const Group gr(a, i);
      keys -= (float)gr.len * a.by_seq.of(gr.rows);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) keys += __shfl_xor_sync(~0u, keys, o);
    const float tiles = (float)((a.rows * a.G + a.own.seg_rows - 1) / a.own.seg_rows * a.Hkv);
    const float own = tiles * (fmaxf(keys, 0.f) * (a.hd / 2048.f) + 3.f * a.B) / kTileUnits;      // in tiles of a prefix
    return min((int)gridDim.x, max((int)gridDim.x / 3, (int)(gridDim.x * (kAhead * total / (total + own)) + 1.f)));
  }
  __device__ __forceinline__ void start(const SharedCall& a, int lane) {
    base = g = 0;
    const int mine = lane < a.sh.n ? Group(a, lane).places(a) : 0;
    int total = __reduce_add_sync(~0u, mine);
    for (int i = 32; i < a.sh.n; i += 32) total += __reduce_add_sync(~0u, i + lane < a.sh.n ? Group(a, i + lane).places(a) : 0);
    parts = Parts(total, min(ctas(a, lane, total), max(1, total / kMinTiles)));
    x = parts.begin(blockIdx.x);
    x1 = parts.begin(blockIdx.x + 1);
    for (int i = 0; x < x1 && i < a.sh.n; i += 32) {
      const int v = i == 0 ? mine : i + lane < a.sh.n ? Group(a, i + lane).places(a) : 0;
      int incl = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(~0u, incl, o);
        if (lane >= o) incl += u;
      }
      const uint32_t past = __ballot_sync(~0u, base + incl > x);
      if (past) {
        const int l = __ffs(past) - 1;
        base += __shfl_sync(~0u, incl - v, l);
        g = i + l;
        break;
      }
      base += __shfl_sync(~0u, incl, 31);
    }
  }
  // the next piece; one without tiles past the last
  __device__ __forceinline__ Item next(const SharedCall& a) {
    Item im{};
    while (x < x1) {
      const Group gr(a, g);
      const int per = gr.tiles + kExtra, places = gr.places(a);
      if (x >= base + places) {                 // (also a group without places)
        base += places;
        if (++g >= a.sh.n) break;
        continue;
      }
      // a segment: pair by pair, head by head
      const int s = (x - base) / per, pair = s / a.Hkv, hk = s - pair * a.Hkv;
      const int xs = base + s * per, end = xs + gr.tiles, t0 = x - xs, n = min(end, x1) - x;
      x = min(xs + per, x1);
      if (n <= 0) continue;                     // only places of its end
      im.b0 = gr.b0;
      im.first = pair * kPrefixRows;
      im.rows = min(kPrefixRows, gr.rows - im.first);
      im.hk = hk;
      im.t0 = t0;
      im.len = gr.len;
      im.n[0] = n;
      im.n[1] = im.rows > kRows ? n : 0;
      im.more = t0 > 0;
      at = prefix_record(gr.before, g, pair, kPrefixRows, hk, a.Hkv);
      pieces = parts.part_of(end - 1) - blockIdx.x + 1;      // (parts up to the one of the segment's last tile)
      break;
    }
    return im;
  }
};

template <typename T, int HD>
__global__ void __launch_bounds__(kThreads, 1) k_prefix(const __grid_constant__ CUtensorMap map, const SharedCall a) {
  extern __shared__ __align__(1024) uint8_t sm[];
  constexpr int ST = kStages<HD>, AT = HD / 64;
  constexpr uint32_t TILE = kTile<HD>;
  Bars& b = *reinterpret_cast<Bars*>(sm + (2 + ST) * TILE);
  const uint32_t sQ = smem_u32(sm), sKV = sQ + 2 * TILE;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (sQ & 1023) {                              // (uniform) swizzle atoms need the alignment
    if (t == 0) atomicOr(a.err, kErrInternal);
    return;
  }
  if (t == 64) {
    auto init = [](uint64_t* p, uint32_t n) { mbar_init(smem_u32(p), n); };
    init(&b.q_full, 8);                         // the softmax warps, which copy Q
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
    for (int i = 0; i < ST; ++i) {
      init(&b.kv_full[i], 1);
      init(&b.kv_empty[i], 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // the load warp finds the first item, and its first tile's pages, before the barrier
  Walk walk;
  Item im;
  int id = -1;
  // lane x < 8 looks up box x of a tile
  auto look = [&](int tile) -> int {
    const int key = tile * kKeys + lane * kGran;
    return lane < kGrans && key < im.len ? __ldg(a.table + (int64_t)im.b0 * a.width + a.by_page.of(key)) : -1;
  };
  if (warp == 0) {
    walk.start(a, lane);
    im = walk.next(a);
    if (lane == 0) b.item[0] = im;
    if (im.n[0] > 0) id = look(im.t0);
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
  if (blockIdx.x > 0 && b.item[0].n[0] == 0) {      // (uniform) no part: the SM is the next kernel's
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    return;
  }

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
    if (warp == 0) {
      // ------------------------------------------------------ items and copies
      bool ok = true;
      int ring = 0, tails = 0;
      auto wait = [&](uint64_t* bar, uint32_t parity) -> bool { return __all_sync(~0u, mbar_wait(smem_u32(bar), parity, a.err)); };
      for (int it = 0;; ++it) {
        const int slot = it & 1;
        if (it > 0) {
          im = walk.next(a);
          ok = wait(&b.item_empty[slot], ((it >> 1) & 1) ^ 1);
          if (!ok) break;
          if (lane == 0) b.item[slot] = im;
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(smem_u32(&b.item_full[slot]));
        if (im.n[0] == 0) break;                // (an item without sub-tiles ends the others)
        if (it > 0) id = look(im.t0);
        if (lane == 0 && !im.more && walk.at < a.pre.segments) a.pre.rec[walk.at] = Record{(int)blockIdx.x, walk.pieces};
        const int t0 = im.t0, n = im.n[0], hk = im.hk;
        for (int j = t0; ok && j < t0 + n; ++j) {
          const int key = j * kKeys + lane * kGran, left = im.len - j * kKeys;
          // (a box outside of the map: zeros)
          const bool in = id >= 0 && id < a.n_pages;
          const int page = in ? id : (int)a.n_pages, row = in ? key - a.by_page.of(key) * a.page : 0;
          if (lane < kGrans && key < im.len && !in) atomicOr(a.err, KF_DEV_BAD_PAGE);
          if (j + 1 < t0 + n) id = look(j + 1);
          for (int kv = 0; ok && kv < 2; ++kv, ++ring) {
            const int st = ring % ST;
            ok = wait(&b.kv_empty[st], ((ring / ST) & 1) ^ 1);
            if (!ok) break;
            const uint32_t dst = sKV + st * TILE;
            // V rows past the prefix's end: their probabilities are 0, and 0 times them has to be 0
            const bool tail = kv == 1 && left < kKeys && left % kGran != 0;
            uint64_t* bar = tail ? &b.tail : &b.kv_full[st];
            if (lane == 0) mbar_expect_tx(smem_u32(bar), TILE);
            __syncwarp();
            if (lane < kGrans)
              for (int y = 0; y < AT; ++y)
                tma_load_4d(dst + y * kAtom + lane * kGran * 128, &map, smem_u32(bar), 64 * y, row, kv * a.Hkv + hk, page);
            __syncwarp();
            if (tail) {
              ok = wait(&b.tail, tails++ & 1);
              if (!ok) break;
              uint8_t* p = sm + (2 + st) * TILE;
              const int to = (left + kGran - 1) / kGran * kGran * 128;
              for (int y = 0; y < AT; ++y)
                for (int i = left * 128 + lane * 16; i < to; i += 32 * 16)
                  *reinterpret_cast<uint4*>(p + y * kAtom + i) = make_uint4(0u, 0u, 0u, 0u);
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) mbar_arrive(smem_u32(&b.kv_full[st]));
            }
          }
        }
        if (!ok) break;
      }
      if (blockIdx.x == 0) {
        bool bad = false;
        for (int i = lane; i < a.sh.n; i += 32) {
          const int p = a.sh.groups[i], e = a.sh.groups[i + 1], n = a.sh.shared[i];
          bad |= p < 0 || e < p || e > a.B || (i == 0 && p != 0) || (i == a.sh.n - 1 && e != a.B) || n < 0 || n > a.width * a.page;
        }
        if (__any_sync(~0u, bad) && lane == 0) atomicOr(a.err, KF_DEV_BAD_ROW);
      }
      if (!ok && lane == 0)
        // let the copies still in flight land before the CTA ends (bounded)
        for (int i = max(0, ring - ST); i < ring; ++i) mbar_wait(smem_u32(&b.kv_full[i % ST]), (i / ST) & 1, a.err);
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
      if (im.n[0] == 0) break;
      const int n = im.n[sub];
      if (it > 0) ok = wait(&b.q_empty, (it - 1) & 1);
      if (!ok) break;
      if (n > 0) {
        // this warp's 32 rows of Q, swizzled; rows that the segment does not have are zeros
        constexpr int CH = HD / 8, RP = 32 / CH;
        const int ch = lane % CH;
#pragma unroll 2
        for (int p = 0; p < CH; ++p) {
          const int lr = 32 * quarter + p * RP + lane / CH, r = sub * kRows + lr;
          const Row w(a, im, r);
          const T* from = static_cast<const T*>(a.q) + (im.b0 + w.seq) * a.q_seq + w.tok * a.q_row + (int64_t)(im.hk * a.G + w.j) * a.q_head + 8 * ch;
          const bool in = r < im.rows;
          mma::cp_async16(sQ + sub * TILE + (ch / 8) * kAtom + lr * 128 + (((ch % 8) ^ (lr & 7)) << 4), in ? from : static_cast<const T*>(a.q), in ? 16 : 0);
        }
        mma::cp_commit();
        mma::cp_wait<0>();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      }
      arrive(&b.q_full);
      if (n == 0) continue;
      // this thread's row: its place among all rows, and the keys that it sees
      const int r = sub * kRows + row;
      const Row w(a, im, r);
      const bool mine = r < im.rows;
      int see = 0x7fffffff;                     // (a row that is not there, of zeros, asks for no mask)
      if (mine) see = min(im.len, min(max(__ldg(a.lens + im.b0 + w.seq), 0), a.width * a.page) - a.rows + w.tok + 1);
      const int32_t* ids = a.table + (int64_t)im.b0 * a.width;
      auto look = [&](int tile) -> int {        // the tile's page of box `lane`
        const int key = tile * kKeys + lane * kGran;
        return lane < kGrans && key < im.len ? __ldg(ids + a.by_page.of(key)) : 0;
      };
      int id = look(im.t0);
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < n; ++j, ++g) {
        const uint32_t open = __ballot_sync(~0u, id >= 0 && id < a.n_pages);
        if (j + 1 < n) id = look(im.t0 + j + 1);
        const int lim = see - (im.t0 + j) * kKeys;      // keys below it are seen
        const bool all = open == ~0u && __all_sync(~0u, lim >= kKeys);
        ok = sx.short_tile(b, sc, j == 0, g, m, l, a.err, [&](int c, uint32_t* s) {
          if (!all) {
            const int lc = lim - 64 * c;
#pragma unroll
            for (int e = 0; e < 64; ++e) s[e] = e < lc && ((open >> (4 * c + e / 16)) & 1u) ? s[e] : 0xff800000u;
          }
        });
        if (!ok) break;
      }
      if (!ok) break;
      if (!wait(&b.o_full[sub], (g - 1) & 1)) { ok = false; break; }
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int64_t at = im.more ? (int64_t)blockIdx.x * kPrefixRows + r
                                 : ((int64_t)(im.b0 + w.seq) * a.rows + w.tok) * a.Hq + im.hk * a.G + w.j;
      float* dst = (im.more ? a.pre.more_o : a.pre.first_o) + at * HD;
      if (mine) (im.more ? a.pre.more_ml : a.pre.first_ml)[at] = make_float2(m, l);
#pragma unroll 1
      for (int c = 0; c < HD / 32; ++c) {
        float o[32];
        tmem_ld32(sx.tO + 32 * c, o);
        if (c == HD / 32 - 1) {
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          arrive(&b.o_free[sub]);
        }
        if (mine) {
#pragma unroll
          for (int d = 0; d < 32; d += 8) st_32(dst + 32 * c + d, reinterpret_cast<const uint32_t*>(o + d));
        }
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

// The pieces of a query row added, those of its group's prefix and those of its sequence's own keys: HD / 8 lanes a row, so that
// many rows are one wave of blocks; of few rows W times as many lanes share the pieces (each every W-th; their sums then in order).
// What a call takes here is a chain of loads: the first pieces, whose places need no record, come with the records
constexpr int kJoinThreads = 256;
template <typename T, int HD>
__global__ void __launch_bounds__(kJoinThreads) k_add(const __grid_constant__ SharedCall a, int W) {
  constexpr int LANES = HD / 8, GR = kJoinThreads / LANES;      // of a row; rows' worth of lanes in a block
  __shared__ float4 so[GR][2][LANES];
  __shared__ float2 sml[GR];
  const int v = threadIdx.x % LANES, gr = threadIdx.x / LANES, part = gr % W;
  const int rows = a.B * a.rows * a.Hq, at = min(rows - 1, (int)blockIdx.x * (GR / W) + gr / W);
  const int bt = a.by_heads.of(at), h = at - bt * a.Hq, b = a.by_rows.of(bt), tok = bt - b * a.rows;
  const int hk = a.by_group.of(h), r = tok * a.G + h - hk * a.G;
  const int g = group_of(a.sh, b);
  const int2 in = members(a.sh, g, a.B);
  const bool prefixed = b >= in.x && b < in.y && prefix_of(a.sh, g, a.width * a.page) > 0;
  const int x = (b - in.x) * a.rows * a.G + r;
  // (segments have 16, 32 or 256 rows)
  const int own_shift = a.own.seg_rows == 16 ? 4 : 5, pre_shift = a.pre.seg_rows == 256 ? 8 : own_shift;
  const int MT = (a.rows * a.G + a.own.seg_rows - 1) >> own_shift;
  const int own_rec = (b * a.Hkv + hk) * MT + (r >> own_shift);
  const int pre_rec = prefixed ? min(a.pre.segments - 1, prefix_record((int64_t)in.x * a.rows * a.G, g, x >> pre_shift, a.pre.seg_rows, hk, a.Hkv)) : 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // (written by the kernels before this one: not through the read-only path; a record of groups that are not as they
  // should be may hold anything)
  const int2 own = __ldcg(reinterpret_cast<const int2*>(a.own.rec) + own_rec);
  const int2 pre = prefixed ? __ldcg(reinterpret_cast<const int2*>(a.pre.rec) + pre_rec) : make_int2(0, 0);
  float m = -INFINITY, l = 0.f;
  float4 o0 = make_float4(0.f, 0.f, 0.f, 0.f), o1 = o0;
  auto add = [&](float2 ml, float4 y0, float4 y1) {
    const float mm = fmaxf(m, ml.x);
    const float fa = m == -INFINITY ? 0.f : mma::ex2((m - mm) * a.scale2), fb = ml.x == -INFINITY ? 0.f : mma::ex2((ml.x - mm) * a.scale2);
    m = mm;
    l = l * fa + ml.y * fb;
    o0 = make_float4(o0.x * fa + y0.x * fb, o0.y * fa + y0.y * fb, o0.z * fa + y0.z * fb, o0.w * fa + y0.w * fb);
    o1 = make_float4(o1.x * fa + y1.x * fb, o1.y * fa + y1.y * fb, o1.z * fa + y1.z * fb, o1.w * fa + y1.w * fb);
  };
  auto piece = [&](const float* po, const float2* pml, int64_t q) {
    const float4* y = reinterpret_cast<const float4*>(po + q * HD) + 2 * v;
    add(__ldcg(pml + q), __ldcg(y), __ldcg(y + 1));
  };
  auto later = [&](const Partials& p, int2 rc, int row) {
    const int c = max(rc.x, 0), n = min(p.parts - c, rc.y);
#pragma unroll 4
    for (int i = part > 0 ? part : W; i < n; i += W) piece(p.more_o, p.more_ml, (int64_t)(c + i) * p.seg_rows + row);
  };
  if (part == 0) {
    piece(a.own.first_o, a.own.first_ml, at);
    if (prefixed) piece(a.pre.first_o, a.pre.first_ml, at);
  }
  later(a.own, own, r & (a.own.seg_rows - 1));
  if (prefixed) later(a.pre, pre, x & (a.pre.seg_rows - 1));
  if (W > 1) {                                  // (uniform)
    so[gr][0][v] = o0;
    so[gr][1][v] = o1;
    if (v == 0) sml[gr] = make_float2(m, l);
    __syncthreads();
    if (part != 0) return;
    for (int i = 1; i < W; ++i) add(sml[gr + i], so[gr + i][0][v], so[gr + i][1][v]);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;   // (no key seen: zeros)
  reinterpret_cast<uint4*>(static_cast<T*>(a.out) + (int64_t)at * HD)[v] =
      make_uint4(pack2<T>(o0.x * inv, o0.y * inv), pack2<T>(o0.z * inv, o0.w * inv), pack2<T>(o1.x * inv, o1.y * inv), pack2<T>(o1.z * inv, o1.w * inv));
}

// ------------------------------------------------------------------ host
template <typename T, int HD>
int launch(int32_t type, const SharedCall& c, bool tiles, const CUtensorMap& map, cudaStream_t s) {
  if (tiles) {
    static PerDevice attr;
    set_smem_attr(attr, k_prefix<T, HD>, kSmem<HD>);
    launch_cluster(k_prefix<T, HD>, dim3(c.pre.parts), dim3(kThreads), kSmem<HD>, 1, false, s, map, c);
  }
  launch_rows(type, c, !tiles, s);
  // lanes for every second piece that a row may have, as far as they fit the SMs at once
  const int64_t rows = (int64_t)c.B * c.rows * c.Hq;
  constexpr int GR = kJoinThreads / (HD / 8);
  const int pieces = c.own.parts / c.own.segments + c.pre.parts / c.pre.segments;
  int W = 1;
  while (W < 8 && W * 4 <= pieces && rows * (HD / 8) * W * 2 <= (int64_t)device_sms() * 2048) W *= 2;
  const int64_t per = GR / W;
  launch_cluster(k_add<T, HD>, dim3((unsigned)((rows + per - 1) / per)), dim3(kJoinThreads), 0, 1, true, s, c, W);
  return launched("kf_op_shared_attention");
}

// pages of K and V heads of rows, in boxes of 16 rows x 64 elements
bool pool_map(CUtensorMap* m, const void* pool, int64_t n_pages, int Hkv, int page, int hd) {
  const uint64_t dims[4] = {(uint64_t)hd, (uint64_t)page, (uint64_t)2 * Hkv, (uint64_t)n_pages};
  const uint64_t strides[3] = {(uint64_t)hd * 2, (uint64_t)page * hd * 2, (uint64_t)2 * Hkv * page * hd * 2};
  const uint32_t box[4] = {64, kGran, 1, 1};
  return encode_map_bf16(m, pool, 4, dims, strides, box);      // (fp16 is copied the same way)
}

// The scratch, in 256-byte pieces; its size where work is NULL.  tiles: the prefixes on tcgen05
int64_t layout(SharedCall& c, bool tiles, void* work) {
  int64_t at = 0;
  auto take = [&](int64_t bytes) -> void* {
    const int64_t p = at;
    at += (bytes + 255) / 256 * 256;
    return static_cast<uint8_t*>(work) + p;
  };
  const int64_t rows = (int64_t)c.B * c.rows * c.Hq, per = c.rows * c.G;
  const RowsPlan own = plan_rows((int)per, c.hd);
  c.own.parts = own.parts;
  c.own.seg_rows = own.seg_rows;
  c.own.segments = (int)((int64_t)c.B * c.Hkv * ceil_div((int)per, own.seg_rows));
  c.pre.seg_rows = tiles ? kPrefixRows : own.seg_rows;
  const int64_t pre_tiles = c.B * per / c.pre.seg_rows + c.sh.n;
  c.pre.segments = (int)((pre_tiles + 1) * c.Hkv);
  // no more CTAs than the longest list that the table could hold fills
  const int64_t places = pre_tiles * c.Hkv * (((int64_t)c.width * c.page + kKeys - 1) / kKeys + kExtra);
  c.pre.parts = tiles ? (int)std::max<int64_t>(1, std::min<int64_t>(device_sms(), places / kMinTiles)) : own.parts;
  for (Partials* p : {&c.own, &c.pre}) {
    p->first_o = static_cast<float*>(take(rows * c.hd * (int64_t)sizeof(float)));
    p->first_ml = static_cast<float2*>(take(rows * (int64_t)sizeof(float2)));
    p->rec = static_cast<Record*>(take(p->segments * (int64_t)sizeof(Record)));
    if (p == &c.pre && !tiles) {                // (a part has one later piece, of either kind)
      p->more_o = c.own.more_o;
      p->more_ml = c.own.more_ml;
    } else {
      p->more_o = static_cast<float*>(take((int64_t)p->parts * p->seg_rows * c.hd * (int64_t)sizeof(float)));
      p->more_ml = static_cast<float2*>(take((int64_t)p->parts * p->seg_rows * (int64_t)sizeof(float2)));
    }
  }
  return at;
}
const char* sizes_fault(int B, int rows, int Hq, int Hkv, int hd, int page, int width, int n) {
  if (const char* f = paged_sizes_fault(B, rows, Hq, Hkv, hd, page, width)) return f;
  if (n < 0 || (B > 0 && n < 1)) return "groups out of range";
  return nullptr;
}
// whether places, records and rows of these sizes can be counted in 31 bits
bool countable(int B, int rows, int G, int Hkv, int page, int width, int n) {
  const int64_t tiles = 2 * ((int64_t)B * ceil_div(rows * G, 16) + n + 1) * Hkv;      // of 16 rows, over prefixes and own keys
  return n <= (1 << 24) && (int64_t)B * rows * G * Hkv <= (1 << 30) && tiles <= (1 << 30) && tiles * ((int64_t)width * page / 16 + 8) <= 0x7fffffff;
}
// What reads a call's prefixes.  The lengths are on the device, so the rule takes what the table and the pool could hold.  (Short prefixes in
// a table of a model's longest context so go a slower way than they could: eight candidates after 517 tokens, 12 heads over 4 of 64, in tables of
// 592 to 4,096, 8,192 to 32,768 and 131,072 tokens 7.5, 10.4 and 13.0 us; 32 over 8 of 128 in 1,024, 8,192 and 131,072 10.5, 11.1 and 14.5.)
//   paged attention, once a sequence, where nothing is shared, sizes pass what the others count in, or the reads of all sequences
//   would be few (they come from L2 at about 10 TB/s, and two launches less); MB of those reads and us, paged and the better of the others:
//     5: 7.9  10.9   24: 11.2  11.8   44: 9.3  11.8   66: 14.6  13.1   82: 16.2  15.8   120: 19.4  14.5   272: 47.2  37.2
//   tiles of 16 or 32 rows, each reading the prefix, while those reads are few; MB and us, those and tcgen05:
//     17: 14.5  17.7   28: 15.3  19.6   204: 38.1  37.2   629: 70.9  61.2   2,200: 252  69
enum Way { PAGED, ROWS, TILES };
constexpr double kPagedBytes = 48 << 20, kRowsBytes = 128 << 20;
Way way_of(int B, int rows, int G, int Hkv, int hd, int64_t n_pages, int page, int width, int n) {
  if (n >= B || n_pages == 0 || !countable(B, rows, G, Hkv, page, width, n)) return PAGED;
  const int seg = plan_rows(rows * G, hd).seg_rows;
  const double keys = (double)std::min((int64_t)width, n_pages) * page * hd * 4 * Hkv;      // bytes of a prefix, at most
  if ((double)B * ceil_div(rows * G, seg) * keys <= kPagedBytes) return PAGED;
  const double tiles = (double)(((int64_t)B * rows * G + seg - 1) / seg + n);
  return tiles * keys <= kRowsBytes ? ROWS : TILES;
}

}  // namespace
}  // namespace kf

using namespace kf;

extern "C" int64_t kf_op_shared_attention_work(int32_t B, int32_t rows, int32_t Hq, int32_t Hkv, int32_t hd, int64_t n_pages, int32_t page,
                                               int32_t width, int32_t n) {
  if (B <= 0 || n_pages < 0 || sizes_fault(B, rows, Hq, Hkv, hd, page, width, n)) return 0;
  const Way way = way_of(B, rows, Hq / Hkv, Hkv, hd, n_pages, page, width, n);
  if (way == PAGED) return kf_op_paged_attention_work(B, rows, Hq, Hkv, hd, page, width);
  SharedCall c{};
  c.B = B;
  c.rows = rows;
  c.Hq = Hq;
  c.Hkv = Hkv;
  c.G = Hq / Hkv;
  c.hd = hd;
  c.n_pages = n_pages;
  c.page = page;
  c.width = width;
  c.sh.n = n;
  return layout(c, way == TILES, nullptr);
}

extern "C" int kf_op_shared_attention(int32_t type, int32_t B, int32_t rows, int32_t Hq, int32_t Hkv, int32_t hd, const void* q, int64_t q_seq,
                                      int64_t q_row, int64_t q_head, const void* pool, int64_t n_pages, int32_t page, const int32_t* table,
                                      int32_t width, const int32_t* lens, int32_t n, const int32_t* groups, const int32_t* shared,
                                      float scale, void* out, void* work, void* stream) {
  const char* what = "kf_op_shared_attention";
  if (type != KF_TYPE_BF16 && type != KF_TYPE_FP16) return refuse(what, "the type is bf16 or fp16");
  if (const char* f = sizes_fault(B, rows, Hq, Hkv, hd, page, width, n)) return refuse(what, f);
  if (n_pages < 0 || n_pages > 0x7fffffffll) return refuse(what, "pages out of range");
  if (!(scale > 0.f) || std::isinf(scale)) return refuse(what, "scale is a positive number");
  if (B == 0) return KF_OK;
  if (!groups || !shared || !aligned(groups, 4) || !aligned(shared, 4)) return refuse(what, "groups or shared: null or misaligned");
  const Way way = way_of(B, rows, Hq / Hkv, Hkv, hd, n_pages, page, width, n);
  const bool no_work = !work && kf_op_shared_attention_work(B, rows, Hq, Hkv, hd, n_pages, page, width, n) > 0;
  if (!q || !out || !lens || no_work || (n_pages && !pool) || (width && !table)) return refuse(what, "a null array");
  if (!aligned(q, 16) || !aligned(pool, 16) || !aligned(out, 16) || !aligned(work, 256) || !aligned(table, 4) || !aligned(lens, 4))
    return refuse(what, "q, pool and out are 16-byte aligned, work 256-byte");
  if (q_seq % 8 || q_row % 8 || q_head % 8) return refuse(what, "q's strides are multiples of 8 elements");
  if (way == PAGED)
    return kf_op_paged_attention(type, B, rows, Hq, Hkv, hd, q, q_seq, q_row, q_head, pool, n_pages, page, table, width, lens, scale, out, work, stream);
  SharedCall c{q, q_seq, q_row, q_head, pool, table, lens, out, n_pages, Sharing{groups, shared, n}, {}, {}, serving_error_word(),
               B, rows, Hq, Hkv, Hq / Hkv, hd, page, width, scale * 1.4426950408889634f, Div(page), Div(Hq / Hkv), Div(rows * (Hq / Hkv)), Div(Hq), Div(rows)};
  if (!c.err) return refuse(what, "no error word", KF_E_CUDA);
  const bool tiles = way == TILES;
  layout(c, tiles, work);
  CUtensorMap map{};
  if (tiles && !pool_map(&map, pool, n_pages, Hkv, page, hd)) return refuse(what, "a tensor map is refused (the pool)");
  cudaStream_t s = (cudaStream_t)stream;
  if (type == KF_TYPE_BF16) return hd == 64 ? launch<__nv_bfloat16, 64>(type, c, tiles, map, s) : launch<__nv_bfloat16, 128>(type, c, tiles, map, s);
  return hd == 64 ? launch<__half, 64>(type, c, tiles, map, s) : launch<__half, 128>(type, c, tiles, map, s);
}
