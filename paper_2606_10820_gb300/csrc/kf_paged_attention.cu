// Attention of the newest rows of each sequence over a paged cache
// (kf_op_paged_attention): grouped heads, head_dim 64 or 128, bf16 or fp16.
//
// The query rows of one (sequence, KV head) are its rows x group heads; tiles of
// 16 of them run on warp-level MMA (m16n8k16, fp32 accumulation) with the
// softmax in registers, so K and V are read once for all heads of a group (and at
// head_dim 64 for 32 rows at a time, which the registers hold there; at 128 two tiles of a large
// cache take turns on each unit, so that the second read comes from L2).
// What bounds it is those bytes, so the layout serves the loads:
//   - The keys of all (sequence, KV head, tile) segments, in units of 8 KB of K
//     and V (16 keys of 128, 32 of 64), form one list that the CTAs share
//     evenly: a ragged batch and a single long sequence fill the SMs alike.  A segment counts
//     kExtra units more than it has, for its start and end.  One that
//     ends in another CTA than it began in leaves fp32 partials, which k_join
//     adds in list order (so the same list gives the same bits).
//   - In a CTA unit x belongs to warp x mod 4, which copies it into
//     a ring of its own (cp.async, ahead of the products and across segment ends)
//     and waits for nobody; the warps of a segment meet once, to merge.
//   - Two CTAs per SM with two units a warp under way, or (head_dim 64, one tile) three
//     with one: 128 or 96 KB a SM, twice and more what DRAM latency asks for at 45 GB/s a SM.
// Measured (bf16): 128 sequences of 512 to 8,192, 32 heads over 8 of 128, one row, in 340 us (6.7
// TB/s); one of 37,013 in 33 us (4.6 TB/s, the start and the join); 256 of 128 to 1,024, 12 over 4
// of 64, eight rows, fp16, in 51 us (3.1 TB/s: the products of 24 rows, 32 with the padding).
#include <algorithm>

#include "kf_mma.cuh"
#include "kf_serving.cuh"

namespace kf {
namespace {

constexpr int NW = 4, kThreads = 32 * NW;     // warps of a CTA
constexpr int kUnitBytes = 8192;              // K and V of a unit
constexpr int kMinUnits = 4;                  // units of a CTA where the work allows it: one per warp
constexpr int kDirect = 16;                   // units of a segment that one CTA takes as a whole where the CTAs suffice
constexpr int64_t kL2Bytes = 128 << 20;
constexpr int kExtra = 6;                     // a segment's start and end, in units
// what a (head_dim, tiles of 16 rows per segment) pair of kernels uses
// head_dim 128 has registers for one tile a warp: of two tiles the warps take turns (units come twice, once for
// each tile, to neighbouring warps), so that their keys come from DRAM once and the second time from L2
template <int HD, int TILES> constexpr bool kTurns = HD == 128 && TILES == 2;
template <int HD, int TILES> constexpr int kHeld = kTurns<HD, TILES> ? 1 : TILES;      // tiles of a warp
template <int HD, int TILES> constexpr bool kThree = HD == 64 && TILES == 1;
template <int HD, int TILES> constexpr int kStages = kThree<HD, TILES> ? 2 : 3;
template <int HD, int TILES> constexpr int kCtasPerSm = kThree<HD, TILES> ? 3 : 2;
constexpr int kMostCtasPerSm = 3, kMostRows = 32, kMostValues = 4096;      // of a segment: rows, rows x hd

// a segment that CTA c began and others went on with
struct Split { int b, s, pieces, pad; };

struct Args {
  const void* q;
  int64_t q_seq, q_row, q_head;
  const void* pool;
  const int32_t *table, *lens;
  void* out;
  float* part_o;        // [2 CTAs][rows of a segment][hd]
  float2* part_ml;      // [2 CTAs][kMostRows]
  Split* split;         // [CTAs]
  int* err;
  int64_t n_pages;
  int B, rows, Hq, Hkv, G, MT, page, page_shift, width;    // page_shift: -1 where page is no power of two
  int direct;           // a CTA per segment
  float scale2;         // scale log2(e): scores in base-2 units
  __device__ __forceinline__ int page_of(int key) const { return page_shift >= 0 ? key >> page_shift : key / page; }
};

template <int HD> constexpr int kUnit = kUnitBytes / (4 * HD);      // keys

template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if constexpr (std::is_same<T, __half>::value) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    return mma::pack_bf16(lo, hi);
  }
}
template <typename T>
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<T, __half>::value)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    mma::mma16816(d, a, b0, b1);
}

__device__ __forceinline__ int seq_len(const Args& a, int b) {
  return min(max(__ldg(a.lens + b), 0), a.width * a.page);
}
// units of each of a sequence's segments (one without keys has a unit too: its rows are written)
template <int HD> __device__ __forceinline__ int units_of(const Args& a, int b) {
  return max(1, (seq_len(a, b) + kUnit<HD> - 1) / kUnit<HD>);
}

// The list: sequence by sequence, each one's Hkv * MT segments, each one's units and kExtra
// places more.  Part c of `parts` even ones is [x0, x1); b and base: the sequence that x0 lies
// in, and its first place.  Called by the whole block.
struct Part {
  long long total, x0, x1, base;
  int b, parts;
};
template <int HD, int TILES>
__device__ __forceinline__ int places_of(const Args& a, int b) { return units_of<HD>(a, b) * (kTurns<HD, TILES> ? 2 : 1); }
__device__ __forceinline__ long long part_begin(long long total, int parts, int c) { return total * c / parts; }
template <int HD, int TILES>
__device__ Part find_part(const Args& a, int c, int ctas) {
  __shared__ long long warp_sum[NW];
  __shared__ Part found;
  const int t = threadIdx.x, per = (a.B + kThreads - 1) / kThreads, sb = a.Hkv * a.MT;
  const int first = min(a.B, t * per), last = min(a.B, first + per);
  long long mine = 0;
  for (int b = first; b < last; ++b) mine += places_of<HD, TILES>(a, b) + kExtra;
  mine *= sb;
  long long incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(~0u, incl, o);
    if ((t & 31) >= o) incl += v;
  }
  if ((t & 31) == 31) warp_sum[t >> 5] = incl;
  __syncthreads();
  long long before = 0, total = 0;
  for (int w = 0; w < NW; ++w) {
    if (w < (t >> 5)) before += warp_sum[w];
    total += warp_sum[w];
  }
  const int parts = (int)min((long long)ctas, max(1ll, total / kMinUnits));
  const long long x0 = part_begin(total, parts, c), lo = before + incl - mine;
  if (c < parts && x0 >= lo && x0 < lo + mine) {
    long long base = lo;
    int b = first;
    for (long long n = (long long)(places_of<HD, TILES>(a, b) + kExtra) * sb; x0 >= base + n; n = (long long)(places_of<HD, TILES>(a, b) + kExtra) * sb) {
      base += n;
      ++b;
    }
    found = Part{total, x0, part_begin(total, parts, c + 1), base, b, parts};
  }
  if (t == 0 && c >= parts) found = Part{total, total, total, 0, a.B, parts};
  __syncthreads();
  return found;
}

// one segment's places within a CTA's part
template <int HD, int TILES>
struct Piece {
  long long xs, xa, xb, xe;    // the segment's first unit; the piece's units [xa, xb) (or none) and its end
  int b, s, n, len;            // sequence, segment of it, units of the segment, tokens
  __device__ __forceinline__ int unit(long long x) const { return (int)(x - xs) >> (kTurns<HD, TILES> ? 1 : 0); }
  __device__ __forceinline__ void cut(const Part& p) {
    xa = max(xs, p.x0);
    xb = min(xs + n, p.x1);
    xe = min(xs + n + kExtra, p.x1);
  }
  __device__ __forceinline__ void at(const Args& a, const Part& p) {
    b = p.b;
    n = places_of<HD, TILES>(a, b);
    len = seq_len(a, b);
    s = (int)((p.x0 - p.base) / (n + kExtra));
    xs = p.base + (long long)s * (n + kExtra);
    cut(p);
  }
  // the next piece; false past the part's end
  __device__ __forceinline__ bool next(const Args& a, const Part& p) {
    if (xe >= p.x1) return false;
    if (++s == a.Hkv * a.MT) {
      s = 0;
      ++b;
      n = places_of<HD, TILES>(a, b);
      len = seq_len(a, b);
    }
    xs = xe;
    cut(p);
    return true;
  }
};

// a warp's copies: unit after unit of its own, ahead of the products
template <typename T, int HD, int TILES>
struct Feed {
  static constexpr int U = kUnit<HD>, kHalves = U / 16;
  Piece<HD, TILES> pc;
  long long x;
  int page[kHalves];       // pages of unit x
  bool more;
  __device__ __forceinline__ void look(const Args& a) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      const int key = pc.unit(x) * U + 16 * h;
      page[h] = key < pc.len ? __ldg(a.table + (size_t)pc.b * a.width + a.page_of(key)) : -1;
    }
  }
  __device__ __forceinline__ void skip(const Args& a, const Part& p) {
    while (more && x >= pc.xb) {
      more = pc.next(a, p);
      if (x < pc.xa) x += (pc.xa - x + NW - 1) / NW * NW;
    }
    if (more) look(a);
  }
  __device__ __forceinline__ void start(const Args& a, const Part& p, int warp) {
    pc.at(a, p);
    x = p.x0 + ((warp - (int)(p.x0 % NW) + NW) % NW);
    more = true;
    skip(a, p);
  }
  // copies unit x into the stage (one commit group, empty past the end); *open:
  // bit h: the stage's 16 keys h are in a page of the pool
  __device__ __forceinline__ void copy(const Args& a, const Part& p, uint32_t stage, uint32_t* open, int lane) {
    if (more) {
      constexpr int CH = HD / 8, RP = 32 / CH;      // 16-byte chunks of a row; rows of one warp copy
      const int hk = pc.s / a.MT, c = lane % CH;
      uint32_t ok = 0;
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const int key0 = pc.unit(x) * U + 16 * h, left = pc.len - key0;
        const bool in = page[h] >= 0 && page[h] < a.n_pages;
        if (in) ok |= 1u << h;
        else if (left > 0 && lane == 0) atomicOr(a.err, KF_DEV_BAD_PAGE);
        const T* kb = static_cast<const T*>(a.pool) +
                      (((in ? (int64_t)page[h] : 0) * 2 * a.Hkv + hk) * a.page + key0 - a.page_of(key0) * a.page) * HD + c * 8;
        const T* vb = kb + (int64_t)a.Hkv * a.page * HD;
#pragma unroll
        for (int i = 0; i < 16 / RP; ++i) {
          const int r = i * RP + lane / CH, row = 16 * h + r;
          const int bytes = in && r < left ? 16 : 0;      // (0: zeros, nothing is read)
          const uint32_t d = stage + row * (HD * 2) + ((c ^ (row & 7)) << 4);
          mma::cp_async16(d, bytes ? kb + r * HD : static_cast<const T*>(a.pool), bytes);
          mma::cp_async16(d + kUnitBytes / 2, bytes ? vb + r * HD : static_cast<const T*>(a.pool), bytes);
        }
      }
      if (lane == 0) *open = ok;
      x += NW;
      skip(a, p);
    }
    mma::cp_commit();
  }
};

template <int HD, int TILES> constexpr int kMergeFloats = 16 * kHeld<HD, TILES> * (HD + 2);    // one warp's O, m and l
template <int HD, int TILES>
constexpr size_t kSmem = NW * kStages<HD, TILES> * kUnitBytes + (NW / 2) * kMergeFloats<HD, TILES> * 4 + NW * kStages<HD, TILES> * 4;
// an SM's 228 KB hold the CTAs, their static arrays (find_part's, at most 128 bytes) and 1 KB for each
template <int HD, int TILES> constexpr bool kFits = kCtasPerSm<HD, TILES> * (kSmem<HD, TILES> + 128 + 1024) <= 233472;
static_assert(sizeof(Part) + NW * sizeof(long long) <= 128, "the static arrays");
static_assert(kFits<64, 1> && kFits<64, 2> && kFits<128, 1> && kFits<128, 2>, "the CTAs of an SM");

template <typename T, int HD, int TILES>
__global__ void __launch_bounds__(kThreads, kCtasPerSm<HD, TILES>) k_paged(const Args a) {
  extern __shared__ __align__(128) uint8_t sm[];
  constexpr int ST = kStages<HD, TILES>, ROWS = 16 * TILES, HELD = kHeld<HD, TILES>;
  constexpr int PARTS = kTurns<HD, TILES> ? 2 : 1;      // warps of a piece that hold its rows in the end
  constexpr int U = kUnit<HD>, NT = U / 8, KS = HD / 16, DT = HD / 8;   // key tiles, dim steps of S, dim tiles of O
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31, g = lane >> 2, c = lane & 3;
  float* merge = reinterpret_cast<float*>(sm + NW * ST * kUnitBytes);
  uint32_t* open = reinterpret_cast<uint32_t*>(merge + (NW / 2) * kMergeFloats<HD, TILES>) + warp * ST;
  const uint32_t ring = mma::smem_addr(sm) + warp * ST * kUnitBytes;

  if (blockIdx.x == 0)
    for (int b = t; b < a.B; b += kThreads) {
      const int n = a.lens[b];
      if (n < 0 || n > a.width * a.page) atomicOr(a.err, KF_DEV_BAD_ROW);
    }
  Part part;
  if (a.direct) {
    // this segment's places are the whole list: [0, n + kExtra)
    const int sb = a.Hkv * a.MT, b = blockIdx.x / sb, n = places_of<HD, TILES>(a, b) + kExtra;
    part = Part{n, 0, n, -(long long)(blockIdx.x - b * sb) * n, b, 1};
  } else {
    if (t == 0) a.split[blockIdx.x].pieces = 0;
    part = find_part<HD, TILES>(a, blockIdx.x, gridDim.x);
  }
  if (part.x0 < part.x1) {
    Feed<T, HD, TILES> feed;
    feed.start(a, part, warp);
#pragma unroll
    for (int i = 0; i < ST - 1; ++i) feed.copy(a, part, ring + i * kUnitBytes, open + i, lane);
    int st = 0;

    Piece<HD, TILES> pc;
    pc.at(a, part);
    do {
      if (pc.xa >= pc.xb) continue;                // (uniform) only places without units
      const int hk = pc.s / a.MT, seg0 = (pc.s % a.MT) * ROWS, R = a.rows * a.G;
      const int f = (int)(pc.xa % NW), nw = (int)min((long long)NW, pc.xb - pc.xa);
      const int j = (warp - f + NW) % NW;          // this warp's place among the piece's
      const int tile = PARTS > 1 ? ((int)(pc.xa - pc.xs) + j) & 1 : 0, r0 = seg0 + 16 * tile;
      // this lane's rows of tile i: r0 + 16 i + g and 8 more.  m: raw scores' maximum
      float m[HELD][2], l[HELD][2], o[HELD][DT][4];
#pragma unroll
      for (int i = 0; i < HELD; ++i) {
        m[i][0] = m[i][1] = -INFINITY;
        l[i][0] = l[i][1] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[i][d][0] = o[i][d][1] = o[i][d][2] = o[i][d][3] = 0.f;
      }
      if (j < nw) {
        uint32_t q[HELD][KS][4];
        int last[HELD][2];                         // the last key each row sees
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = r0 + 16 * i + g + 8 * h, tok = r / a.G;
            last[i][h] = r < R ? pc.len - a.rows + tok : -1;
            const T* qp = static_cast<const T*>(a.q) + pc.b * a.q_seq + tok * a.q_row + (int64_t)(hk * a.G + r - tok * a.G) * a.q_head;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              q[i][k][h] = r < R ? __ldg(reinterpret_cast<const uint32_t*>(qp + 16 * k + 2 * c)) : 0u;
              q[i][k][h + 2] = r < R ? __ldg(reinterpret_cast<const uint32_t*>(qp + 16 * k + 8 + 2 * c)) : 0u;
            }
          }
        const int free_to = pc.len - a.rows;        // keys up to here are seen by every row
        for (long long x = pc.xa + j; x < pc.xb; x += NW) {
          mma::cp_wait<ST - 2>();
          __syncwarp();                             // all lanes' copies; and the stage before this one is free
          const uint32_t ok = open[st];
          const uint32_t kst = ring + st * kUnitBytes, vst = kst + kUnitBytes / 2;
          const int fr = st == 0 ? ST - 1 : st - 1;
          feed.copy(a, part, ring + fr * kUnitBytes, open + fr, lane);
          st = st + 1 == ST ? 0 : st + 1;
          float s[HELD][NT][4];
#pragma unroll
          for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n) s[i][n][0] = s[i][n][1] = s[i][n][2] = s[i][n][3] = 0.f;
          // S: 16 keys x 16 dims per ldmatrix
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
              const int row = 8 * n + (lane & 7) + ((lane >> 4) << 3), ch = 2 * k + ((lane >> 3) & 1);
              uint32_t kb[4];
              mma::ldsm_x4(kst + row * (HD * 2) + ((ch ^ (row & 7)) << 4), kb);
#pragma unroll
              for (int i = 0; i < HELD; ++i) {
                mma16816<T>(s[i][n], q[i][k], kb[0], kb[1]);
                mma16816<T>(s[i][n + 1], q[i][k], kb[2], kb[3]);
              }
            }
          const int key0 = pc.unit(x) * U;
          if (key0 + U - 1 > free_to || ok != (1u << (U / 16)) - 1) {       // (uniform)
#pragma unroll
            for (int i = 0; i < HELD; ++i)
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (key0 + 8 * n + 2 * c + (e & 1) > last[i][e >> 1] || !((ok >> (n >> 1)) & 1u)) s[i][n][e] = -INFINITY;
          }
#pragma unroll
          for (int i = 0; i < HELD; ++i) {
            float nm[2], fac[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float mx = fmaxf(s[i][0][2 * h], s[i][0][2 * h + 1]);
#pragma unroll
              for (int n = 1; n < NT; ++n) mx = fmaxf(mx, fmaxf(s[i][n][2 * h], s[i][n][2 * h + 1]));
              mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 1));
              mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 2));
              mx = fmaxf(mx, m[i][h]);
              fac[h] = m[i][h] == -INFINITY ? 1.f : mma::ex2((m[i][h] - mx) * a.scale2);     // (nothing to scale yet)
              nm[h] = mx == -INFINITY ? 0.f : -mx * a.scale2;
              m[i][h] = mx;
            }
            if (__any_sync(~0u, fac[0] != 1.f || fac[1] != 1.f)) {
#pragma unroll
              for (int h = 0; h < 2; ++h) l[i][h] *= fac[h];
#pragma unroll
              for (int d = 0; d < DT; ++d) {
                o[i][d][0] *= fac[0];
                o[i][d][1] *= fac[0];
                o[i][d][2] *= fac[1];
                o[i][d][3] *= fac[1];
              }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                s[i][n][e] = mma::ex2(fmaf(s[i][n][e], a.scale2, nm[e >> 1]));
                l[i][e >> 1] += s[i][n][e];
              }
          }
          // O: 16 keys x 16 dims of V per ldmatrix; the probabilities are rounded to the
          // cache's type, the tensor cores' operand (the sum l is not)
#pragma unroll
          for (int n = 0; n < NT; n += 2) {
            uint32_t p[HELD][4];
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
              p[i][0] = pack2<T>(s[i][n][0], s[i][n][1]);
              p[i][1] = pack2<T>(s[i][n][2], s[i][n][3]);
              p[i][2] = pack2<T>(s[i][n + 1][0], s[i][n + 1][1]);
              p[i][3] = pack2<T>(s[i][n + 1][2], s[i][n + 1][3]);
            }
#pragma unroll
            for (int d = 0; d < DT; d += 2) {
              const int row = 8 * n + (lane & 15), ch = d + (lane >> 4);
              uint32_t vb[4];
              mma::ldsm_x4_t(vst + row * (HD * 2) + ((ch ^ (row & 7)) << 4), vb);
#pragma unroll
              for (int i = 0; i < HELD; ++i) {
                mma16816<T>(o[i][d], p[i], vb[0], vb[1]);
                mma16816<T>(o[i][d + 1], p[i], vb[2], vb[3]);
              }
            }
          }
        }
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            l[i][h] += __shfl_xor_sync(~0u, l[i][h], 1);
            l[i][h] += __shfl_xor_sync(~0u, l[i][h], 2);
          }
      }
      // the piece's warps merge in pairs: j + w into j
#pragma unroll
      for (int w = NW / 2; w >= PARTS; w >>= 1) {
        if (nw <= w) continue;                      // (uniform)
        if (j >= w && j < min(2 * w, nw)) {
          float* d = merge + (j - w) * kMergeFloats<HD, TILES>;
#pragma unroll
          for (int i = 0; i < HELD; ++i) {
#pragma unroll
            for (int x = 0; x < DT; ++x)
              *reinterpret_cast<float4*>(d + ((i * DT + x) * 32 + lane) * 4) = make_float4(o[i][x][0], o[i][x][1], o[i][x][2], o[i][x][3]);
            if (c == 0)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                *reinterpret_cast<float2*>(d + 16 * HELD * HD + 2 * (16 * i + g + 8 * h)) = make_float2(m[i][h], l[i][h]);
          }
        }
        __syncthreads();
        if (j < w && j + w < nw) {
          const float* d = merge + j * kMergeFloats<HD, TILES>;
#pragma unroll
          for (int i = 0; i < HELD; ++i) {
            float fa[2], fb[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float2 ml = *reinterpret_cast<const float2*>(d + 16 * HELD * HD + 2 * (16 * i + g + 8 * h));
              const float mm = fmaxf(m[i][h], ml.x);
              fa[h] = m[i][h] == -INFINITY ? 0.f : mma::ex2((m[i][h] - mm) * a.scale2);
              fb[h] = ml.x == -INFINITY ? 0.f : mma::ex2((ml.x - mm) * a.scale2);
              l[i][h] = l[i][h] * fa[h] + ml.y * fb[h];
              m[i][h] = mm;
            }
#pragma unroll
            for (int x = 0; x < DT; ++x) {
              const float4 v = *reinterpret_cast<const float4*>(d + ((i * DT + x) * 32 + lane) * 4);
              o[i][x][0] = o[i][x][0] * fa[0] + v.x * fb[0];
              o[i][x][1] = o[i][x][1] * fa[0] + v.y * fb[0];
              o[i][x][2] = o[i][x][2] * fa[1] + v.z * fb[1];
              o[i][x][3] = o[i][x][3] * fa[1] + v.w * fb[1];
            }
          }
        }
        __syncthreads();
      }
      if (j < PARTS) {                             // (of a piece of one unit the second warp's rows are empty)
        const long long end = pc.xs + pc.n;
        const bool whole = pc.xa == pc.xs && pc.xb == end;
        const int slot = 2 * blockIdx.x + (pc.xa == pc.xs);       // 0: a segment begun elsewhere, 1: one that goes on elsewhere
        // (parts up to the last that begins before the segment's end: total p / parts < end)
        if (!whole && pc.xa == pc.xs && j == 0 && lane == 0)
          a.split[blockIdx.x] = Split{pc.b, pc.s, (int)((end * part.parts + part.total - 1) / part.total) - (int)blockIdx.x, 0};
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int rr = 16 * (tile + i) + g + 8 * h, r = seg0 + rr, tok = r / a.G;
            if (r >= R) continue;
            if (whole) {
              const float inv = l[i][h] == 0.f ? 0.f : 1.f / l[i][h];     // (no key seen: zeros)
              T* op = static_cast<T*>(a.out) + (((int64_t)pc.b * a.rows + tok) * a.Hq + hk * a.G + r - tok * a.G) * HD;
#pragma unroll
              for (int d = 0; d < DT; ++d)
                *reinterpret_cast<uint32_t*>(op + 8 * d + 2 * c) = pack2<T>(o[i][d][2 * h] * inv, o[i][d][2 * h + 1] * inv);
            } else {
              float* op = a.part_o + ((int64_t)slot * ROWS + rr) * HD;
#pragma unroll
              for (int d = 0; d < DT; ++d) *reinterpret_cast<float2*>(op + 8 * d + 2 * c) = make_float2(o[i][d][2 * h], o[i][d][2 * h + 1]);
              if (c == 0) a.part_ml[slot * kMostRows + rr] = make_float2(m[i][h], l[i][h]);
            }
          }
      }
    } while (pc.next(a, part));
    mma::cp_wait<0>();
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Block (c, y): rows y, y + gridDim.y, ... of the segment that CTA c began and others went on
// with: its pieces (slot 1 of c, slot 0 of c + 1, c + 2, ...) added in order
constexpr int kJoinThreads = 256;
template <typename T, int HD, int TILES>
__global__ void __launch_bounds__(kJoinThreads) k_join(const Args a) {
  constexpr int ROWS = 16 * TILES, V4 = HD / 4, GR = kJoinThreads / V4;      // float4s of a row; groups that share the pieces
  __shared__ float4 so[GR][V4];
  __shared__ float2 sml[GR];
  const int t = threadIdx.x, c = blockIdx.x, v = t % V4, gr = t / V4;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // (written by the kernel before this one: not through the read-only path)
  const int4 sp = __ldcg(reinterpret_cast<const int4*>(a.split + c));
  const int n = sp.z, r0 = (sp.y % a.MT) * ROWS, hk = sp.y / a.MT;
  if (n == 0) return;
  for (int rr = blockIdx.y; rr < min(ROWS, a.rows * a.G - r0); rr += gridDim.y) {
    auto slot = [&](int i) { return (int64_t)(i == 0 ? 2 * c + 1 : 2 * (c + i)); };
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float m2, float l2, float4 x) {
      const float mm = fmaxf(m, m2);
      const float fa = m == -INFINITY ? 0.f : mma::ex2((m - mm) * a.scale2), fb = m2 == -INFINITY ? 0.f : mma::ex2((m2 - mm) * a.scale2);
      m = mm;
      l = l * fa + l2 * fb;
      o = make_float4(o.x * fa + x.x * fb, o.y * fa + x.y * fb, o.z * fa + x.z * fb, o.w * fa + x.w * fb);
    };
#pragma unroll 4
    for (int i = gr; i < n; i += GR) {
      const float2 ml = __ldcg(a.part_ml + slot(i) * kMostRows + rr);
      add(ml.x, ml.y, __ldcg(reinterpret_cast<const float4*>(a.part_o + (slot(i) * ROWS + rr) * HD) + v));
    }
    so[gr][v] = o;
    if (v == 0) sml[gr] = make_float2(m, l);
    __syncthreads();
    if (gr == 0) {
      for (int i = 1; i < min(GR, n); ++i) add(sml[i].x, sml[i].y, so[i][v]);
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int r = r0 + rr, tok = r / a.G;
      T* op = static_cast<T*>(a.out) + (((int64_t)sp.x * a.rows + tok) * a.Hq + hk * a.G + r - tok * a.G) * HD;
      reinterpret_cast<uint2*>(op)[v] = make_uint2(pack2<T>(o.x * inv, o.y * inv), pack2<T>(o.z * inv, o.w * inv));
    }
    __syncthreads();
  }
}

int64_t most_ctas() { return (int64_t)kMostCtasPerSm * device_sms(); }

// Segments of at most kDirect units by the table's width, no more of them than CTAs fit at once: one CTA each, no
// search, no scratch and no join (3 sequences of 150 tokens, 64 heads over 8 of 64, 8 rows: 14.6 -> 7.5 us)
struct Shape {
  int tiles, MT, longest;      // tiles of 16 rows per segment, segments of a (sequence, KV head), units of the widest sequence
  long long segments;
  bool direct;
};
// (tokens: at most so many in the sequences)
Shape shape_of(int B, int rows, int G, int Hkv, int hd, int page, int width, int64_t tokens) {
  Shape s;
  s.longest = std::max(1, ceil_div(width * page, kUnitBytes / (4 * hd)));
  auto split = [&](int tiles) {
    s.tiles = tiles;
    s.MT = ceil_div(rows * G, 16 * tiles);
    s.segments = (long long)B * Hkv * s.MT;
  };
  split(hd == 64 && rows * G > 16 ? 2 : 1);
  s.direct = s.longest <= kDirect && s.segments <= (hd == 64 && s.tiles == 1 ? kCtasPerSm<64, 1> : 2) * device_sms();
  // Tiles that take turns pay where the second read of the keys would be one from DRAM: a cache larger than the L2
  // (8 rows, 32 heads over 8, one tile and turns, us: 128 sequences of 512 to 8,192  685  450, 64 of 128 to 1,024  60  53; 8
  // heads over 2: 64 of 2,000, 131 MB  42.3  41.6, 16 of them  18.5  21.6); an odd tile would be read with nothing beside it
  // (24 heads over 4, 32 of 1,000 to 4,000: 66  77)
  if (hd == 128 && s.MT % 2 == 0 && !s.direct && tokens * Hkv * hd * 4 > kL2Bytes) {
    split(2);
    s.longest *= 2;
  }
  return s;
}

template <typename T, int HD, int TILES>
int launch(Args a, const Shape& sh, void* work, cudaStream_t s) {
  const int64_t most = most_ctas();
  a.MT = sh.MT;
  a.direct = sh.direct;
  a.split = static_cast<Split*>(work);
  a.part_ml = reinterpret_cast<float2*>(a.split + most);
  a.part_o = reinterpret_cast<float*>(a.part_ml + 2 * most * kMostRows);
  // no more CTAs than the longest list that the table could hold fills
  const int grid = (int)(sh.direct ? sh.segments : std::min<long long>(kCtasPerSm<HD, TILES> * device_sms(),
                                                                       std::max(1ll, sh.segments * (sh.longest + kExtra) / kMinUnits)));
  // few segments in many pieces: a row of one for each of more blocks (2 sequences of 4000, 8 heads over 2, 8 rows, with 4, 8
  // and 16 blocks: 20.2, 15.1, 13.1 us; 128 of 512 to 8192, 32 heads over 8: 685, 686, 691)
  const int by = (int)std::min<long long>(16, std::max(4ll, 2 * grid / sh.segments));
  static PerDevice attr;
  set_smem_attr(attr, k_paged<T, HD, TILES>, kSmem<HD, TILES>);
  launch_cluster(k_paged<T, HD, TILES>, dim3(grid), dim3(kThreads), kSmem<HD, TILES>, 1, false, s, a);
  if (!sh.direct && grid > 1) launch_cluster(k_join<T, HD, TILES>, dim3(grid, std::min(by, a.rows * a.G)), dim3(kJoinThreads), 0, 1, true, s, a);
  return launched("kf_op_paged_attention");
}
template <typename T>
int launch_any(int hd, const Args& a, const Shape& sh, void* work, cudaStream_t s) {
  if (hd == 128) return sh.tiles == 2 ? launch<T, 128, 2>(a, sh, work, s) : launch<T, 128, 1>(a, sh, work, s);
  return sh.tiles == 2 ? launch<T, 64, 2>(a, sh, work, s) : launch<T, 64, 1>(a, sh, work, s);
}
// the arguments' sizes; nullptr if they are fine
const char* sizes_fault(int B, int rows, int Hq, int Hkv, int hd, int page, int width) {
  if (hd != 64 && hd != 128) return "head_dim is 64 or 128";
  if (B < 0 || rows < 1 || Hkv < 1 || Hq < 1 || Hq % Hkv || Hq > 4096 || rows > 4096) return "sequences, rows or heads out of range";
  if (page < 16 || page % 16 || page > 4096 || width < 0 || (int64_t)width * page > (1 << 30)) return "page is a multiple of 16, width * page at most 2^30";
  if ((long long)B * Hkv * ceil_div(rows * (Hq / Hkv), 16) * (width * (long long)page / 16 + kExtra + 1) > (1ll << 40)) return "too many keys";
  return nullptr;
}

}  // namespace
}  // namespace kf

using namespace kf;

extern "C" int64_t kf_op_paged_attention_work(int32_t B, int32_t rows, int32_t Hq, int32_t Hkv, int32_t hd, int32_t page, int32_t width) {
  if (B <= 0 || sizes_fault(B, rows, Hq, Hkv, hd, page, width)) return 0;
  if (shape_of(B, rows, Hq / Hkv, Hkv, hd, page, width, 0).direct) return 0;
  return most_ctas() * (int64_t)(sizeof(Split) + 2 * (kMostRows * sizeof(float2) + kMostValues * sizeof(float)));
}

extern "C" int kf_op_paged_attention(int32_t type, int32_t B, int32_t rows, int32_t Hq, int32_t Hkv, int32_t hd,
                                     const void* q, int64_t q_seq, int64_t q_row, int64_t q_head, const void* pool,
                                     int64_t n_pages, int32_t page, const int32_t* table, int32_t width,
                                     const int32_t* lens, float scale, void* out, void* work, void* stream) {
  const char* what = "kf_op_paged_attention";
  if (type != KF_TYPE_BF16 && type != KF_TYPE_FP16) return refuse(what, "the type is bf16 or fp16");
  if (const char* f = sizes_fault(B, rows, Hq, Hkv, hd, page, width)) return refuse(what, f);
  if (n_pages < 0 || n_pages > 0x7fffffffll) return refuse(what, "pages out of range");
  if (!(scale > 0.f) || std::isinf(scale)) return refuse(what, "scale is a positive number");
  if (B == 0) return KF_OK;
  const int G = Hq / Hkv;
  const Shape sh = shape_of(B, rows, G, Hkv, hd, page, width, std::min((int64_t)B * width, n_pages) * page);
  if (!q || !out || !lens || (!work && !sh.direct) || (width && !table) || (n_pages && !pool)) return refuse(what, "a null array");
  if (!aligned(q, 16) || !aligned(pool, 16) || !aligned(out, 16) || !aligned(work, 256) || !aligned(table, 4) || !aligned(lens, 4))
    return refuse(what, "q, pool and out are 16-byte aligned, work 256-byte");
  if (q_seq % 8 || q_row % 8 || q_head % 8) return refuse(what, "q's strides are multiples of 8 elements");
  int shift = -1;
  if ((page & (page - 1)) == 0)
    for (shift = 0; (1 << shift) < page;) ++shift;
  if (!n_pages) pool = q;      // (nothing of it is read)
  const Args a{q, q_seq, q_row, q_head, pool, table, lens, out, nullptr, nullptr, nullptr, serving_error_word(), n_pages,
               B, rows, Hq, Hkv, G, 0, page, shift, width, 0, scale * 1.4426950408889634f};
  if (!a.err) return refuse(what, "no error word", KF_E_CUDA);
  cudaStream_t s = (cudaStream_t)stream;
  return type == KF_TYPE_BF16 ? launch_any<__nv_bfloat16>(hd, a, sh, work, s) : launch_any<__half>(hd, a, sh, work, s);
}
