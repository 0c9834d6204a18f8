// Attention of few query rows over stretches of a paged cache (kf_op_shared_attention): the keys of each sequence
// from its group's prefix on, and with few rows a group the prefixes too.  head_dim 64 or 128, bf16 or fp16.
//
// A segment is a tile of 16 query rows (32 at head_dim 64 where there are more than 16) and the keys that they read: a
// sequence's rows and its own keys, or rows of a group's sequences and the prefix.  Products are warp-level MMA
// (m16n8k16), the softmax stays in registers.  The list of all segments, in units of 8 KB of K and V (16 keys of 128, 32 of
// 64) and kExtra places more a segment, is shared evenly by warps: each one streams its units through a ring of its own (cp.async, ahead
// of the products and across segments) and meets nobody.  (A team of four warps a segment, whose rows have to be merged, took
// 3 us a segment of three units: 256 sequences of 8 rows and 72 own keys in 16 us of which 2 were copies.)  Segments of up to
// kWhole units are not cut.
// What bounds it: the bytes of long stretches; short ones the chain of a segment (Q, pages, K and V, products).
// Measured: the own keys (1 to 700) of 128 sequences, 32 heads over 8 of 128, 184 MB, in 32 us, 6 of them to the first data; those (1 to
// 1,024) of 64 sequences, 135 MB, in 20 us from there (6.7 TB/s).
#include <algorithm>

#include "kf_mma16.cuh"
#include "kf_shared.cuh"

namespace kf {
namespace {

constexpr int NW = 4, kThreads = 32 * NW;        // warps of a CTA
constexpr int kUnitBytes = 8192;                 // K and V of a unit
constexpr int kStages = 3;                       // units of a warp's ring
constexpr int kExtra = 2;                        // a segment's start and end, in units
constexpr int kMinPlaces = 4;                    // places of a part, at least
constexpr int kWhole = 6;                        // units of a segment that is not cut
constexpr int kCtasPerSm = 2;
template <int HD> constexpr int kUnit = kUnitBytes / (4 * HD);      // keys
constexpr size_t kSmem = (size_t)NW * kStages * kUnitBytes + NW * kStages * 4;

__device__ __forceinline__ int seq_len(const SharedCall& a, int b) { return min(max(__ldg(a.lens + b), 0), a.width * a.page); }

// An entry of the list: a group's prefix (e < groups) or a sequence's own keys; its rows, and its keys [key0, end)
template <int HD, int ROWS, bool PREFIX>
struct Entry {
  bool prefix;
  int g, b, rows, lo, end;       // group; first sequence; rows under a KV head; the first key and the end
  int tiles, units;              // tiles of rows; units of a segment
  __device__ __forceinline__ Entry() {}
  __device__ __forceinline__ Entry(const SharedCall& a, int e) {
    prefix = PREFIX && e < a.sh.n;
    if (prefix) {
      g = e;
      const int2 m = members(a.sh, g, a.B);
      b = m.x;
      rows = (m.y - m.x) * a.rows * a.G;
      lo = 0;
      end = prefix_of(a.sh, g, a.width * a.page);
      units = (end + kUnit<HD> - 1) / kUnit<HD>;
      tiles = units > 0 ? (rows + ROWS - 1) / ROWS : 0;
    } else {
      b = PREFIX ? e - a.sh.n : e;
      g = group_of(a.sh, b);
      rows = a.rows * a.G;
      lo = prefix_of(a.sh, g, a.width * a.page);
      end = seq_len(a, b);
      // (one without keys has a unit too: its rows are written)
      units = max(1, (end - key0() + kUnit<HD> - 1) / kUnit<HD>);
      tiles = (rows + ROWS - 1) / ROWS;
    }
  }
  __device__ __forceinline__ int key0() const { return lo & ~15; }      // (units begin where 16 keys of a page do)
  __device__ __forceinline__ int places(const SharedCall& a) const { return tiles * a.Hkv * (units + kExtra); }
};

// A warp's walk over its part's pieces
template <int HD, int ROWS, bool PREFIX>
struct Walk {
  Parts parts;
  Entry<HD, ROWS, PREFIX> en;
  int e, s, x0, x1, base;        // the entry and the segment of it; the part; the entry's first place
  int xs, xa, xb;                // the segment's first unit; the piece's units
  __device__ __forceinline__ int entries(const SharedCall& a) const { return (PREFIX ? a.sh.n : 0) + a.B; }
  __device__ __forceinline__ bool whole() const { return en.units <= kWhole; }
  // the next piece with units, from segment s of entry e on; false past the part's end
  __device__ __forceinline__ bool settle(const SharedCall& a) {
    for (;;) {
      const int segs = en.tiles * a.Hkv;
      if (s >= segs) {
        base += en.places(a);
        if (base >= x1 || ++e >= entries(a)) return false;
        en = Entry<HD, ROWS, PREFIX>(a, e);
        s = 0;
        continue;
      }
      xs = base + s * (en.units + kExtra);
      if (xs >= x1) return false;
      xa = whole() ? xs : max(xs, x0);
      xb = whole() ? xs + en.units : min(xs + en.units, x1);
      if (xa < xb && (!whole() || xs >= x0)) return true;
      ++s;
    }
  }
  __device__ __forceinline__ bool start(const SharedCall& a, const Parts& p, int c, int entry, int base_) {
    parts = p;
    x0 = p.begin(c);
    x1 = p.begin(c + 1);
    e = entry;
    base = base_;
    if (x0 >= x1) return false;
    en = Entry<HD, ROWS, PREFIX>(a, e);
    s = (x0 - base) / (en.units + kExtra);
    return settle(a);
  }
  __device__ __forceinline__ bool next(const SharedCall& a) {
    ++s;
    return settle(a);
  }
  __device__ __forceinline__ int key(int x) const { return en.key0() + (x - xs) * kUnit<HD>; }
};

// The list's parts, and for each warp of the CTA the entry that its part begins in.  Called by the whole block
struct Found { int entry, base; };
template <int HD, int ROWS, bool PREFIX>
__device__ Parts find_parts(const SharedCall& a, int most, Found* found) {
  __shared__ int warp_sum[NW];
  const int t = threadIdx.x, n = (PREFIX ? a.sh.n : 0) + a.B, per = (n + kThreads - 1) / kThreads;
  const int first = min(n, t * per), last = min(n, first + per);
  int mine = 0;
  for (int e = first; e < last; ++e) mine += Entry<HD, ROWS, PREFIX>(a, e).places(a);
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(~0u, incl, o);
    if ((t & 31) >= o) incl += v;
  }
  if ((t & 31) == 31) warp_sum[t >> 5] = incl;
  __syncthreads();
  int before = 0, total = 0;
  for (int w = 0; w < NW; ++w) {
    if (w < (t >> 5)) before += warp_sum[w];
    total += warp_sum[w];
  }
  const Parts p(total, min(most, max(1, total / kMinPlaces)));
  const int lo = before + incl - mine;
  for (int w = 0; w < NW; ++w) {
    const int c = blockIdx.x * NW + w, x = p.begin(c);
    if (c >= p.parts || x < lo || x >= lo + mine) continue;
    int base = lo, e = first;
    for (int v; x >= base + (v = Entry<HD, ROWS, PREFIX>(a, e).places(a)); ++e) base += v;
    found[w] = Found{e, base};
  }
  __syncthreads();
  return p;
}

template <typename T, int HD, int TILES, bool PREFIX>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) k_rows(const __grid_constant__ SharedCall a, int most) {
  extern __shared__ __align__(128) uint8_t sm[];
  __shared__ Found found[NW];
  constexpr int ST = kStages, ROWS = 16 * TILES, U = kUnit<HD>, kHalves = U / 16;
  constexpr int NT = U / 8, KS = HD / 16, DT = HD / 8;   // key tiles, dim steps of S, dim tiles of O
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31, g = lane >> 2, c = lane & 3, part = blockIdx.x * NW + warp;
  uint32_t* open = reinterpret_cast<uint32_t*>(sm + NW * ST * kUnitBytes) + warp * ST;
  const uint32_t ring = mma::smem_addr(sm) + warp * ST * kUnitBytes;
  using W = Walk<HD, ROWS, PREFIX>;
  const Parts parts = find_parts<HD, ROWS, PREFIX>(a, most, found);
  if (blockIdx.x == 0) {
    bool bad = false;
    for (int b = t; b < a.B; b += kThreads) {
      const int n = a.lens[b];
      bad |= n < 0 || n > a.width * a.page;
    }
    for (int i = t; PREFIX && i < a.sh.n; i += kThreads) {
      const int p = a.sh.groups[i], e = a.sh.groups[i + 1], n = a.sh.shared[i];
      bad |= p < 0 || e < p || e > a.B || (i == 0 && p != 0) || (i == a.sh.n - 1 && e != a.B) || n < 0 || n > a.width * a.page;
    }
    if (bad) atomicOr(a.err, KF_DEV_BAD_ROW);
  }
  W pc;
  if (pc.start(a, parts, part, found[warp].entry, found[warp].base)) {
    // the copies: unit after unit, ahead of the products
    W fd = pc;
    int fx = fd.xa, fslot = 0, page[kHalves];
    bool more = true;
    auto look = [&] {
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const int key = fd.key(fx) + 16 * h;
        page[h] = key < fd.en.end ? __ldg(a.table + (int64_t)fd.en.b * a.width + a.by_page.of(key)) : -1;
      }
    };
    look();
    // unit fx into the next slot (one commit group, empty past the end); open[slot], bit h: its 16 keys h are in a page of the pool
    auto copy = [&] {
      if (more) {
        constexpr int CH = HD / 8, RP = 32 / CH;      // 16-byte chunks of a row; rows of one warp copy
        const int hk = fd.s - fd.s / a.Hkv * a.Hkv, ch = lane % CH;
        const uint32_t stage = ring + fslot * kUnitBytes;
        uint32_t ok = 0;
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          const int key0 = fd.key(fx) + 16 * h, left = fd.en.end - key0, skip = fd.en.lo - key0;
          const bool in = page[h] >= 0 && page[h] < a.n_pages;
          if (in) ok |= 1u << h;
          else if (left > 0 && lane == 0) atomicOr(a.err, KF_DEV_BAD_PAGE);
          const T* kb = static_cast<const T*>(a.pool) +
                        (((in ? (int64_t)page[h] : 0) * 2 * a.Hkv + hk) * a.page + key0 - a.by_page.of(key0) * a.page) * HD + ch * 8;
          const T* vb = kb + (int64_t)a.Hkv * a.page * HD;
#pragma unroll
          for (int i = 0; i < 16 / RP; ++i) {
            const int r = i * RP + lane / CH, row = 16 * h + r;
            const int bytes = in && r < left && r >= skip ? 16 : 0;      // (0: zeros, nothing is read)
            const uint32_t d = stage + row * (HD * 2) + ((ch ^ (row & 7)) << 4);
            mma::cp_async16(d, bytes ? kb + r * HD : static_cast<const T*>(a.pool), bytes);
            mma::cp_async16(d + kUnitBytes / 2, bytes ? vb + r * HD : static_cast<const T*>(a.pool), bytes);
          }
        }
        if (lane == 0) open[fslot] = ok;
        if (++fx >= fd.xb) {
          more = fd.next(a);
          fx = fd.xa;
        }
        if (more) look();
      }
      fslot = fslot + 1 == ST ? 0 : fslot + 1;
      mma::cp_commit();
    };
#pragma unroll 1
    for (int i = 0; i < ST - 1; ++i) copy();
    int st = 0;
    do {
      const int hk = pc.s - pc.s / a.Hkv * a.Hkv, tile = pc.s / a.Hkv, r0 = tile * ROWS;
      // this lane's rows of 16-row tile i: r0 + 16 i + g and 8 more.  m: raw scores' maximum
      float m[TILES][2], l[TILES][2], o[TILES][DT][4];
      uint32_t q[TILES][KS][4];
      int last[TILES][2], at[TILES][2];               // the last key each row sees; its place among all rows (-1: none)
      int free_to = 0x7fffffff;                       // keys up to here are seen by every row
#pragma unroll
      for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          m[i][h] = -INFINITY;
          l[i][h] = 0.f;
#pragma unroll
          for (int d = 0; d < DT; ++d) o[i][d][2 * h] = o[i][d][2 * h + 1] = 0.f;
          const int r = r0 + 16 * i + g + 8 * h;
          const bool in = r < pc.en.rows;
          const int seq = PREFIX ? a.by_seq.of(r) : 0, y = r - seq * (int)a.by_seq.d, tok = a.by_group.of(y), j = y - tok * a.G;
          const int b = pc.en.b + seq;
          last[i][h] = -1;
          at[i][h] = in ? (b * a.rows + tok) * a.Hq + hk * a.G + j : -1;
          if (in) {
            last[i][h] = min(pc.en.end, (PREFIX ? seq_len(a, b) : pc.en.end) - a.rows + tok + 1) - 1;
            free_to = min(free_to, last[i][h]);
          }
          const T* qp = static_cast<const T*>(a.q) + b * a.q_seq + tok * a.q_row + (int64_t)(hk * a.G + j) * a.q_head;
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            q[i][k][h] = in ? __ldg(reinterpret_cast<const uint32_t*>(qp + 16 * k + 2 * c)) : 0u;
            q[i][k][h + 2] = in ? __ldg(reinterpret_cast<const uint32_t*>(qp + 16 * k + 8 + 2 * c)) : 0u;
          }
        }
      free_to = __reduce_min_sync(~0u, free_to);
#pragma unroll 1
      for (int x = pc.xa; x < pc.xb; ++x) {
        mma::cp_wait<ST - 2>();
        __syncwarp();                             // all lanes' copies; and the stage before this one is free
        const uint32_t ok = open[st];
        const uint32_t kst = ring + st * kUnitBytes, vst = kst + kUnitBytes / 2;
        copy();
        st = st + 1 == ST ? 0 : st + 1;
        float s[TILES][NT][4];
#pragma unroll
        for (int i = 0; i < TILES; ++i)
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
            for (int i = 0; i < TILES; ++i) {
              mma16816<T>(s[i][n], q[i][k], kb[0], kb[1]);
              mma16816<T>(s[i][n + 1], q[i][k], kb[2], kb[3]);
            }
          }
        const int key0 = pc.key(x);
        if (key0 + U - 1 > free_to || key0 < pc.en.lo || ok != (1u << kHalves) - 1) {       // (uniform)
#pragma unroll
          for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int key = key0 + 8 * n + 2 * c + (e & 1);
                if (key > last[i][e >> 1] || key < pc.en.lo || !((ok >> (n >> 1)) & 1u)) s[i][n][e] = -INFINITY;
              }
        }
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
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
          uint32_t p[TILES][4];
#pragma unroll
          for (int i = 0; i < TILES; ++i) {
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
            for (int i = 0; i < TILES; ++i) {
              mma16816<T>(o[i][d], p[i], vb[0], vb[1]);
              mma16816<T>(o[i][d + 1], p[i], vb[2], vb[3]);
            }
          }
        }
      }
      const bool begins = pc.xa == pc.xs;
      const Partials& to = PREFIX && pc.en.prefix ? a.pre : a.own;
      if (begins && lane == 0) {
        const int rec = PREFIX && pc.en.prefix ? prefix_record((int64_t)pc.en.b * a.rows * a.G, pc.en.g, tile, ROWS, hk, a.Hkv)
                                               : (pc.en.b * a.Hkv + hk) * pc.en.tiles + tile;
        if (rec < to.segments) to.rec[rec] = Record{part, pc.whole() ? 1 : parts.part_of(pc.xs + pc.en.units - 1) - part + 1};
      }
#pragma unroll
      for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          l[i][h] += __shfl_xor_sync(~0u, l[i][h], 1);
          l[i][h] += __shfl_xor_sync(~0u, l[i][h], 2);
          if (at[i][h] < 0) continue;
          const int64_t q = begins ? (int64_t)at[i][h] : (int64_t)part * ROWS + 16 * i + g + 8 * h;
          float* op = (begins ? to.first_o : to.more_o) + q * HD;
#pragma unroll
          for (int d = 0; d < DT; ++d) *reinterpret_cast<float2*>(op + 8 * d + 2 * c) = make_float2(o[i][d][2 * h], o[i][d][2 * h + 1]);
          if (c == 0) (begins ? to.first_ml : to.more_ml)[q] = make_float2(m[i][h], l[i][h]);
        }
    } while (pc.next(a));
    mma::cp_wait<0>();
  }
  // What comes after waits for this kernel alone and is to see the prefixes' kernel before it too: this one does not end before
  // that.  (One CTA waits; the others leave their SM to those that have not started)
  if (!PREFIX && blockIdx.x == gridDim.x - 1) asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <typename T, int HD, int TILES, bool PREFIX>
void launch(const SharedCall& c, cudaStream_t s) {
  static PerDevice attr;
  set_smem_attr(attr, k_rows<T, HD, TILES, PREFIX>, kSmem);
  launch_cluster(k_rows<T, HD, TILES, PREFIX>, dim3(c.own.parts / NW), dim3(kThreads), kSmem, 1, !PREFIX, s, c, c.own.parts);
}
template <typename T, bool PREFIX>
void launch_any(const SharedCall& c, cudaStream_t s) {
  if (c.hd == 128) launch<T, 128, 1, PREFIX>(c, s);
  else if (c.own.seg_rows == 16) launch<T, 64, 1, PREFIX>(c, s);
  else launch<T, 64, 2, PREFIX>(c, s);
}

}  // namespace

RowsPlan plan_rows(int rows_of_seq, int hd) { return RowsPlan{device_sms() * kCtasPerSm * NW, hd == 64 && rows_of_seq > 16 ? 32 : 16}; }

void launch_rows(int32_t type, const SharedCall& c, bool prefixes, cudaStream_t s) {
  if (type == KF_TYPE_BF16) prefixes ? launch_any<__nv_bfloat16, true>(c, s) : launch_any<__nv_bfloat16, false>(c, s);
  else prefixes ? launch_any<__half, true>(c, s) : launch_any<__half, false>(c, s);
}

}  // namespace kf
