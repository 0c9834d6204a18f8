// Attention of the newest rows of each sequence over a paged cache
// (kf_op_paged_attention): grouped heads, head_dim 64 or 128, bf16 or fp16.
//
// The query rows of one (sequence, KV head) are its rows x group heads; tiles of
// 16 of them run on warp-level MMA (m16n8k16, fp32 accumulation) with the
// softmax in registers, so K and V are read once for all heads of a group.
// What bounds it is those bytes, so the layout serves the loads:
//   - The keys of all (sequence, KV head, tile) segments, in units of 8 KB of K
//     and V (16 keys of 128, 32 of 64), form one list that the CTAs share
//     evenly: a ragged batch and a single long sequence fill the SMs alike.  A segment that
//     ends in another CTA than it began in leaves fp32 partials, which k_join
//     adds in list order (so the same lengths give the same bits).
//   - In a CTA unit x belongs to warp x mod 4, which copies it into
//     a ring of its own (cp.async, two units ahead, across segment ends)
//     and waits for nobody; the warps of a segment meet once, to merge.
//   - Two CTAs per SM: 8 warps with two units in flight are 128 KB a SM, about
//     three times what DRAM latency asks for at 45 GB/s a SM.
#include <algorithm>

#include "kf_mma.cuh"
#include "kf_serving.cuh"

namespace kf {
namespace {

constexpr int NW = 4, kThreads = 32 * NW;     // warps of a CTA
constexpr int kStages = 3;
constexpr int kCtasPerSm = 2;
constexpr int kUnitBytes = 8192;              // K and V of a unit
constexpr int kTile = 16;                     // query rows of a segment
constexpr int kMinUnits = 4;                  // units of a CTA where the work allows it: one per warp

struct Args {
  const void* q;
  int64_t q_seq, q_row, q_head;
  const void* pool;
  const int32_t *table, *lens;
  void* out;
  float* part_o;        // [2 CTAs][16][hd]
  float2* part_ml;      // [2 CTAs][16]
  int* err;
  int64_t n_pages;
  int B, rows, Hq, Hkv, G, MT, page, width;
  float scale2;         // scale log2(e): scores in base-2 units
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

// The list: sequence by sequence, each one's Hkv * MT segments, each one's units.
// Part c of `parts` even ones is [x0, x1); b and base: the sequence that x0 lies
// in, and its first unit.  Called by the whole block.
struct Part {
  long long total, x0, x1, base;
  int b, parts;
};
template <int HD>
__device__ __forceinline__ long long part_begin(long long total, int parts, int c) {
  return total * c / parts;
}
template <int HD, int THREADS>
__device__ Part find_part(const Args& a, int c, int ctas) {
  __shared__ long long warp_sum[THREADS / 32];
  __shared__ Part found;
  const int t = threadIdx.x, per = (a.B + THREADS - 1) / THREADS, sb = a.Hkv * a.MT;
  const int first = min(a.B, t * per), last = min(a.B, first + per);
  long long mine = 0;
  for (int b = first; b < last; ++b) mine += units_of<HD>(a, b);
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
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < (t >> 5)) before += warp_sum[w];
    total += warp_sum[w];
  }
  const int parts = (int)min((long long)ctas, max(1ll, total / kMinUnits));
  const long long x0 = part_begin<HD>(total, parts, c), lo = before + incl - mine;
  if (c < parts && x0 >= lo && x0 < lo + mine) {
    long long base = lo;
    int b = first;
    for (long long n = (long long)units_of<HD>(a, b) * sb; x0 >= base + n; n = (long long)units_of<HD>(a, b) * sb) {
      base += n;
      ++b;
    }
    found = Part{total, x0, part_begin<HD>(total, parts, c + 1), base, b, parts};
  }
  if (t == 0 && c >= parts) found = Part{total, total, total, 0, a.B, parts};
  __syncthreads();
  return found;
}

// one segment's units within a CTA's part
template <int HD>
struct Piece {
  long long xs, xa, xb;    // the segment's first unit, the piece's units
  int b, s, n, len;        // sequence, segment of it, units of the segment, tokens
  __device__ __forceinline__ void at(const Args& a, const Part& p) {
    b = p.b;
    n = units_of<HD>(a, b);
    len = seq_len(a, b);
    s = (int)((p.x0 - p.base) / n);
    xs = p.base + (long long)s * n;
    xa = p.x0;
    xb = min(xs + n, p.x1);
  }
  // the next piece; false past the part's end
  __device__ __forceinline__ bool next(const Args& a, const Part& p) {
    if (xb >= p.x1) return false;
    if (++s == a.Hkv * a.MT) {
      s = 0;
      ++b;
      n = units_of<HD>(a, b);
      len = seq_len(a, b);
    }
    xs = xa = xb;
    xb = min(xs + n, p.x1);
    return true;
  }
};

// a warp's copies: unit after unit of its own, ahead of the products
template <typename T, int HD>
struct Feed {
  static constexpr int U = kUnit<HD>, kHalves = U / 16;
  Piece<HD> pc;
  long long x;
  int page[kHalves];       // pages of unit x
  bool more;
  __device__ __forceinline__ void look(const Args& a) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      const int key = (int)(x - pc.xs) * U + 16 * h;
      page[h] = key < pc.len ? __ldg(a.table + (size_t)pc.b * a.width + key / a.page) : -1;
    }
  }
  __device__ __forceinline__ void skip(const Args& a, const Part& p) {
    while (more && x >= pc.xb) more = pc.next(a, p);
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
        const int key0 = (int)(x - pc.xs) * U + 16 * h, left = pc.len - key0;
        const bool in = page[h] >= 0 && page[h] < a.n_pages;
        if (in) ok |= 1u << h;
        else if (left > 0 && lane == 0) atomicOr(a.err, KF_DEV_BAD_PAGE);
        const T* kb = static_cast<const T*>(a.pool) +
                      (((in ? (int64_t)page[h] : 0) * 2 * a.Hkv + hk) * a.page + key0 % a.page) * HD + c * 8;
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

template <int HD> constexpr int kMergeFloats = kTile * (HD + 2);    // one warp's O, m and l
// (two CTAs of 114,992 bytes, their static arrays and 1 KB each fit the SM's 228 KB)
template <int HD> constexpr size_t kSmem = NW * kStages * kUnitBytes + (NW / 2) * kMergeFloats<HD> * 4 + NW * kStages * 4;

template <typename T, int HD>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) k_paged(const Args a) {
  extern __shared__ __align__(128) uint8_t sm[];
  constexpr int U = kUnit<HD>, NT = U / 8, KS = HD / 16, DT = HD / 8;   // key tiles, dim steps of S, dim tiles of O
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31, g = lane >> 2, c = lane & 3;
  float* merge = reinterpret_cast<float*>(sm + NW * kStages * kUnitBytes);
  uint32_t* open_all = reinterpret_cast<uint32_t*>(merge + (NW / 2) * kMergeFloats<HD>);
  uint32_t* open = open_all + warp * kStages;
  const uint32_t ring = mma::smem_addr(sm) + warp * kStages * kUnitBytes;

  if (blockIdx.x == 0)
    for (int b = t; b < a.B; b += kThreads) {
      const int n = a.lens[b];
      if (n < 0 || n > a.width * a.page) atomicOr(a.err, KF_DEV_BAD_ROW);
    }
  const Part part = find_part<HD, kThreads>(a, blockIdx.x, gridDim.x);
  if (part.x0 < part.x1) {
    Feed<T, HD> feed;
    feed.start(a, part, warp);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) feed.copy(a, part, ring + i * kUnitBytes, open + i, lane);
    int st = 0;

    Piece<HD> pc;
    pc.at(a, part);
    do {
      const int hk = pc.s / a.MT, r0 = (pc.s % a.MT) * kTile, R = a.rows * a.G;
      const int f = (int)(pc.xa % NW), nw = (int)min((long long)NW, pc.xb - pc.xa);
      const int j = (warp - f + NW) % NW;          // this warp's place among the piece's
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[DT][4];
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f;
      if (j < nw) {
        // this lane's two rows: r0 + g and r0 + g + 8
        uint32_t q[KS][4];
        int last[2];                                // the last key each sees
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = r0 + g + 8 * h, i = r / a.G;
          last[h] = r < R ? pc.len - a.rows + i : -1;
          const T* qp = static_cast<const T*>(a.q) + pc.b * a.q_seq + i * a.q_row + (int64_t)(hk * a.G + r - i * a.G) * a.q_head;
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            q[k][h] = r < R ? __ldg(reinterpret_cast<const uint32_t*>(qp + 16 * k + 2 * c)) : 0u;
            q[k][h + 2] = r < R ? __ldg(reinterpret_cast<const uint32_t*>(qp + 16 * k + 8 + 2 * c)) : 0u;
          }
        }
        const int free_to = pc.len - a.rows;        // keys up to here are seen by every row
        for (long long x = pc.xa + j; x < pc.xb; x += NW) {
          mma::cp_wait<kStages - 2>();
          __syncwarp();
          const uint32_t kst = ring + st * kUnitBytes, vst = kst + kUnitBytes / 2;
          const uint32_t ok = open[st];
          float s[NT][4];
#pragma unroll
          for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
          // S: 16 keys x 16 dims per ldmatrix
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
              const int row = 8 * n + (lane & 7) + ((lane >> 4) << 3), ch = 2 * k + ((lane >> 3) & 1);
              uint32_t kb[4];
              mma::ldsm_x4(kst + row * (HD * 2) + ((ch ^ (row & 7)) << 4), kb);
              mma16816<T>(s[n], q[k], kb[0], kb[1]);
              mma16816<T>(s[n + 1], q[k], kb[2], kb[3]);
            }
          const int key0 = (int)(x - pc.xs) * U;
          const bool masked = key0 + U - 1 > free_to || ok != (1u << (U / 16)) - 1;
          float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float v = s[n][e] * a.scale2;
              if (masked && (key0 + 8 * n + 2 * c + (e & 1) > last[e >> 1] || !((ok >> (n >> 1)) & 1u))) v = -INFINITY;
              s[n][e] = v;
              mx[e >> 1] = fmaxf(mx[e >> 1], v);
            }
          float ref[2], fac[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            mx[h] = fmaxf(mx[h], __shfl_xor_sync(~0u, mx[h], 1));
            mx[h] = fmaxf(mx[h], __shfl_xor_sync(~0u, mx[h], 2));
            mx[h] = fmaxf(mx[h], m[h]);
            fac[h] = m[h] == -INFINITY ? 1.f : mma::ex2(m[h] - mx[h]);    // (nothing to scale yet)
            ref[h] = mx[h] == -INFINITY ? 0.f : mx[h];
            m[h] = mx[h];
          }
          if (__any_sync(~0u, fac[0] != 1.f || fac[1] != 1.f)) {
#pragma unroll
            for (int h = 0; h < 2; ++h) l[h] *= fac[h];
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              o[d][0] *= fac[0];
              o[d][1] *= fac[0];
              o[d][2] *= fac[1];
              o[d][3] *= fac[1];
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              s[n][e] = mma::ex2(s[n][e] - ref[e >> 1]);
              l[e >> 1] += s[n][e];
            }
          // O: 16 keys x 16 dims of V per ldmatrix; the probabilities are rounded to the
          // cache's type, the tensor cores' operand (the sum l is not)
#pragma unroll
          for (int n = 0; n < NT; n += 2) {
            const uint32_t p[4] = {pack2<T>(s[n][0], s[n][1]), pack2<T>(s[n][2], s[n][3]), pack2<T>(s[n + 1][0], s[n + 1][1]),
                                   pack2<T>(s[n + 1][2], s[n + 1][3])};
#pragma unroll
            for (int d = 0; d < DT; d += 2) {
              const int row = 8 * n + (lane & 15), ch = d + (lane >> 4);
              uint32_t vb[4];
              mma::ldsm_x4_t(vst + row * (HD * 2) + ((ch ^ (row & 7)) << 4), vb);
              mma16816<T>(o[d], p, vb[0], vb[1]);
              mma16816<T>(o[d + 1], p, vb[2], vb[3]);
            }
          }
          __syncwarp();                             // the stage before this one is free for all lanes
          feed.copy(a, part, ring + (st + kStages - 1) % kStages * kUnitBytes, open + (st + kStages - 1) % kStages, lane);
          st = (st + 1) % kStages;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          l[h] += __shfl_xor_sync(~0u, l[h], 1);
          l[h] += __shfl_xor_sync(~0u, l[h], 2);
        }
      }
      // the piece's warps merge in pairs: j + w into j
#pragma unroll
      for (int w = NW / 2; w; w >>= 1) {
        if (nw <= w) continue;                      // (uniform)
        if (j >= w && j < min(2 * w, nw)) {
          float* d = merge + (j - w) * kMergeFloats<HD>;
#pragma unroll
          for (int i = 0; i < DT; ++i) *reinterpret_cast<float4*>(d + (i * 32 + lane) * 4) = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
          if (c == 0)
#pragma unroll
            for (int h = 0; h < 2; ++h) *reinterpret_cast<float2*>(d + kTile * HD + 2 * (g + 8 * h)) = make_float2(m[h], l[h]);
        }
        __syncthreads();
        if (j < w && j + w < nw) {
          const float* d = merge + j * kMergeFloats<HD>;
          float fa[2], fb[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float2 ml = *reinterpret_cast<const float2*>(d + kTile * HD + 2 * (g + 8 * h));
            const float mm = fmaxf(m[h], ml.x);
            fa[h] = m[h] == -INFINITY ? 0.f : mma::ex2(m[h] - mm);
            fb[h] = ml.x == -INFINITY ? 0.f : mma::ex2(ml.x - mm);
            l[h] = l[h] * fa[h] + ml.y * fb[h];
            m[h] = mm;
          }
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            const float4 v = *reinterpret_cast<const float4*>(d + (i * 32 + lane) * 4);
            o[i][0] = o[i][0] * fa[0] + v.x * fb[0];
            o[i][1] = o[i][1] * fa[0] + v.y * fb[0];
            o[i][2] = o[i][2] * fa[1] + v.z * fb[1];
            o[i][3] = o[i][3] * fa[1] + v.w * fb[1];
          }
        }
        __syncthreads();
      }
      if (j == 0) {
        const bool whole = pc.xa == pc.xs && pc.xb == pc.xs + pc.n;
        const int slot = 2 * blockIdx.x + (pc.xa == pc.xs);       // 0: a segment begun elsewhere, 1: one that goes on elsewhere
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = r0 + g + 8 * h, i = r / a.G;
          if (r >= R) continue;
          if (whole) {
            const float inv = l[h] == 0.f ? 0.f : 1.f / l[h];     // (no key seen: zeros)
            T* op = static_cast<T*>(a.out) + (((int64_t)pc.b * a.rows + i) * a.Hq + hk * a.G + r - i * a.G) * HD;
#pragma unroll
            for (int d = 0; d < DT; ++d)
              *reinterpret_cast<uint32_t*>(op + 8 * d + 2 * c) = pack2<T>(o[d][2 * h] * inv, o[d][2 * h + 1] * inv);
          } else {
            float* op = a.part_o + ((int64_t)slot * kTile + g + 8 * h) * HD;
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<float2*>(op + 8 * d + 2 * c) = make_float2(o[d][2 * h], o[d][2 * h + 1]);
            if (c == 0) a.part_ml[slot * kTile + g + 8 * h] = make_float2(m[h], l[h]);
          }
        }
      }
    } while (pc.next(a, part));
    mma::cp_wait<0>();
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Block (c, row): the segment that goes on from part c - 1 into part c, if it began
// in part c - 1: its pieces (slot 1 of c - 1, slot 0 of c, c + 1, ...) added in order
template <typename T, int HD>
__global__ void __launch_bounds__(256) k_join(const Args a, int ctas) {
  constexpr int V4 = HD / 4, GR = 256 / V4;          // float4s of a row; groups that share the pieces
  __shared__ float4 so[GR][V4];
  __shared__ float2 sml[GR];
  const int t = threadIdx.x, c = blockIdx.x + 1, v = t % V4, gr = t / V4;
  const Part part = find_part<HD, 256>(a, c, ctas);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (c >= part.parts || part.x0 >= part.x1) return;
  Piece<HD> pc;
  pc.at(a, part);
  if (pc.xs >= part.x0 || pc.xs < part_begin<HD>(part.total, part.parts, c - 1)) return;
  const int r0 = (pc.s % a.MT) * kTile, hk = pc.s / a.MT, r = r0 + blockIdx.y;
  if (r >= a.rows * a.G) return;
  // parts c .. e - 1 begin inside the segment
  const long long end = pc.xs + pc.n;
  int e = c + 1;
  {
    int lo = c + 1, hi = part.parts;                 // the first part that begins at or past the end
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (part_begin<HD>(part.total, part.parts, mid) < end) lo = mid + 1;
      else hi = mid;
    }
    e = lo;
  }
  const int n = e - c + 1;
  auto slot = [&](int i) { return (int64_t)(i == 0 ? 2 * (c - 1) + 1 : 2 * (c + i - 1)) * kTile + blockIdx.y; };
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float m2, float l2, float4 x) {
    const float mm = fmaxf(m, m2), fa = m == -INFINITY ? 0.f : mma::ex2(m - mm), fb = m2 == -INFINITY ? 0.f : mma::ex2(m2 - mm);
    m = mm;
    l = l * fa + l2 * fb;
    o = make_float4(o.x * fa + x.x * fb, o.y * fa + x.y * fb, o.z * fa + x.z * fb, o.w * fa + x.w * fb);
  };
  // (written by the kernel before this one: not through the read-only path)
#pragma unroll 4
  for (int i = gr; i < n; i += GR) {
    const float2 ml = __ldcg(a.part_ml + slot(i));
    add(ml.x, ml.y, __ldcg(reinterpret_cast<const float4*>(a.part_o + slot(i) * HD) + v));
  }
  so[gr][v] = o;
  if (v == 0) sml[gr] = make_float2(m, l);
  __syncthreads();
  if (gr == 0) {
    for (int i = 1; i < min(GR, n); ++i) add(sml[i].x, sml[i].y, so[i][v]);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int i = r / a.G;
    T* op = static_cast<T*>(a.out) + (((int64_t)pc.b * a.rows + i) * a.Hq + hk * a.G + r - i * a.G) * HD;
    reinterpret_cast<uint2*>(op)[v] = make_uint2(pack2<T>(o.x * inv, o.y * inv), pack2<T>(o.z * inv, o.w * inv));
  }
}

int paged_ctas() { return kCtasPerSm * device_sms(); }

template <typename T, int HD>
int launch(Args a, void* work, cudaStream_t s) {
  const int ctas = paged_ctas();
  a.part_ml = static_cast<float2*>(work);
  a.part_o = reinterpret_cast<float*>(a.part_ml + 2 * (size_t)ctas * kTile);
  // no more CTAs than the longest lists the table could hold fill
  const long long units = (long long)a.B * a.Hkv * a.MT * std::max(1, ceil_div(a.width * a.page, kUnit<HD>));
  const int grid = (int)std::min<long long>(ctas, std::max(1ll, units / kMinUnits));
  static PerDevice attr;
  set_smem_attr(attr, k_paged<T, HD>, kSmem<HD>);
  launch_cluster(k_paged<T, HD>, dim3(grid), dim3(kThreads), kSmem<HD>, 1, false, s, a);
  if (grid > 1)
    launch_cluster(k_join<T, HD>, dim3(grid - 1, std::min(kTile, a.rows * a.G)), dim3(256), 0, 1, true, s, a, grid);
  return launched("kf_op_paged_attention");
}

}  // namespace
}  // namespace kf

using namespace kf;

extern "C" int64_t kf_op_paged_attention_work(int32_t hd) {
  return 2ll * paged_ctas() * kTile * (8 + 4ll * hd);
}

extern "C" int kf_op_paged_attention(int32_t type, int32_t B, int32_t rows, int32_t Hq, int32_t Hkv, int32_t hd,
                                     const void* q, int64_t q_seq, int64_t q_row, int64_t q_head, const void* pool,
                                     int64_t n_pages, int32_t page, const int32_t* table, int32_t width,
                                     const int32_t* lens, float scale, void* out, void* work, void* stream) {
  const char* what = "kf_op_paged_attention";
  if (type != KF_TYPE_BF16 && type != KF_TYPE_FP16) return refuse(what, "the type is bf16 or fp16");
  if (hd != 64 && hd != 128) return refuse(what, "head_dim is 64 or 128");
  if (B < 0 || rows < 1 || Hkv < 1 || Hq < 1 || Hq % Hkv || Hq > 4096 || rows > 4096) return refuse(what, "sequences, rows or heads out of range");
  if (page < 16 || page % 16 || page > 4096 || width < 0 || (int64_t)width * page > (1 << 30)) return refuse(what, "page is a multiple of 16, width * page at most 2^30");
  if (n_pages < 0 || n_pages > 0x7fffffffll) return refuse(what, "pages out of range");
  if (!(scale > 0.f) || std::isinf(scale)) return refuse(what, "scale is a positive number");
  if (B == 0) return KF_OK;
  if (!q || !out || !lens || !work || (width && !table) || (n_pages && !pool)) return refuse(what, "a null array");
  if (!aligned(q, 16) || !aligned(pool, 16) || !aligned(out, 16) || !aligned(work, 256) || !aligned(table, 4) || !aligned(lens, 4))
    return refuse(what, "q, pool and out are 16-byte aligned, work 256-byte");
  if (q_seq % 8 || q_row % 8 || q_head % 8) return refuse(what, "q's strides are multiples of 8 elements");
  const int G = Hq / Hkv, MT = ceil_div(rows * G, kTile);
  if ((long long)B * Hkv * MT * (std::max(1, ceil_div(width * page, 16))) > (1ll << 40)) return refuse(what, "too many keys");
  Args a{q, q_seq, q_row, q_head, pool, table, lens, out, nullptr, nullptr, serving_error_word(), n_pages,
         B, rows, Hq, Hkv, G, MT, page, width, scale * 1.4426950408889634f};
  if (!a.err) return refuse(what, "no error word", KF_E_CUDA);
  cudaStream_t s = (cudaStream_t)stream;
  if (type == KF_TYPE_BF16) return hd == 64 ? launch<__nv_bfloat16, 64>(a, work, s) : launch<__nv_bfloat16, 128>(a, work, s);
  return hd == 64 ? launch<__half, 64>(a, work, s) : launch<__half, 128>(a, work, s);
}
