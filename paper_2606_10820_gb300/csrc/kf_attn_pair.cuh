// Attention of pairs of 128-row sub-tiles on tcgen05, shared by the attention of
// prompts and of shared prefixes: a CTA of twelve warps, of which
//   warp 0      takes items and copies K and V tiles (and Q);
//   warp 1      issues S = Q K^T (128 x 128 x hd) and O += P V (128 x hd x 128), the two
//               sub-tiles in turn, so that one's softmax runs under the other's products;
//   warps 4-7, 8-11  the softmax of sub-tile 0 and 1, one thread per row (its TMEM lane).
// The products, the softmax of a tile and the barriers between them are here; what an item is, how
// its operands are loaded, which keys a row sees and where its output goes is the kernels'.
#pragma once

#include "kf_mma16.cuh"
#include "kf_serving.cuh"
#include "kf_tc.cuh"

namespace kf {
namespace pair {

constexpr int kRows = 128, kKeys = 128;
constexpr int kThreads = 384;
// registers a thread after the split of the launch's 384 x 168: 128 x 88 + 256 x 208
constexpr int kRegsFew = 88, kRegsSoftmax = 208;
constexpr uint32_t kAtom = kRows * 128;            // 128 rows of 64 elements: one swizzled box
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColO = 256;
// head_dim 64 leaves TMEM columns for a P of its own: the next S then runs under this one's exponentials
template <int HD> constexpr bool kOwnP = HD == 64;
template <int HD> constexpr uint32_t kColP = kOwnP<HD> ? kColO + 2 * HD : 0;
template <int HD> constexpr uint32_t kPitchP = kOwnP<HD> ? 64 : 128;      // columns from sub-tile 0's P to 1's
constexpr float kRaise = 8.f;
constexpr size_t kBarBytes = 512;
template <int HD> constexpr int kStages = HD == 128 ? 5 : 8;
template <int HD> constexpr uint32_t kTile = kAtom * (HD / 64);
template <int HD> constexpr size_t kSmem = (2 + kStages<HD>) * (size_t)kTile<HD> + kBarBytes;

template <typename T> constexpr uint32_t idesc(int M, int N) {
  // D fp32; A and B bf16 (1) or fp16 (0)
  const uint32_t f = std::is_same<T, __half>::value ? 0u : 1u;
  return (1u << 4) | (f << 7) | (f << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// MN-major operand of hd / 64 swizzled atoms: 64-wide atoms `kAtom` apart, 8-row K groups 1024 bytes apart
__device__ __forceinline__ uint64_t sdesc_v(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr >> 4) & 0x3FFF);
  d |= (uint64_t)(kAtom >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
// The product warp runs its loop as a whole and only the instructions themselves are one lane's
// (`leader`): with a lane's branch around the loop every descriptor went from that
// lane's registers to the uniform ones, about 80 clocks an instruction (3,390 clocks a key tile).
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r;
}
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t tmem_d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader)
      : "memory");
}
// A (M = 128 rows, pairs of 16-bit values) in TMEM
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t tmem_d, uint32_t tmem_a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d),
      "r"(tmem_a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t leader, uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// 32 bytes of one row (a 32-byte aligned address): half as many lines touched as two 16-byte stores
__device__ __forceinline__ void st_32(void* p, const uint32_t* r) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// (I: an item, as the load warp hands it to the others; n[i]: key tiles of sub-tile i, 0: no sub-tile)
template <typename I>
struct PairBars {
  uint64_t q_full, q_empty;
  uint64_t item_full[2], item_empty[2];
  uint64_t s_full[2], s_free[2], p_full[2][2], o_full[2], o_free[2];   // per sub-tile (and half of P)
  uint64_t tail;                                         // a V tile whose last rows are to be cleared has landed
  uint64_t kv_full[8], kv_empty[8];
  I item[2];
  uint32_t tmem;
};

// The product warp: items until one without sub-tiles
template <typename T, int HD, typename B>
__device__ __forceinline__ void product_warp(B& b, uint32_t tmem, uint32_t sQ, uint32_t sKV, int lane, int* err) {
  constexpr int ST = kStages<HD>;
  constexpr uint32_t TILE = kTile<HD>;
  constexpr uint32_t id_s = idesc<T>(kRows, kKeys), id_o = idesc<T>(kRows, HD) | (1u << 16);   // (V is MN-major)
  const uint32_t leader = elect_one();
  const uint32_t tm = __shfl_sync(~0u, tmem, 0);
  const uint64_t q0 = sdesc(sQ), k0 = sdesc(sKV), v0 = sdesc_v(sKV);      // (bytes / 16 are added to their low bits)
  // (uniform over the warp; the ring's position as a stage and a phase)
  int st = 0, ph = 0, parity_s[2] = {1, 1}, parity_p[2] = {0, 0}, parity_o[2] = {1, 1};
  auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(~0u, mbar_wait(smem_u32(bar), parity, err)); };
  auto stage = [&](int ahead) { return st + ahead >= ST ? st + ahead - ST : st + ahead; };
  auto full = [&](int ahead) { return wait(&b.kv_full[stage(ahead)], st + ahead >= ST ? ph ^ 1 : ph); };
  // S of sub-tile i against the K tile `ahead`, once the softmax has read the S before (where P
  // lies over S, its product has waited for that)
  auto s_product = [&](int i, int ahead) -> bool {
    if (kOwnP<HD>) {
      if (!wait(&b.s_free[i], parity_s[i])) return false;
      parity_s[i] ^= 1;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    }
    const uint64_t q = q0 + (i * TILE >> 4), k = k0 + (uint32_t)(stage(ahead) * (TILE >> 4));
#pragma unroll
    for (int kk = 0; kk < HD / 16; ++kk) {
      const uint32_t off = ((kk / 4) * kAtom + (kk % 4) * 32) >> 4;
      mma_ss(leader, tm + i * kKeys, q + off, k + off, id_s, kk > 0 ? 1u : 0u);
    }
    commit(leader, &b.s_full[i]);
    return true;
  };
  // the next K tile's S products of the sub-tiles that have one
  auto next_s = [&](int i, int j, const int* nn, int n) -> bool {
    if (j + 1 >= n) return true;
    if (i == 0 && !full(2)) return false;
    if (j + 1 < nn[i] && !s_product(i, 2)) return false;
    if (i == 1) {
      commit(leader, &b.kv_empty[stage(2)]);
      if (j + 2 == n) commit(leader, &b.q_empty);
    }
    return true;
  };
  bool ok = true;
  for (int it = 0; ok; ++it) {
    const int slot = it & 1;
    if (!wait(&b.item_full[slot], (it >> 1) & 1)) break;
    const int nn[2] = {__shfl_sync(~0u, b.item[slot].n[0], 0), __shfl_sync(~0u, b.item[slot].n[1], 0)};
    const int n = max(nn[0], nn[1]);
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&b.item_empty[slot]));
    if (n == 0) break;
    ok = wait(&b.q_full, it & 1) && full(0);
    if (!ok) break;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (ok && nn[i] > 0) ok = s_product(i, 0);
    if (!ok) break;
    commit(leader, &b.kv_empty[st]);
    if (n == 1) commit(leader, &b.q_empty);
    for (int j = 0; j < n; ++j) {
      if (kOwnP<HD>) {
        ok = next_s(0, j, nn, n) && next_s(1, j, nn, n);
        if (!ok) break;
      }
      ok = full(1);
      if (!ok) break;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (j < nn[i]) {
          if (j == 0) {                     // (the item before has left O)
            ok = wait(&b.o_free[i], parity_o[i]);
            parity_o[i] ^= 1;
            if (!ok) break;
          }
          const uint64_t v = v0 + (uint32_t)(stage(1) * (TILE >> 4));
#pragma unroll
          for (int h = 0; h < 2; ++h) {     // P's halves
            ok = wait(&b.p_full[i][h], parity_p[i]);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
            for (int kk = 4 * h; kk < 4 * h + 4; ++kk)
              mma_ts(leader, tm + kColO + i * HD, tm + kColP<HD> + i * kPitchP<HD> + 8 * kk, v + kk * (2048 >> 4), id_o,
                     (j > 0 || kk > 0) ? 1u : 0u);
          }
          if (!ok) break;
          parity_p[i] ^= 1;
          commit(leader, &b.o_full[i]);
        }
        if (i == 1) commit(leader, &b.kv_empty[stage(1)]);
        if (!kOwnP<HD>) {
          ok = next_s(i, j, nn, n);
          if (!ok) break;
        }
      }
      if (!ok) break;
      if (st + 2 >= ST) ph ^= 1;
      st = stage(2);
    }
  }
}

// One thread's row of a sub-tile
template <typename T, int HD>
struct Softmax {
  uint32_t tS, tO, tP;
  int sub, lane;
  __device__ __forceinline__ Softmax(uint32_t tmem, int sub_, int quarter, int lane_) : sub(sub_), lane(lane_) {
    const uint32_t lanes = tmem + ((uint32_t)(32 * quarter) << 16);
    tS = lanes + sub * kKeys;
    tO = lanes + kColO + sub * HD;
    tP = lanes + kColP<HD> + sub * kPitchP<HD>;
  }
  // The g-th key tile of the sub-tile (`first` of its item): P to TMEM; m: the reference (a raw score), l: the
  // sum.  mask(c, s): closed scores among the 32 from 32 c on to -inf.  false: a wait ran out
  template <typename B, typename M>
  __device__ __forceinline__ bool tile(B& b, float sc, bool first, int g, float& m, float& l, int* err, M mask) const {
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool { return __all_sync(~0u, mbar_wait(smem_u32(bar), parity, err)); };
    auto arrive = [&](uint64_t* bar) {
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(bar));
    };
    if (!wait(&b.s_full[sub], g & 1)) return false;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    uint32_t s[128];
    float mq[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    tmem_ld32_async(tS, s);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      tmem_wait32(s + 32 * c);
      if (c < 3) tmem_ld32_async(tS + 32 * (c + 1), s + 32 * (c + 1));
      mask(c, s + 32 * c);
#pragma unroll
      for (int e = 0; e < 32; e += 8)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          mq[x] = max3f(mq[x], __uint_as_float(s[32 * c + e + 2 * x]), __uint_as_float(s[32 * c + e + 2 * x + 1]));
    }
    if (kOwnP<HD>) {
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      arrive(&b.s_free[sub]);
    }
    const float mx = fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3]));
    const bool raise = first || (mx - m) * sc > kRaise;
    if (!first && __any_sync(~0u, raise)) {
      // O follows the new reference once the product before has been added
      const float f = raise ? mma::ex2((m - mx) * sc) : 1.f;
      if (!wait(&b.o_full[sub], (g - 1) & 1)) return false;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
      for (int c = 0; c < HD / 32; ++c) {
        float o[32];
        tmem_ld32(tO + 32 * c, o);
#pragma unroll
        for (int d = 0; d < 32; ++d) o[d] *= f;
        tmem_st32(tO + 32 * c, o);
      }
      l *= f;
    }
    if (raise) m = mx;
    const float nm = m == -INFINITY ? 0.f : -m * sc;
    const uint64_t sc2 = f2(sc, sc), nm2 = f2(nm, nm);
    uint64_t ps[4] = {0ull, 0ull, 0ull, 0ull};
    if (kOwnP<HD> && g > 0) {               // the product before has read P
      if (!wait(&b.o_full[sub], (g - 1) & 1)) return false;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint32_t pk[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const float2 d = f2_split(fma_f2(f2(__uint_as_float(s[32 * c + 2 * u]), __uint_as_float(s[32 * c + 2 * u + 1])), sc2, nm2));
        const float x = mma::ex2(d.x), y = mma::ex2(d.y);
        ps[u & 3] = add_f2(ps[u & 3], f2(x, y));
        pk[u] = pack2<T>(x, y);
      }
      tmem_st16(tP + 16 * c, pk);
      if (c & 1) {
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        arrive(&b.p_full[sub][c >> 1]);
      }
    }
    const float2 s2 = f2_split(add_f2(add_f2(ps[0], ps[1]), add_f2(ps[2], ps[3])));
    l += s2.x + s2.y;
    return true;
  }
  // The same in a third of the code: the scores come from TMEM twice, 64 at a time, for their maximum and for P.  A call of a few
  // tiles is mostly the first run through its code, at 12 to 15 clocks an instruction: the first tile took 6,000 to 12,000 clocks as above.
  // mask(c, s): closed scores among the 64 from 64 c on
  template <typename B, typename M>
  __device__ __forceinline__ bool short_tile(B& b, float sc, bool first, int g, float& m, float& l, int* err, M mask) const {
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool { return __all_sync(~0u, mbar_wait(smem_u32(bar), parity, err)); };
    auto arrive = [&](uint64_t* bar) {
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(bar));
    };
    uint32_t s[64];
    auto load = [&](int c) {
      tmem_ld32_async(tS + 64 * c, s);
      tmem_ld32_async(tS + 64 * c + 32, s + 32);
      tmem_wait32(s);
      tmem_wait32(s + 32);
      mask(c, s);
    };
    if (!wait(&b.s_full[sub], g & 1)) return false;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    float mq[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
    for (int c = 0; c < 2; ++c) {
      load(c);
#pragma unroll
      for (int e = 0; e < 64; e += 8)
#pragma unroll
        for (int x = 0; x < 4; ++x) mq[x] = max3f(mq[x], __uint_as_float(s[e + 2 * x]), __uint_as_float(s[e + 2 * x + 1]));
    }
    const float mx = fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3]));
    const bool raise = first || (mx - m) * sc > kRaise;
    if (g > 0 && (kOwnP<HD> || (!first && __any_sync(~0u, raise)))) {      // the product before has read P, and been added
      if (!wait(&b.o_full[sub], (g - 1) & 1)) return false;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    }
    if (!first && __any_sync(~0u, raise)) {
      // O follows the new reference
      const float f = raise ? mma::ex2((m - mx) * sc) : 1.f;
#pragma unroll 1
      for (int c = 0; c < HD / 32; ++c) {
        float o[32];
        tmem_ld32(tO + 32 * c, o);
#pragma unroll
        for (int d = 0; d < 32; ++d) o[d] *= f;
        tmem_st32(tO + 32 * c, o);
      }
      l *= f;
    }
    if (raise) m = mx;
    const float nm = m == -INFINITY ? 0.f : -m * sc;
    const uint64_t sc2 = f2(sc, sc), nm2 = f2(nm, nm);
    uint64_t ps[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll 1
    for (int c = 0; c < 2; ++c) {
      load(c);
      if (kOwnP<HD> && c == 1) {            // (S may be written again under the last exponentials)
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        arrive(&b.s_free[sub]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t pk[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) {
          const float2 d = f2_split(fma_f2(f2(__uint_as_float(s[32 * h + 2 * u]), __uint_as_float(s[32 * h + 2 * u + 1])), sc2, nm2));
          const float x = mma::ex2(d.x), y = mma::ex2(d.y);
          ps[u & 3] = add_f2(ps[u & 3], f2(x, y));
          pk[u] = pack2<T>(x, y);
        }
        tmem_st16(tP + 32 * c + 16 * h, pk);
      }
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      arrive(&b.p_full[sub][c]);
    }
    const float2 s2 = f2_split(add_f2(add_f2(ps[0], ps[1]), add_f2(ps[2], ps[3])));
    l += s2.x + s2.y;
    return true;
  }
};

}  // namespace pair
}  // namespace kf
