// One thread block of a kernel's source on the CPU: its threads run as fibers, the
// warps in an order that the caller gives, each as far as the next barrier or collective
// that it has to wait at.  An order that puts a warp last shows what the others may
// do before it: shared memory that is read after a barrier and written before the next one.
// (Warp collectives take all 32 lanes, as the kernels' do.)
#pragma once

#include <ucontext.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <memory>
#include <vector>

#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static
#define __align__(n) alignas(n)

struct Index { unsigned x = 0, y = 0, z = 0; };
static Index threadIdx, blockIdx;
struct int2 { int x, y; };
static inline int2 make_int2(int x, int y) { return {x, y}; }
using std::max;
using std::min;
static inline int64_t min(int64_t a, int b) { return std::min<int64_t>(a, b); }

namespace block {
enum State { kReady, kWarp, kBlock, kDone };
struct Fiber {
  ucontext_t at;
  std::unique_ptr<char[]> stack;
  State state = kReady;
  uint64_t slot = 0;
};
constexpr size_t kStack = 64 << 10;
static std::vector<Fiber> fibers;
static ucontext_t home;
static std::function<void()> body;
static int current;
static std::vector<uint8_t> dynamic_memory;
static uint8_t* dynamic_shared;

static void enter() {
  body();
  fibers[current].state = kDone;
  swapcontext(&fibers[current].at, &home);
}
static void wait(State s) {
  const int me = current;
  fibers[me].state = s;
  swapcontext(&fibers[me].at, &home);
}
// the block of `threads` threads; order: the warps, the one that goes first first
static void run(int threads, const std::vector<int>& order, size_t shared, std::function<void()> f) {
  body = std::move(f);
  dynamic_memory.assign(shared + 1024, 0xa5);
  dynamic_shared = dynamic_memory.data() + (1024 - (reinterpret_cast<uintptr_t>(dynamic_memory.data()) & 1023)) % 1024;
  fibers.clear();
  fibers.resize(threads);
  for (Fiber& x : fibers) {
    x.stack.reset(new char[kStack]);
    getcontext(&x.at);
    x.at.uc_stack.ss_sp = x.stack.get();
    x.at.uc_stack.ss_size = kStack;
    x.at.uc_link = nullptr;
    makecontext(&x.at, enter, 0);
  }
  for (;;) {
    bool ran = false, all_done = true, all_blocked = true;
    for (int w : order) {
      bool warp_waits = true;
      for (int i = 32 * w; i < 32 * w + 32; ++i) {
        while (fibers[i].state == kReady) {
          current = i;
          threadIdx.x = i;
          swapcontext(&home, &fibers[i].at);
          ran = true;
        }
        warp_waits &= fibers[i].state == kWarp;
        all_done &= fibers[i].state == kDone;
        all_blocked &= fibers[i].state == kBlock || fibers[i].state == kDone;
      }
      if (warp_waits) {
        for (int i = 32 * w; i < 32 * w + 32; ++i) fibers[i].state = kReady;
        ran = true;
      }
      if (ran) break;                     // the first warp that can go on goes on
    }
    if (ran) continue;
    if (all_done) return;
    if (!all_blocked) {
      fprintf(stderr, "the block cannot go on\n");
      abort();
    }
    for (Fiber& x : fibers)
      if (x.state == kBlock) x.state = kReady;
  }
}
// f over the warp's slots, once all lanes have posted theirs
template <typename F>
static auto collect(uint64_t mine, F f) {
  const int me = current;
  fibers[me].slot = mine;
  wait(kWarp);
  const auto r = f([me](int lane) { return fibers[(me & ~31) + lane].slot; });
  wait(kWarp);
  return r;
}
}  // namespace block

static inline void __syncthreads() { block::wait(block::kBlock); }
static inline void __syncwarp() { block::wait(block::kWarp); }
static inline int __syncthreads_or(int v) {
  const int me = block::current;
  block::fibers[me].slot = v != 0;
  __syncthreads();
  int r = 0;
  for (const block::Fiber& x : block::fibers) r |= (int)x.slot;
  __syncthreads();
  return r;
}
static inline int __shfl_sync(unsigned, int v, int lane) {
  return block::collect((uint32_t)v, [=](auto at) { return (int)(uint32_t)at(lane); });
}
static inline int __shfl_up_sync(unsigned, int v, int by) {
  const int lane = block::current & 31;
  return block::collect((uint32_t)v, [=](auto at) { return (int)(uint32_t)at(lane >= by ? lane - by : lane); });
}
static inline unsigned __ballot_sync(unsigned, bool p) {
  return block::collect(p, [](auto at) {
    unsigned r = 0;
    for (int i = 0; i < 32; ++i) r |= (at(i) ? 1u : 0u) << i;
    return r;
  });
}
static inline int __reduce_add_sync(unsigned, int v) {
  return block::collect((uint32_t)v, [](auto at) {
    int64_t r = 0;
    for (int i = 0; i < 32; ++i) r += (int)(uint32_t)at(i);
    return (int)r;
  });
}
static inline int __reduce_or_sync(unsigned, int v) {
  return block::collect((uint32_t)v, [](auto at) {
    uint32_t r = 0;
    for (int i = 0; i < 32; ++i) r |= (uint32_t)at(i);
    return (int)r;
  });
}
template <typename T> static inline T __ldcg(const T* p) { return *p; }
template <typename T> static inline T __ldg(const T* p) { return *p; }
static inline int __ffs(int x) { return __builtin_ffs(x); }
static inline int __popc(unsigned x) { return __builtin_popcount(x); }
template <typename T> static inline T atomicAdd(T* p, T v) { const T r = *p; *p += v; return r; }
template <typename T> static inline T atomicSub(T* p, T v) { const T r = *p; *p -= v; return r; }
template <typename T> static inline T atomicOr(T* p, T v) { const T r = *p; *p |= v; return r; }
