// A workgroup of 16 waves on the CPU, as far as csrc/pkv_topk.h needs one: a fiber for each lane.  Lanes of a wave meet at operations
// across lanes; waves meet at barriers alone and run from one to the next in an order that the test chooses, which is what the hardware
// may do.
#pragma once

#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <ucontext.h>

#include <functional>
#include <vector>

#define __device__
#define __global__
#define __forceinline__ inline

typedef int hipError_t;
constexpr hipError_t hipSuccess = 0, hipErrorInvalidDevice = 101;
constexpr int hipFuncAttributeMaxDynamicSharedMemorySize = 8;
inline hipError_t hipFuncSetAttribute(const void*, int, int) { return hipSuccess; }

namespace emulated {

struct Index {
  unsigned x;
};
enum State { kRuns, kAtReadlane, kAtOther, kAtBarrier, kDone };
struct Lane {
  ucontext_t context;
  Index index;
  State state;
  uint64_t given, met[64], there;  // what the wave's lanes gave at the last operation, and which of them took part
};
inline std::vector<Lane> lanes;
inline Lane* current;
inline ucontext_t scheduler;
inline std::function<void()> body;

inline void park(State s) {
  Lane* const me = current;
  me->state = s;
  swapcontext(&me->context, &scheduler);
}
inline const Lane& across(uint64_t x, State s) {
  current->given = x;
  park(s);
  return *current;
}
inline void start() {
  body();
  park(kDone);
}

// Runs `kernel` in 16 waves, those with a low rank first; false: more than `most` barriers.
inline bool run(const std::vector<int>& rank, int most, std::function<void()> kernel) {
  constexpr int kWaves = 16, kStack = 1 << 16;
  static std::vector<char> stacks((size_t)kWaves * 64 * kStack);
  body = std::move(kernel);
  lanes.assign(kWaves * 64, Lane());
  for (int i = 0; i < kWaves * 64; ++i) {
    Lane& l = lanes[i];
    getcontext(&l.context);
    l.context.uc_stack.ss_sp = &stacks[(size_t)i * kStack];
    l.context.uc_stack.ss_size = kStack;
    l.context.uc_link = nullptr;
    l.index.x = (unsigned)i;
    l.state = kRuns;
    makecontext(&l.context, start, 0);
  }
  std::vector<int> order(kWaves);
  for (int w = 0; w < kWaves; ++w) order[rank[w]] = w;
  for (int barriers = 0;; ++barriers) {
    bool all_done = true;
    for (int w : order) {
      Lane* const of = &lanes[w * 64];
      for (;;) {
        for (int l = 0; l < 64; ++l) {
          if (of[l].state != kRuns) continue;
          current = &of[l];
          swapcontext(&scheduler, &of[l].context);
        }
        uint64_t readlane = 0, other = 0;
        for (int l = 0; l < 64; ++l) {
          readlane |= (uint64_t)(of[l].state == kAtReadlane) << l;
          other |= (uint64_t)(of[l].state == kAtOther) << l;
        }
        const uint64_t now = readlane ? readlane : other;  // (lanes that a condition kept from a readlane wait behind it)
        if (!now) break;
        for (int l = 0; l < 64; ++l) {
          if (!(now >> l & 1)) continue;
          for (int k = 0; k < 64; ++k) of[l].met[k] = of[k].given;
          of[l].there = now;
          of[l].state = kRuns;
        }
      }
      all_done = all_done && of[0].state == kDone;
    }
    if (all_done) return true;
    if (barriers == most) return false;
    for (Lane& l : lanes)
      if (l.state == kAtBarrier) l.state = kRuns;
  }
}

}  // namespace emulated

#define threadIdx (emulated::current->index)

inline void __syncthreads() { emulated::park(emulated::kAtBarrier); }
inline uint64_t __ballot(bool x) {
  const emulated::Lane& l = emulated::across(x, emulated::kAtOther);
  uint64_t r = 0;
  for (int k = 0; k < 64; ++k) r |= (uint64_t)((l.there >> k & 1) && l.met[k]) << k;
  return r;
}
inline int __shfl_xor(int x, int o) { return (int)emulated::across((uint32_t)x, emulated::kAtOther).met[(threadIdx.x & 63) ^ o]; }
inline int __builtin_amdgcn_readlane(int x, int lane) { return (int)emulated::across((uint32_t)x, emulated::kAtReadlane).met[lane]; }
inline int __builtin_amdgcn_readfirstlane(int x) {
  const emulated::Lane& l = emulated::across((uint32_t)x, emulated::kAtReadlane);
  return (int)l.met[__builtin_ctzll(l.there)];
}
inline int __builtin_amdgcn_mbcnt_lo(uint32_t m, int x) {
  const int lane = threadIdx.x & 63;
  return x + __builtin_popcount(m & (lane >= 32 ? ~0u : (1u << lane) - 1));
}
inline int __builtin_amdgcn_mbcnt_hi(uint32_t m, int x) {
  const int lane = threadIdx.x & 63;
  return x + (lane < 32 ? 0 : __builtin_popcount(m & ((1u << (lane - 32)) - 1)));
}
inline int __popcll(uint64_t x) { return __builtin_popcountll(x); }
inline int __clz(int x) { return x ? __builtin_clz((unsigned)x) : 32; }
inline uint32_t __float_as_uint(float x) {
  uint32_t u;
  memcpy(&u, &x, 4);
  return u;
}
inline uint32_t atomicAdd(uint32_t* p, uint32_t x) {
  const uint32_t old = *p;
  *p = old + x;
  return old;
}
template <typename T>
inline T min(T a, T b) { return b < a ? b : a; }
template <typename T>
inline T max(T a, T b) { return a < b ? b : a; }
