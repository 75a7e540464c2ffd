// The k largest of n keys, found by one workgroup (pkv_evict.hip, pkv_blocks.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pkv_attn.h"

namespace pkv {
namespace {

constexpr int kThreads = 1024, kWavesOf = kThreads / 64;  // of a workgroup that selects

// Order of floats as unsigned numbers: -inf 0x007FFFFF .. +inf 0xFF800000; a zero's sign does not count.
__device__ __forceinline__ uint32_t key_of_float(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// A workgroup's n keys: wave w looks after a run of them, 64 neighbours at a time, so that ranks need the waves' counts alone.  Numbers
// behind the last one are looked up as the last, so that no look-up waits for a comparison.
constexpr int kLookups = 8;  // on their way together
template <typename KeyAt>
struct Keys {
  const KeyAt key_at;
  const int n, steps, first;  // `first`: the lane's first key
  __device__ __forceinline__ Keys(int n_, KeyAt key_at_)
      : key_at(key_at_), n(n_), steps((n_ + kThreads - 1) / kThreads),
        first((int)(threadIdx.x >> 6) * steps * 64 + (int)(threadIdx.x & 63)) {}
  // f(number, key, whether there is such a key) in ascending order, in all lanes of a wave alike
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    for (int i0 = 0; i0 < steps; i0 += kLookups) {
      uint32_t key[kLookups];
#pragma unroll
      for (int i = 0; i < kLookups; ++i) key[i] = key_at(min(first + 64 * (i0 + i), n - 1));
#pragma unroll
      for (int i = 0; i < kLookups; ++i)
        if (i0 + i < steps) f(first + 64 * (i0 + i), key[i], first + 64 * (i0 + i) < n);
    }
  }
};

// Keys that wait in LDS between the passes over them: up to so many, as far as a cache can hold that many (kernels take the room as
// dynamic LDS; a workgroup with all of it has a compute unit to itself).  All others are formed again for each pass.
constexpr int kKeysInLds = 32 * kThreads;
// Raises a kernel's dynamic LDS limit to that, once per device (no allocation).
inline hipError_t grant_keys(const void* kernel, bool* granted) {
  const int dev = current_device_slot();
  if (dev < 0) return hipErrorInvalidDevice;
  if (granted[dev]) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kKeysInLds * (int)sizeof(uint32_t));
  if (e == hipSuccess) granted[dev] = true;
  return e;
}
inline int keys_in_lds(int64_t most) { return (int)(most < kKeysInLds ? (most + 255) / 256 * 256 : kKeysInLds); }

// What a workgroup's selection needs of LDS.
struct SelectLds {
  uint32_t bins[2048];
  int sums[kWavesOf][3];
  int found[3];
  uint64_t keys[kWavesOf];
};

// The k-th largest key (1 <= k <= n), and how many of those that equal it are among the k largest, from the first on (`every`: all).
// Eleven bits at a time, by a count of the keys that agree with what is known so far: with fewer bits the first count would meet a
// few exponents' bins only, and additions to one word of LDS wait for one another.  Where all of 64 neighbours meet the same bin,
// they are added at once.
struct Cutoff {
  uint32_t key;
  int equal;
  bool every;
};
template <typename K>
__device__ __forceinline__ Cutoff cutoff_of(const K& keys, int k, SelectLds& lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t known = 0, mask = 0;
  int left = k, met = 0;
#pragma unroll 1
  for (int shift = 21; shift >= 0; shift = shift == 10 ? 0 : shift - 11) {
    const uint32_t wide = shift == 0 ? 1023 : 2047;
    lds.bins[threadIdx.x] = lds.bins[threadIdx.x + kThreads] = 0;
    __syncthreads();
    keys.each([&](int, uint32_t key, bool there) {
      const bool mine = there && (key & mask) == known;
      const uint64_t some = __ballot(mine);
      if (some == 0) return;
      const uint32_t bin = key >> shift & wide;
      const int lead = __builtin_ctzll(some);
      if (__ballot(mine && bin == (uint32_t)__builtin_amdgcn_readlane((int)bin, lead)) == some) {
        if (lane == lead) atomicAdd(&lds.bins[bin], (uint32_t)__popcll(some));
      } else if (mine) {
        atomicAdd(&lds.bins[bin], 1u);
      }
    });
    __syncthreads();
    // a thread: two bins, the largest first
    const int top = 2047 - 2 * (int)threadIdx.x;
    const int c0 = (int)lds.bins[top], c1 = (int)lds.bins[top - 1], upto = sum_upto(c0 + c1);
    if (lane == 63) lds.sums[wave][0] = upto;
    __syncthreads();
    int before = upto - c0 - c1;
    for (int w = 0; w < wave; ++w) before += lds.sums[w][0];
    if (before < left && left <= before + c0 + c1) {
      const bool second = left > before + c0;
      lds.found[0] = top - second;
      lds.found[1] = left - before - (second ? c0 : 0);
      lds.found[2] = second ? c1 : c0;
    }
    __syncthreads();
    known |= (uint32_t)lds.found[0] << shift;
    left = lds.found[1];
    met = lds.found[2];
    mask |= wide << shift;
  }
  return {known, left, left == met};
}

__device__ __forceinline__ int below_me(uint64_t flags) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(flags >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)flags, 0));
}

// The sums of the earlier waves' numbers a, b, and of all; column `at` and the next of lds.sums.
struct Two {
  int a, b;
};
__device__ __forceinline__ Two before_wave(int a, int b, Two& all, SelectLds& lds) {
  const int wave = threadIdx.x >> 6;
  __syncthreads();  // (what was there has been read)
  if ((threadIdx.x & 63) == 0) {
    lds.sums[wave][1] = a;
    lds.sums[wave][2] = b;
  }
  __syncthreads();
  Two mine = {0, 0};
  all = {0, 0};
#pragma unroll
  for (int w = 0; w < kWavesOf; ++w) {
    if (w == wave) mine = all;
    all = {all.a + lds.sums[w][1], all.b + lds.sums[w][2]};
  }
  return mine;
}

// f(number, whether it is one of the k largest, whether there is such a key) in ascending order.
template <typename K, typename F>
__device__ __forceinline__ void each_of_largest(const K& keys, const Cutoff& cut, int equal_before, F f) {
  int equal = equal_before;  // of the keys before
  keys.each([&](int r, uint32_t key, bool there) {
    bool in = there && key >= cut.key;
    if (!cut.every) {
      const uint64_t same = __ballot(there && key == cut.key);
      in = in && (key != cut.key || equal + below_me(same) < cut.equal);
      equal += __popcll(same);
    }
    f(r, in, there);
  });
}
// What the waves before have of keys that equal the cutoff (0 where all of those are taken).
template <typename K>
__device__ __forceinline__ int equal_before(const K& keys, const Cutoff& cut, SelectLds& lds) {
  if (cut.every) return 0;
  int equal = 0;
  keys.each([&](int, uint32_t key, bool there) { equal += __popcll(__ballot(there && key == cut.key)); });
  Two all;
  return before_wave(equal, 0, all, lds).a;
}

}  // namespace
}  // namespace pkv
