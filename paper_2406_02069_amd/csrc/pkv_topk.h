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

// A workgroup's keys: wave w looks after a run of them, kBatch times 64 neighbours at a time, so that ranks need the waves' counts alone.
// The runs are filled up with keys of 0, which all others are above: no pass has an end to look out for.
constexpr int kBatch = 8;
constexpr int kRun = kBatch * kThreads;
template <typename KeyAt>
struct Keys {
  const KeyAt key_at;
  const int steps, first;  // batches of a wave; the lane's first key
  __device__ __forceinline__ Keys(int n, KeyAt key_at_)
      : key_at(key_at_), steps((n + kRun - 1) / kRun), first((int)(threadIdx.x >> 6) * steps * (64 * kBatch) + (int)(threadIdx.x & 63)) {}
  // f(number of the first, keys): keys `number`, number + 64, ..
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    uint32_t next[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) next[k] = key_at(first + 64 * k);
    for (int i = 0; i < steps; ++i) {
      uint32_t key[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) key[k] = next[k];
      const int ahead = first + 64 * kBatch * min(i + 1, steps - 1);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) next[k] = key_at(ahead + 64 * k);
      f(first + 64 * kBatch * i, key);
    }
  }
};

// Keys that wait in LDS between the passes over them: up to so many, as far as a cache can hold that many (kernels take the room as
// dynamic LDS; a workgroup with all of it has a compute unit to itself).  Of more keys, eviction's wait in its workspace, and those of blocks
// are formed again from the scores for each pass.
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
inline int keys_in_lds(int64_t most) { return (int)(most < kKeysInLds ? (most + kRun - 1) / kRun * kRun : kKeysInLds); }

// What a workgroup's selection needs of LDS.
struct SelectLds {
  uint32_t bins[2048];
  int sums[kWavesOf][3];
  int found[3];
  uint64_t keys[kWavesOf];
};

// The sum of the earlier waves' numbers in a column of lds.sums, and of all.
struct Before {
  int mine, all;
};
__device__ __forceinline__ Before before_wave(const SelectLds& lds, int column) {
  static_assert(kWavesOf == 16, "a row of lanes");
  int x = lds.sums[threadIdx.x & 15][column];
  x = add_from<0x111, 0xF>(x);  // row_shr 1, 2, 4, 8
  x = add_from<0x112, 0xF>(x);
  x = add_from<0x114, 0xF>(x);
  x = add_from<0x118, 0xF>(x);
  const int wave = this_wave();
  return {wave > 0 ? __builtin_amdgcn_readlane(x, wave - 1) : 0, __builtin_amdgcn_readlane(x, 15)};
}

__device__ __forceinline__ uint32_t min_of_row(uint32_t x) {  // over 16 lanes
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) x = min(x, (uint32_t)__shfl_xor((int)x, o));
  return x;
}

// The k-th largest key (there are k above 0), and how many of those that equal it are among the k largest, from the first on (`every`:
// all).  Keys of kTop come first, whatever their number; the others' range is counted in up to 2048 parts, then the part that holds the
// k-th key in as many, until all keys of a part are taken or they are equal.  (Eleven bits of the keys themselves at a time, without
// their range, meet a few exponents' parts only where values are alike, and additions to one word of LDS wait for one another: 8192
// scores 14.4 us.)  Where neighbours all meet the same part, they are added at once.
constexpr uint32_t kTop = 0xFFFFFFFFu;
struct Cutoff {
  uint32_t key;
  int equal;
  bool every;
};
// What a thread has met: of keys that are neither 0 nor kTop the least, less one, and the greatest, and one; keys of kTop.
struct Met {
  uint32_t least = ~0u, most = 0;
  int tops = 0;
  __device__ __forceinline__ void meet(uint32_t key) {
    least = min(least, key - 1);
    most = max(most, key + 1);
    tops += key == kTop;
  }
};
template <typename K>
__device__ __forceinline__ Cutoff cutoff_of(const K& keys, const Met& own, int k, SelectLds& lds) {
  const int lane = threadIdx.x & 63;
  uint32_t least = min_of_row(own.least), most = ~min_of_row(~own.most);
  __syncthreads();  // (keys in LDS are there; lds.sums has been read)
  least = min(least, min((uint32_t)__builtin_amdgcn_readlane((int)least, 16), min((uint32_t)__builtin_amdgcn_readlane((int)least, 32), (uint32_t)__builtin_amdgcn_readlane((int)least, 48))));
  most = max(most, max((uint32_t)__builtin_amdgcn_readlane((int)most, 16), max((uint32_t)__builtin_amdgcn_readlane((int)most, 32), (uint32_t)__builtin_amdgcn_readlane((int)most, 48))));
  int tops = __builtin_amdgcn_readlane(sum_upto(own.tops), 63);
  if (lane == 0) {
    lds.sums[this_wave()][0] = tops;
    lds.sums[this_wave()][1] = (int)least;
    lds.sums[this_wave()][2] = (int)most;
  }
  __syncthreads();
  tops = before_wave(lds, 0).all;
  uint32_t low = (uint32_t)__builtin_amdgcn_readfirstlane((int)min_of_row((uint32_t)lds.sums[lane & 15][1])) + 1;
  const uint32_t high = (uint32_t)__builtin_amdgcn_readfirstlane((int)~min_of_row(~(uint32_t)lds.sums[lane & 15][2])) - 1;
  if (tops >= k) {
    __syncthreads();  // (all waves have read lds.sums: equal_before writes there)
    return {kTop, k, tops == k};
  }
  int left = k - tops, met = 0;
  uint32_t span = high - low;  // of the part that is looked at, less one
  for (;;) {
    const int shift = max(21 - __clz((int)(span | 1)), 0);
    lds.bins[threadIdx.x] = lds.bins[threadIdx.x + kThreads] = 0;
    __syncthreads();
    keys.each([&](int, const uint32_t(&key)[kBatch]) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const bool mine = key[i] - low <= span;
        const uint64_t some = __ballot(mine);
        if (some == 0) continue;
        const uint32_t bin = (key[i] - low) >> shift;
        const int lead = __builtin_ctzll(some);
        if (__popcll(some) >= 16 && __ballot(mine && bin == (uint32_t)__builtin_amdgcn_readlane((int)bin, lead)) == some) {
          if (lane == lead) atomicAdd(&lds.bins[bin], (uint32_t)__popcll(some));
        } else if (mine) {
          atomicAdd(&lds.bins[bin], 1u);
        }
      }
    });
    __syncthreads();
    // a thread: two parts, the highest first
    const int top = 2047 - 2 * (int)threadIdx.x;
    const int c0 = (int)lds.bins[top], c1 = (int)lds.bins[top - 1], upto = sum_upto(c0 + c1);
    if (lane == 63) lds.sums[this_wave()][0] = upto;
    __syncthreads();
    const int before = before_wave(lds, 0).mine + upto - c0 - c1;
    if (before < left && left <= before + c0 + c1) {
      const bool second = left > before + c0;
      lds.found[0] = top - second;
      lds.found[1] = left - before - (second ? c0 : 0);
      lds.found[2] = second ? c1 : c0;
    }
    __syncthreads();
    low += (uint32_t)lds.found[0] << shift;
    span = (1u << shift) - 1;
    left = lds.found[1];
    met = lds.found[2];
    if (shift == 0 || left == met) return {low, left, left == met};  // (all above `low` are taken, or all that equal it alike)
  }
}

__device__ __forceinline__ int below_me(uint64_t flags) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(flags >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)flags, 0));
}

// Which of a batch's keys are among the k largest; `equal`: of the keys that equal the cutoff, those before (moves on).
__device__ __forceinline__ void among_largest(const uint32_t (&key)[kBatch], const Cutoff& cut, int& equal, bool (&in)[kBatch]) {
#pragma unroll
  for (int i = 0; i < kBatch; ++i) in[i] = key[i] >= cut.key;
  if (!cut.every) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const uint64_t same = __ballot(key[i] == cut.key);
      in[i] = in[i] && (key[i] != cut.key || equal + below_me(same) < cut.equal);
      equal += __popcll(same);
    }
  }
}
// What the waves before have of keys that equal the cutoff (0 where all of those are taken).
template <typename K>
__device__ __forceinline__ int equal_before(const K& keys, const Cutoff& cut, SelectLds& lds) {
  if (cut.every) return 0;
  int equal = 0;
  keys.each([&](int, const uint32_t(&key)[kBatch]) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) equal += __popcll(__ballot(key[i] == cut.key));
  });
  lds.sums[this_wave()][0] = equal;
  __syncthreads();
  return before_wave(lds, 0).mine;
}

}  // namespace
}  // namespace pkv
