// The k largest of n keys, found by one workgroup (pkv_evict.hip, pkv_blocks.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pkv_attn.h"

namespace pkv {
namespace {

// Order of floats as unsigned numbers: -inf 0x007FFFFF .. +inf 0xFF800000; a zero's sign does not count.
__device__ __forceinline__ uint32_t key_of_float(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// The k-th largest of keys 0 .. n - 1 (1 <= k <= n), and how many of those that equal it are among the k largest: eight bits at a time, by
// a count of the keys that agree with what is known so far.  Called by all THREADS threads; `lds`: 258 words.
struct Cutoff {
  uint32_t key;
  int equal;
};
template <int THREADS, typename KeyAt>
__device__ __forceinline__ Cutoff cutoff_of(int n, int k, KeyAt key_at, uint32_t* lds) {
  uint32_t known = 0, mask = 0;
  int left = k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += THREADS) lds[i] = 0;
    __syncthreads();
    for (int r = threadIdx.x; r < n; r += THREADS) {
      const uint32_t key = key_at(r);
      if ((key & mask) == known) atomicAdd(&lds[key >> shift & 255], 1u);
    }
    __syncthreads();
    if (threadIdx.x < 64) {  // lane i: bins 255 - 4 i and the three below
      const int lane = threadIdx.x;
      int c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += c[i] = (int)lds[255 - 4 * lane - i];
      int before = sum_upto(sum) - sum;
      if (before < left && before + sum >= left) {
        int i = 0;
        while (i < 3 && before + c[i] < left) before += c[i++];
        lds[256] = 255 - 4 * lane - i;
        lds[257] = left - before;
      }
    }
    __syncthreads();
    known |= lds[256] << shift;
    left = (int)lds[257];
    mask |= 255u << shift;
    __syncthreads();
  }
  return {known, left};
}

// Numbers of the set flags before a thread's own, in the order of the threads, for two flags at once; `sums`: the numbers of all.
// Called by all THREADS threads; `lds`: 2 * THREADS / 64 words.
struct Two {
  int a, b;
};
template <int THREADS>
__device__ __forceinline__ Two count_before(bool a, bool b, Two& sums, int* lds) {
  constexpr int WAVES = THREADS / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t wa = __ballot(a), wb = __ballot(b), below = ((uint64_t)1 << lane) - 1;
  __syncthreads();  // (what was there has been read)
  if (lane == 0) {
    lds[2 * wave] = __popcll(wa);
    lds[2 * wave + 1] = __popcll(wb);
  }
  __syncthreads();
  Two mine = {(int)__popcll(wa & below), (int)__popcll(wb & below)};
  sums = {0, 0};
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w == wave) mine = {mine.a + sums.a, mine.b + sums.b};
    sums = {sums.a + lds[2 * w], sums.b + lds[2 * w + 1]};
  }
  return mine;
}

}  // namespace
}  // namespace pkv
