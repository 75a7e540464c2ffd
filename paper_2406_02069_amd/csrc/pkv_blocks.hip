// Attention over the blocks of a cache that a bound on their scores selects (include/pkv.h: pkv_block_bounds, pkv_block_select,
// pkv_decode_attention_blocks).
//
//   bounds  a wave takes a block's rows whole, eight channels a lane, and joins the lanes that have the same channels.  HBM-bound: 2 x 8
//           heads of 32k rows, d 128 (134 MB), 26.6 us, 5 TB/s; a chunk of 300 rows in 8 sequences of 4 heads 7.6.
//   select  sum_h sum_i q_hi (q_hi < 0 ? lo_i : hi_i) = sum_i P_i hi_i + N_i lo_i with P_i = sum_h max(q_hi, 0), N_i = sum_h min(q_hi, 0)
//           (where bounds are finite): one product of 2 d numbers a block for all heads of a group, in 64 bits (16-bit numbers'
//           products and their sums are exact there but for extreme spreads), so that which blocks are taken does not hang on an
//           order of additions.
//           HBM-bound, 512 bytes a block at d 128: 164k blocks 17.5 us, 4.8 TB/s.
//           Then a workgroup per (sequence, KV head) finds the smallest score that is taken (pkv_topk.h) and lists the blocks in
//           order: 7.5 us of 512 blocks, 9.4 of 8192, launch and barriers for the most part.
//   attention  pkv_decode_long.hip's kernel, which looks its rows up in the list.
#include "pkv_long.h"
#include "pkv_topk.h"

namespace pkv {
namespace {

struct BoundsArgs {
  const uint16_t* K;
  const int32_t *table, *count, *new_lens;
  uint16_t* bounds;
  int32_t B, Hkv, k_cap, page_size, num_pages, max_pages, shift;
  uint32_t page_magic;
  int64_t c_sb, c_sh, c_st, b_sb, b_sh;
};

// Pairs of 16-bit numbers as integers in the numbers' order (its own inverse); a NaN lies beyond the infinity of its sign.
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ s16x2 as_pair(uint32_t x) { return __builtin_bit_cast(s16x2, x); }
__device__ __forceinline__ uint32_t as_word(s16x2 x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ s16x2 in_order(s16x2 x) { return x ^ (s16x2)((x >> 15) & (short)0x7FFF); }
// The least (MAX: the greatest) of both halves' pairs, over the lanes that have the same channels.
template <bool MAX>
__device__ __forceinline__ s16x2 better(s16x2 x, s16x2 y) { return MAX ? __builtin_elementwise_max(x, y) : __builtin_elementwise_min(x, y); }
template <int LANES, bool MAX>
__device__ __forceinline__ s16x2 over_rows(s16x2 x) {
  const u32x2 h = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(as_word(x), as_word(x), false, false));
  x = better<MAX>(as_pair(h[0]), as_pair(h[1]));
  const u32x2 q = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(as_word(x), as_word(x), false, false));
  x = better<MAX>(as_pair(q[0]), as_pair(q[1]));
  if constexpr (LANES == 8)  // row_ror 8
    x = better<MAX>(x, as_pair((uint32_t)__builtin_amdgcn_update_dpp(0, (int)as_word(x), 0x128, 0xF, 0xF, true)));
  return x;
}

// blockIdx: (sequence, KV head) x chunks of four blocks, a wave each, from the first one that is asked for on.
constexpr int kAtOnce = 4;  // loads of a lane on their way together
template <typename T, int D>
__global__ __launch_bounds__(256) void bounds_kernel(const BoundsArgs a, int chunks) {
  constexpr int LANES = D / 8, ROWS = 64 / LANES;
  constexpr short INF = __is_same(T, __bf16) ? 0x7F80 : 0x7C00, MINUS_INF = ~INF;  // in order
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int unit = blockIdx.x / chunks, b = unit / a.Hkv, g = unit % a.Hkv;
  const int n = min(max(a.count[b], 0), a.k_cap), fresh = a.new_lens ? min(max(a.new_lens[b], 0), n) : n;
  if (fresh == 0) return;
  const int end = (n - 1) >> a.shift;
  const int32_t* const table = a.table + (int64_t)b * a.max_pages;
  for (int blk = ((n - fresh) >> a.shift) + (int)(blockIdx.x % chunks) * 4 + wave; blk <= end; blk += 4 * chunks) {
    s16x2 lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = (s16x2)(short)0x7FFF;
      hi[i] = (s16x2)(short)0x8000;
    }
    bool some = false;
    const int last = min(((blk + 1) << a.shift) - 1, n - 1);
    for (int j0 = blk << a.shift; j0 <= last; j0 += kAtOnce * ROWS) {
      int64_t at[kAtOnce];
      bool is[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {  // (rows behind the last one are taken as the last)
        const int j = min(j0 + k * ROWS + lane / LANES, last);
        at[k] = b * a.c_sb + g * a.c_sh + j * a.c_st;
        is[k] = true;
        if (a.page_size) {
          uint32_t p = __umulhi((uint32_t)j, a.page_magic);
          if ((uint32_t)j - p * a.page_size >= (uint32_t)a.page_size) ++p;
          const uint32_t page = (uint32_t)table[p];
          is[k] = page < (uint32_t)a.num_pages;
          at[k] = is[k] ? (((int64_t)page * a.Hkv + g) * a.page_size + (j - p * a.page_size)) * D : 0;
        }
      }
      u32x4 v[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) v[k] = *reinterpret_cast<const u32x4*>(a.K + at[k] + 8 * (lane % LANES));
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        some = some || is[k];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const s16x2 x = in_order(as_pair(v[k][i]));
          lo[i] = is[k] ? better<false>(lo[i], x) : lo[i];
          hi[i] = is[k] ? better<true>(hi[i], x) : hi[i];
        }
      }
    }
    const bool any = __any(some);
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s16x2 l = over_rows<LANES, false>(lo[i]), h = over_rows<LANES, true>(hi[i]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const bool nan = l[e] < MINUS_INF || h[e] > INF;
        l[e] = nan ? MINUS_INF : l[e];
        h[e] = nan ? INF : h[e];
      }
      w[i] = any ? as_word(in_order(lane < LANES ? l : h)) : 0;  // the first lanes write the least values, the next the greatest
    }
    if (lane < 2 * LANES) *reinterpret_cast<u32x4*>(a.bounds + b * a.b_sb + g * a.b_sh + (int64_t)blk * 2 * D + 8 * lane) = w;
  }
}

struct SelectArgs {
  const uint16_t *q, *bounds;
  const int32_t* count;
  int32_t* blocks;
  float* scores;  // [B][Hkv][all]
  int32_t B, Hkv, G, k_cap, shift, all, most, first, recent;
  int32_t in_lds;  // keys that the launch of block_list_kernel has room for
  int64_t q_sb, q_sh, b_sb, b_sh;
};

// A wave: kLoads times 1 KB of neighbouring blocks' bounds, requested together, 16 bytes of a block's 2 D numbers a lane.  A block's sum
// is spread over LANES lanes: the first steps of adding up halve the number of sums that a lane looks after.
constexpr int kLoads = 8;
template <int D>
constexpr int blocks_of_wave() { return kLoads * 64 / (D / 4); }
template <typename T, int D>
__global__ __launch_bounds__(256) void block_score_kernel(const SelectArgs a, int chunks) {
  constexpr int LANES = D / 4, AT_ONCE = 64 / LANES, OWN = blocks_of_wave<D>();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, piece = lane % LANES;
  const int unit = blockIdx.x / chunks, b = unit / a.Hkv, g = unit % a.Hkv;
  const int n = min(max(a.count[b], 0), a.k_cap), have = (n + (1 << a.shift) - 1) >> a.shift;
  __shared__ __align__(16) double coefficients[2 * D];
  if ((int64_t)(blockIdx.x % chunks) * 4 * OWN >= have) return;
  int blk0 = (int)(blockIdx.x % chunks * 4 + wave) * OWN;
  const uint16_t* const from = a.bounds + b * a.b_sb + g * a.b_sh + 8 * piece;
  u32x4 v[kLoads], w[kLoads];
  auto load = [&](int blk, u32x4 (&v)[kLoads]) {
    if (blk + OWN <= have) {
      const uint16_t* const first = from + (int64_t)(blk + lane / LANES) * (2 * D);
#pragma unroll
      for (int k = 0; k < kLoads; ++k) v[k] = *reinterpret_cast<const u32x4*>(first + k * AT_ONCE * 2 * D);
      return;
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      v[k] = *reinterpret_cast<const u32x4*>(from + (int64_t)min(blk + k * AT_ONCE + lane / LANES, have - 1) * (2 * D));
  };
  load(min(blk0, have - 1), v);
  // the heads' coefficients, a thread each: of the least values first
  static_assert(2 * D <= 256, "a thread for each coefficient");
  if (threadIdx.x < 2 * D) {
    const uint16_t* const qp = a.q + b * a.q_sb + (int64_t)g * a.G * a.q_sh + threadIdx.x % D;
    double c = 0.0;
    for (int h0 = 0; h0 < a.G; h0 += 8) {  // eight heads' loads at once
      uint16_t q[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) q[k] = qp[min(h0 + k, a.G - 1) * a.q_sh];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float x = unpack<T>(q[k], 0);
        c += h0 + k < a.G && (x != x || (x < 0.0f) == (threadIdx.x < D)) ? (double)x : 0.0;
      }
    }
    coefficients[threadIdx.x] = c;
  }
  __syncthreads();
  double f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = coefficients[8 * piece + i];
  while (blk0 < have) {
    const int next = blk0 + chunks * 4 * OWN;  // (blocks are 2^26 at most, a turn of all chunks 2^17)
    if (next < have) load(next, w);
    double s[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      s[k] = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) s[k] = __builtin_fma(f[i], (double)unpack<T>(v[k][i >> 1], i & 1), s[k]);
    }
    static_assert(kLoads == 8, "three halvings");
#pragma unroll
    for (int i = 0; i < 3; ++i) {
#pragma unroll
      for (int k = 0; k < kLoads / 2; ++k) {
        const int half = kLoads >> (i + 1), o = 1 << i;
        if (k < half) {
          const bool upper = lane & o;
          const double x = s[k], y = s[k + half], keep = upper ? y : x, give = upper ? x : y;
          s[k] = keep + __shfl_xor(give, o);
        }
      }
    }
#pragma unroll
    for (int o = kLoads; o < LANES; o <<= 1) s[0] += __shfl_xor(s[0], o);
    // (lane bits 0, 1, 2 chose bits 2, 1, 0 of the load's number)
    const int blk = blk0 + (((lane & 1) << 2) | (lane & 2) | ((lane >> 2) & 1)) * AT_ONCE + lane / LANES;
    if (piece < kLoads && blk < have) {
      float x = (float)s[0];
      if (__builtin_expect(!(fabsf(x) < __builtin_inff()), 0)) {  // a coefficient of 0 times a bound that is not finite: term by term
        const uint16_t *const qp = a.q + b * a.q_sb + (int64_t)g * a.G * a.q_sh, *const own = a.bounds + b * a.b_sb + g * a.b_sh + (int64_t)blk * (2 * D);
        double sum = 0.0;
#pragma unroll 1
        for (int h = 0; h < a.G; ++h) {
#pragma unroll 8
          for (int i = 0; i < D; ++i) {
            const float y = unpack<T>(qp[h * a.q_sh + i], 0);
            sum = __builtin_fma((double)y, (double)unpack<T>(own[(y < 0.0f ? 0 : D) + i], 0), sum);
          }
        }
        x = (float)sum;
      }
      a.scores[(int64_t)unit * a.all + blk] = x == x ? x : __builtin_inff();
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k) v[k] = w[k];
    blk0 = next;
  }
}

template <typename KeyAt>
__device__ __forceinline__ void list_blocks(const SelectArgs& a, int unit, int have, KeyAt key_at, const Met& met, SelectLds& lds) {
  int32_t* const out = a.blocks + (int64_t)unit * a.most;
  const Keys<KeyAt> keys(have, key_at);
  const Cutoff cut = cutoff_of(keys, met, a.most, lds);
  const int equal0 = equal_before(keys, cut, lds);
  int equal = equal0, taken = 0;
  keys.each([&](int, const uint32_t(&key)[kBatch]) {
    bool in[kBatch];
    among_largest(key, cut, equal, in);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) taken += __popcll(__ballot(in[i]));
  });
  lds.sums[this_wave()][2] = taken;
  __syncthreads();
  taken = before_wave(lds, 2).mine;
  equal = equal0;
  keys.each([&](int k, const uint32_t(&key)[kBatch]) {
    bool in[kBatch];
    among_largest(key, cut, equal, in);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const uint64_t some = __ballot(in[i]);
      if (in[i]) out[taken + below_me(some)] = k + 64 * i;
      taken += __popcll(some);
    }
  });
}

__global__ __launch_bounds__(kThreads) void block_list_kernel(const SelectArgs a) {
  __shared__ SelectLds lds;
  extern __shared__ uint32_t kept[];
  const int unit = blockIdx.x, b = unit / a.Hkv;
  const int n = min(max(a.count[b], 0), a.k_cap), have = (n + (1 << a.shift) - 1) >> a.shift;
  const float* const score = a.scores + (int64_t)unit * a.all;
  auto key_at = [&](int k) {
    const uint32_t key = key_of_float(score[min(k, have - 1)]);
    return k >= have ? 0u : k < a.first || k >= have - a.recent ? kTop : key;
  };
  Met met;
  if (have <= a.most) {
    for (int i = threadIdx.x; i < a.most; i += kThreads) a.blocks[(int64_t)unit * a.most + i] = i < have ? i : -1;
  } else if (have <= a.in_lds) {
    for (int k0 = 0; k0 < have; k0 += kRun) {
      uint32_t key[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) key[i] = key_at(k0 + (int)threadIdx.x + i * kThreads);
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        met.meet(key[i]);
        kept[k0 + (int)threadIdx.x + i * kThreads] = key[i];
      }
    }
    list_blocks(a, unit, have, [&](int k) { return kept[k]; }, met, lds);  // (its first barrier comes before the first look-up)
  } else {
    for (int k0 = 0; k0 < have; k0 += kRun) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) met.meet(key_at(k0 + (int)threadIdx.x + i * kThreads));
    }
    list_blocks(a, unit, have, key_at, met, lds);
  }
}

int shift_of(int block) {
  for (int s = 4; s <= 8; ++s)
    if (block == 1 << s) return s;
  return -1;
}

// What all three calls ask; `queries`: those that take some.
int check_block_desc(const pkv_block_desc* desc, bool queries, bool cache) {
  if (!desc) return PKV_ERR_INVALID_ARG;
  const pkv_block_desc& d = *desc;
  if (d.B < 1 || d.Hkv < 1 || d.k_cap < 1 || d.block < 1 || d.reserved != 0 || (d.dtype != PKV_BF16 && d.dtype != PKV_FP16)) return PKV_ERR_INVALID_ARG;
  if (queries && (check_scores(d) != PKV_OK || d.most < 1)) return PKV_ERR_INVALID_ARG;
  if (cache && check_pages(d) != PKV_OK) return PKV_ERR_INVALID_ARG;
  if (shift_of(d.block) < 0) return PKV_ERR_UNSUPPORTED;
  if ((int64_t)d.B * d.Hkv >= 1 << 22) return PKV_ERR_UNSUPPORTED;  // (workgroups of 1024: 2^32 threads)
  if (queries && (d.most > 1 << 30 || d.Hq / d.Hkv > 128 || (int64_t)d.B * d.Hq > kMaxGrid)) return PKV_ERR_UNSUPPORTED;
  if (cache) return check_cache_limits(d);
  return (d.d != 64 && d.d != 128) || d.B > 65535 || d.Hkv > 65535 || d.k_cap > (1 << 30) ? PKV_ERR_UNSUPPORTED : PKV_OK;
}
int check_select_desc(const pkv_block_desc* desc) {
  const int rc = check_block_desc(desc, true, false);
  if (rc != PKV_OK && rc != PKV_ERR_UNSUPPORTED) return rc;
  if (desc->first < 0 || desc->recent < 0 || (int64_t)desc->first + desc->recent > desc->most || !good_strides(desc->b_sb, desc->b_sh, 0))
    return PKV_ERR_INVALID_ARG;
  return rc;
}
int check_attention_desc(const pkv_block_desc* desc) {
  const int rc = check_block_desc(desc, true, true);
  if (rc != PKV_OK) return rc;
  if (check_factors(*desc) != PKV_OK) return PKV_ERR_INVALID_ARG;
  return (int64_t)desc->most * desc->block > 1 << 30 ? PKV_ERR_UNSUPPORTED : PKV_OK;
}

int64_t blocks_of(const pkv_block_desc& d) { return ((int64_t)d.k_cap + d.block - 1) / d.block; }

Grid grid_of(const pkv_block_desc& d) {
  const int64_t listed = (int64_t)d.most * d.block;
  return grid_of(d.B, d.Hkv, d.Hq / d.Hkv, listed < d.k_cap ? listed : d.k_cap);
}

// Workgroups of `per` blocks each for every head: as many as a cache's blocks need, but in all no more than the device holds at a time.
// Most of the blocks of a large cache are not there, or not asked for, and a workgroup that finds nothing to do still has to be started:
// the bounds of one new row of 4 x 8 heads with room for 128k rows take 31 us in 65536 workgroups.
int chunks_of(int64_t blocks, int per, int64_t units, int at_a_time) {
  const int64_t chunks = (blocks + per - 1) / per, most = (at_a_time + units - 1) / units;
  return (int)(chunks < most ? chunks : most);
}

}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

int pkv_block_bounds(const pkv_block_desc* desc, const void* K_cache, const int32_t* block_table, const int32_t* count,
                     const int32_t* new_lens, void* bounds, void* stream) {
  if (!desc || !K_cache || !count || !bounds) return PKV_ERR_INVALID_ARG;
  const int rc = check_block_desc(desc, false, true);
  if (rc != PKV_OK) return rc;
  const pkv_block_desc& d = *desc;
  if (!good_strides(d.b_sb, d.b_sh, 0) || !aligned(K_cache, 16) || !aligned(bounds, 16) || !aligned(block_table, 4) || !aligned(count, 4) ||
      !aligned(new_lens, 4) || (d.page_size > 0 && !block_table) || !apart(blocks_of(d) * 2 * d.d, {{d.B, d.b_sb}, {d.Hkv, d.b_sh}}))
    return PKV_ERR_INVALID_ARG;
  BoundsArgs a;
  memset(&a, 0, sizeof(a));
  a.K = static_cast<const uint16_t*>(K_cache);
  a.table = block_table; a.count = count; a.new_lens = new_lens;
  a.bounds = static_cast<uint16_t*>(bounds);
  a.B = d.B; a.Hkv = d.Hkv; a.k_cap = d.k_cap; a.page_size = d.page_size; a.num_pages = d.num_pages; a.max_pages = d.max_pages;
  a.shift = shift_of(d.block);
  a.page_magic = magic_of(d.page_size);
  a.c_sb = d.c_sb; a.c_sh = d.c_sh; a.c_st = d.c_st; a.b_sb = d.b_sb; a.b_sh = d.b_sh;
  const int64_t units = (int64_t)d.B * d.Hkv;
  const int chunks = chunks_of(blocks_of(d), 4, units, 2048);
  const dim3 grid((unsigned)(units * chunks)), block(256);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (d.dtype == PKV_BF16) {
    if (d.d == 128) hipLaunchKernelGGL((bounds_kernel<__bf16, 128>), grid, block, 0, st, a, chunks);
    else hipLaunchKernelGGL((bounds_kernel<__bf16, 64>), grid, block, 0, st, a, chunks);
  } else {
    if (d.d == 128) hipLaunchKernelGGL((bounds_kernel<_Float16, 128>), grid, block, 0, st, a, chunks);
    else hipLaunchKernelGGL((bounds_kernel<_Float16, 64>), grid, block, 0, st, a, chunks);
  }
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

size_t pkv_block_select_workspace_bytes(const pkv_block_desc* desc) {
  return check_select_desc(desc) == PKV_OK ? (size_t)desc->B * desc->Hkv * blocks_of(*desc) * sizeof(float) : 0;
}

int pkv_block_select(const pkv_block_desc* desc, const void* q, const void* bounds, const int32_t* count, int32_t* blocks_out,
                     float* scores_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc || !q || !bounds || !count || !blocks_out) return PKV_ERR_INVALID_ARG;
  const int rc = check_select_desc(desc);
  if (rc != PKV_OK) return rc;
  const pkv_block_desc& d = *desc;
  if (!aligned(q, 16) || !aligned(bounds, 16) || !aligned(count, 4) || !aligned(blocks_out, 4) || !aligned(scores_out, 4)) return PKV_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < pkv_block_select_workspace_bytes(desc)) return PKV_ERR_WORKSPACE;
  SelectArgs a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const uint16_t*>(q);
  a.bounds = static_cast<const uint16_t*>(bounds);
  a.count = count; a.blocks = blocks_out;
  a.scores = scores_out ? scores_out : static_cast<float*>(workspace);
  a.B = d.B; a.Hkv = d.Hkv; a.G = d.Hq / d.Hkv; a.k_cap = d.k_cap; a.shift = shift_of(d.block); a.all = (int32_t)blocks_of(d);
  a.most = d.most; a.first = d.first; a.recent = d.recent;
  a.q_sb = d.q_sb; a.q_sh = d.q_sh; a.b_sb = d.b_sb; a.b_sh = d.b_sh;
  a.in_lds = keys_in_lds(a.all);
  static bool granted[kMaxDevices];
  if (grant_keys(reinterpret_cast<const void*>(block_list_kernel), granted) != hipSuccess) return PKV_ERR_HIP;
  const int64_t units = (int64_t)d.B * d.Hkv;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int chunks = chunks_of(a.all, 4 * (d.d == 128 ? blocks_of_wave<128>() : blocks_of_wave<64>()), units, 1024);
  const dim3 grid((unsigned)(units * chunks)), block(256);
  if (d.dtype == PKV_BF16) {
    if (d.d == 128) hipLaunchKernelGGL((block_score_kernel<__bf16, 128>), grid, block, 0, st, a, chunks);
    else hipLaunchKernelGGL((block_score_kernel<__bf16, 64>), grid, block, 0, st, a, chunks);
  } else {
    if (d.d == 128) hipLaunchKernelGGL((block_score_kernel<_Float16, 128>), grid, block, 0, st, a, chunks);
    else hipLaunchKernelGGL((block_score_kernel<_Float16, 64>), grid, block, 0, st, a, chunks);
  }
  if (hipGetLastError() != hipSuccess) return PKV_ERR_HIP;
  hipLaunchKernelGGL(block_list_kernel, dim3((unsigned)units), dim3(kThreads), (size_t)a.in_lds * sizeof(uint32_t), st, a);
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

size_t pkv_decode_blocks_workspace_bytes(const pkv_block_desc* desc) {
  if (check_attention_desc(desc) != PKV_OK) return 0;
  return parts_bytes(grid_of(*desc), desc->Hq / desc->Hkv, desc->d);
}

int pkv_decode_attention_blocks(const pkv_block_desc* desc, const void* q, const void* K_cache, const void* V_cache,
                                const int32_t* block_table, const int32_t* count, const int32_t* blocks, void* out, float* lse_out,
                                void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc || !q || !K_cache || !V_cache || !count || !blocks || !out) return PKV_ERR_INVALID_ARG;
  const int rc = check_attention_desc(desc);
  if (rc != PKV_OK) return rc;
  const pkv_block_desc& d = *desc;
  if (!aligned(q, 16) || !aligned(K_cache, 16) || !aligned(V_cache, 16) || !aligned(out, 16) || !aligned(block_table, 4) ||
      !aligned(count, 4) || !aligned(blocks, 4) || !aligned(lse_out, 4) || (d.page_size > 0 && !block_table))
    return PKV_ERR_INVALID_ARG;
  const size_t need = pkv_decode_blocks_workspace_bytes(desc);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return PKV_ERR_WORKSPACE;
  BlocksArgs a;
  memset(&a, 0, sizeof(a));
  const Grid grid = grid_of(d);
  fill_long(a, d, grid, d.Hq / d.Hkv, q, K_cache, V_cache, out, workspace);
  a.table = block_table; a.count = count; a.blocks = blocks;
  a.lse = lse_out;
  a.most = d.most; a.shift = shift_of(d.block);
  const hipError_t e = launch_long(a, d.dtype, d.d, grid.workgroups, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
