// Attention over the blocks of a cache that a bound on their scores selects (include/pkv.h: pkv_block_bounds, pkv_block_select,
// pkv_decode_attention_blocks).
//
//   bounds  a wave takes a block's rows whole, eight channels a lane, and joins the lanes that have the same channels.
//   select  sum_h sum_i max(q_hi lo_i, q_hi hi_i) = sum_i P_i hi_i + N_i lo_i with P_i = sum_h max(q_hi, 0), N_i = sum_h min(q_hi, 0):
//           one product of 2 d numbers a block for all heads of a group, in 64 bits (16-bit numbers' products and their sums are
//           exact there but for extreme spreads), so that which blocks are taken does not hang on an order of additions.
//           Then a workgroup per (sequence, KV head) finds the smallest score that is taken and lists the blocks in order.
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

// blockIdx: (sequence, KV head) x chunks of four blocks, a wave each, from the first one that is asked for on.
template <typename T, int D>
__global__ __launch_bounds__(256) void bounds_kernel(const BoundsArgs a, int chunks) {
  constexpr int LANES = D / 8, ROWS = 64 / LANES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int unit = blockIdx.x / chunks, b = unit / a.Hkv, g = unit % a.Hkv;
  const int n = min(max(a.count[b], 0), a.k_cap), fresh = a.new_lens ? min(max(a.new_lens[b], 0), n) : n;
  if (fresh == 0) return;
  const int end = (n - 1) >> a.shift;
  for (int blk = ((n - fresh) >> a.shift) + (int)(blockIdx.x % chunks) * 4 + wave; blk <= end; blk += 4 * chunks) {
    float lo[8], hi[8];
    int odd[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[i] = __builtin_inff();
      hi[i] = -__builtin_inff();
      odd[i] = 0;
    }
    bool some = false;
    const int last = min(((blk + 1) << a.shift) - 1, n - 1);
    for (int j = (blk << a.shift) + lane / LANES; j <= last; j += ROWS) {
      int64_t at = b * a.c_sb + g * a.c_sh + j * a.c_st;
      if (a.page_size) {
        uint32_t p = __umulhi((uint32_t)j, a.page_magic);
        if ((uint32_t)j - p * a.page_size >= (uint32_t)a.page_size) ++p;
        const int32_t page = a.table[(int64_t)b * a.max_pages + p];
        if ((uint32_t)page >= (uint32_t)a.num_pages) continue;
        at = (((int64_t)page * a.Hkv + g) * a.page_size + (j - p * a.page_size)) * D;
      }
      const u32x4 v = *reinterpret_cast<const u32x4*>(a.K + at + 8 * (lane % LANES));
      some = true;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = unpack<T>(v[i >> 1], i & 1);
        odd[i] |= x != x;
        lo[i] = fminf(lo[i], x);
        hi[i] = fmaxf(hi[i], x);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int o = LANES; o < 64; o <<= 1) {
        lo[i] = fminf(lo[i], __shfl_xor(lo[i], o));
        hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], o));
        odd[i] |= __shfl_xor(odd[i], o);
      }
      if (odd[i]) {
        lo[i] = -__builtin_inff();
        hi[i] = __builtin_inff();
      }
    }
    if (!__any(some)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) lo[i] = hi[i] = 0.0f;
    }
    if (lane < 2 * LANES) {  // the first lanes write the least values, the next the greatest
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = lane < LANES ? pack2<T>(lo[2 * i], lo[2 * i + 1]) : pack2<T>(hi[2 * i], hi[2 * i + 1]);
      *reinterpret_cast<u32x4*>(a.bounds + b * a.b_sb + g * a.b_sh + (int64_t)blk * 2 * D + 8 * lane) = w;
    }
  }
}

struct SelectArgs {
  const uint16_t *q, *bounds;
  const int32_t* count;
  int32_t* blocks;
  float* scores;  // [B][Hkv][all]
  int32_t B, Hkv, G, k_cap, shift, all, most, first, recent;
  int64_t q_sb, q_sh, b_sb, b_sh;
};

// A wave: 64 / (D / 4) blocks at a time, 16 bytes of a block's 2 D numbers a lane.
constexpr int kScoreBlocks = 64;  // of a workgroup
template <typename T, int D>
__global__ __launch_bounds__(256) void block_score_kernel(const SelectArgs a, int chunks) {
  constexpr int LANES = D / 4, AT_ONCE = 64 / LANES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, piece = lane % LANES;
  const int unit = blockIdx.x / chunks, b = unit / a.Hkv, g = unit % a.Hkv;
  const int n = min(max(a.count[b], 0), a.k_cap), have = (n + (1 << a.shift) - 1) >> a.shift;
  const bool least = piece < LANES / 2;
  int c = (int)(blockIdx.x % chunks);
  if ((int64_t)c * kScoreBlocks >= have) return;
  double f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = 0.0;
  for (int h = 0; h < a.G; ++h) {
    const u32x4 q = *reinterpret_cast<const u32x4*>(a.q + b * a.q_sb + (g * a.G + h) * a.q_sh + 8 * (piece % (LANES / 2)));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = unpack<T>(q[i >> 1], i & 1);
      f[i] += x != x ? (double)x : (x < 0.0f) == least ? (double)x : 0.0;
    }
  }
  const uint16_t* const from = a.bounds + b * a.b_sb + g * a.b_sh + 8 * piece;
  for (; (int64_t)c * kScoreBlocks < have; c += chunks) {
    for (int k = AT_ONCE * wave; k < kScoreBlocks; k += 4 * AT_ONCE) {
      const int blk = c * kScoreBlocks + k + lane / LANES;
      const u32x4 v = *reinterpret_cast<const u32x4*>(from + (int64_t)min(blk, have - 1) * 2 * D);
      double s = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __builtin_fma(f[i], (double)unpack<T>(v[i >> 1], i & 1), s);
#pragma unroll
      for (int o = 1; o < LANES; o <<= 1) s += __shfl_xor(s, o);
      if (piece == 0 && blk < have) {
        const float x = (float)s;
        a.scores[(int64_t)unit * a.all + blk] = x == x ? x : __builtin_inff();
      }
    }
  }
}

constexpr int kThreads = 1024;
__global__ __launch_bounds__(kThreads) void block_list_kernel(const SelectArgs a) {
  __shared__ uint32_t lds[258];
  __shared__ int lds_sums[2 * kThreads / 64];
  const int unit = blockIdx.x, b = unit / a.Hkv;
  const int n = min(max(a.count[b], 0), a.k_cap), have = (n + (1 << a.shift) - 1) >> a.shift;
  int32_t* const out = a.blocks + (int64_t)unit * a.most;
  if (have <= a.most) {
    for (int i = threadIdx.x; i < a.most; i += kThreads) out[i] = i < have ? i : -1;
    return;
  }
  const float* const score = a.scores + (int64_t)unit * a.all;
  auto key_at = [&](int k) { return k < a.first || k >= have - a.recent ? 0xFFFFFFFFu : key_of_float(score[k]); };
  const Cutoff cut = cutoff_of<kThreads>(have, a.most, key_at, lds);
  int equal = 0, taken = 0;
  for (int k0 = 0; k0 < have; k0 += kThreads) {
    const int k = k0 + threadIdx.x;
    const uint32_t key = k < have ? key_at(k) : 0;
    const bool is = k < have && key == cut.key, over = k < have && key > cut.key;
    Two sums;
    const Two at = count_before<kThreads>(is, over, sums, lds_sums);
    // (equal ones are taken while there is room for them)
    const int mine = min(equal + at.a, cut.equal) + taken + at.b;
    if (over || (is && equal + at.a < cut.equal)) out[mine] = k;
    equal += sums.a;
    taken += sums.b;
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
  if ((int64_t)d.B * d.Hkv > 1 << 22) return PKV_ERR_UNSUPPORTED;
  if (queries && (d.Hq / d.Hkv > 128 || (int64_t)d.B * d.Hq > kMaxGrid)) return PKV_ERR_UNSUPPORTED;
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

// Workgroups of `per` blocks each that all blocks of a head can need, as many as a launch holds for all heads.
int chunks_of(int64_t blocks, int per, int64_t units) {
  const int64_t chunks = (blocks + per - 1) / per, most = kMaxGrid / units;
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
      !aligned(new_lens, 4) || (d.page_size > 0 && !block_table))
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
  const int chunks = chunks_of(blocks_of(d), 4, units);
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
  const int64_t units = (int64_t)d.B * d.Hkv;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int chunks = chunks_of(a.all, kScoreBlocks, units);
  const dim3 grid((unsigned)(units * chunks)), block(256);
  if (d.dtype == PKV_BF16) {
    if (d.d == 128) hipLaunchKernelGGL((block_score_kernel<__bf16, 128>), grid, block, 0, st, a, chunks);
    else hipLaunchKernelGGL((block_score_kernel<__bf16, 64>), grid, block, 0, st, a, chunks);
  } else {
    if (d.d == 128) hipLaunchKernelGGL((block_score_kernel<_Float16, 128>), grid, block, 0, st, a, chunks);
    else hipLaunchKernelGGL((block_score_kernel<_Float16, 64>), grid, block, 0, st, a, chunks);
  }
  if (hipGetLastError() != hipSuccess) return PKV_ERR_HIP;
  hipLaunchKernelGGL(block_list_kernel, dim3((unsigned)units), dim3(kThreads), 0, st, a);
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
