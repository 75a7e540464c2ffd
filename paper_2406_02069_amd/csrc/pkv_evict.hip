// Eviction by accumulated weights, in place (include/pkv.h: pkv_cache_evict).
//
// Two launches.  The first, a workgroup per (sequence, KV head), finds the smallest weight that stays and pairs the rows behind the
// budget that stay with the holes before it: sources lie behind all destinations, so that the second can copy the pairs' rows in any
// order, in place.
#include <string.h>

#include "pkv_attn.h"
#include "pkv_long.h"
#include "pkv_topk.h"

namespace pkv {
namespace {

constexpr int kThreads = 1024;
constexpr int kPairs = 32;  // of a workgroup of the second launch

struct EvictArgs {
  char *K, *V;
  const int32_t *table, *count, *positions;
  const float* weights;
  int32_t* positions_out;
  float* weights_out;
  int32_t* count_out;
  int32_t* moves;  // [unit]
  int32_t* pairs;  // [unit][2][most]: destinations, sources
  int32_t B, Hkv, d, k_cap, page_size, num_pages, max_pages, budget, recent, first, most;
  uint32_t page_magic;
  int64_t c_sb, c_sh, c_st, p_sb, p_sh, w_sb, w_sh, po_sb, po_sh, wo_sb, wo_sh;
};

// Where row j of a sequence and head lies, in bytes; -1: on a page that does not exist.
__device__ __forceinline__ int64_t row_at(const EvictArgs& a, int b, int g, int j) {
  if (a.page_size == 0) return (b * a.c_sb + g * a.c_sh + j * a.c_st) * 2;
  uint32_t p = __umulhi((uint32_t)j, a.page_magic);
  if ((uint32_t)j - p * a.page_size >= (uint32_t)a.page_size) ++p;
  const int32_t page = a.table[(int64_t)b * a.max_pages + p];
  if ((uint32_t)page >= (uint32_t)a.num_pages) return -1;
  return (((int64_t)page * a.Hkv + g) * a.page_size + (j - p * a.page_size)) * a.d * 2;
}

__global__ __launch_bounds__(kThreads) void evict_select_kernel(const EvictArgs a) {
  __shared__ uint32_t lds[258];
  __shared__ int lds_sums[2 * kThreads / 64], lds_newest[kThreads / 64];
  const int unit = blockIdx.x, b = unit / a.Hkv, g = unit % a.Hkv;
  const int n = min(max(a.count[b], 0), a.k_cap), kept = min(n, a.budget);
  const int32_t* const pos = a.positions + b * a.p_sb + g * a.p_sh;
  const float* const weight = a.weights + b * a.w_sb + g * a.w_sh;
  int32_t* const pos_out = a.positions_out + b * a.po_sb + g * a.po_sh;
  float* const weight_out = a.weights_out + b * a.wo_sb + g * a.wo_sh;
  if (g == 0 && threadIdx.x == 0 && a.count_out) a.count_out[b] = kept;
  if (n <= a.budget) {
    for (int r = threadIdx.x; r < n; r += kThreads) {
      pos_out[r] = pos[r];
      weight_out[r] = weight[r];
    }
    if (threadIdx.x == 0) a.moves[unit] = 0;
    return;
  }
  int newest = -1;
  for (int r = threadIdx.x; r < n; r += kThreads) newest = max(newest, pos[r]);
  newest = wave_max(newest);
  if ((threadIdx.x & 63) == 0) lds_newest[threadIdx.x >> 6] = newest;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) newest = max(newest, lds_newest[w]);
  auto key_at = [&](int r) {
    const int32_t p = pos[r];
    if (p < 0) return 0u;
    if (p < a.first || p > newest - a.recent) return 0xFFFFFFFFu;
    const float w = weight[r];
    return w == w ? key_of_float(w) : 1u;
  };
  const Cutoff cut = cutoff_of<kThreads>(n, a.budget, key_at, lds);

  int32_t *const to = a.pairs + (int64_t)unit * 2 * a.most, *const from = to + a.most;
  int equal = 0, holes = 0, late = 0;
  for (int r0 = 0; r0 < n; r0 += kThreads) {
    const int r = r0 + threadIdx.x;
    const uint32_t key = r < n ? key_at(r) : 0;
    Two sums;
    const Two eq = count_before<kThreads>(r < n && key == cut.key, false, sums, lds_sums);
    const bool stays = r < n && (key > cut.key || (key == cut.key && equal + eq.a < cut.equal));
    equal += sums.a;
    const bool hole = r < a.budget && !stays, moves = r >= a.budget && stays;
    const Two at = count_before<kThreads>(hole, moves, sums, lds_sums);
    if (hole) to[holes + at.a] = r;
    if (moves) from[late + at.b] = r;
    holes += sums.a;
    late += sums.b;
    if (r < a.budget && stays) {
      const int32_t p = pos[r];
      const float w = weight[r];
      pos_out[r] = p;
      weight_out[r] = w;
    }
  }
  __threadfence_block();
  __syncthreads();  // (holes == late)
  for (int i = threadIdx.x; i < late; i += kThreads) {
    const bool there = row_at(a, b, g, to[i]) >= 0 && row_at(a, b, g, from[i]) >= 0;
    pos_out[to[i]] = there ? pos[from[i]] : -1;
    weight_out[to[i]] = weight[from[i]];
  }
  __syncthreads();
  for (int r = a.budget + threadIdx.x; r < n; r += kThreads) {
    pos_out[r] = -1;
    weight_out[r] = 0.0f;
  }
  if (threadIdx.x == 0) a.moves[unit] = late;
}

// A workgroup: kPairs rows of K and of V, 16 bytes a thread at a time.
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs a, int chunks) {
  const int unit = blockIdx.x / chunks, chunk = blockIdx.x % chunks, b = unit / a.Hkv, g = unit % a.Hkv;
  const int moves = a.moves[unit], lanes = a.d / 8;
  const int32_t *const to = a.pairs + (int64_t)unit * 2 * a.most, *const from = to + a.most;
  for (int64_t c = chunk; c * kPairs < moves; c += chunks) {
    for (int i = threadIdx.x; i < kPairs * lanes; i += 256) {
      const int p = (int)(c * kPairs) + i / lanes;
      if (p >= moves) break;
      const int64_t dst = row_at(a, b, g, to[p]), src = row_at(a, b, g, from[p]);
      if (dst < 0 || src < 0) continue;
      const int piece = 16 * (i % lanes);
      const u32x4 k = *reinterpret_cast<const u32x4*>(a.K + src + piece), v = *reinterpret_cast<const u32x4*>(a.V + src + piece);
      *reinterpret_cast<u32x4*>(a.K + dst + piece) = k;
      *reinterpret_cast<u32x4*>(a.V + dst + piece) = v;
    }
  }
}

int check_evict_desc(const pkv_evict_desc* desc) {
  if (!desc) return PKV_ERR_INVALID_ARG;
  const pkv_evict_desc& d = *desc;
  if (d.B < 1 || d.Hkv < 1 || d.budget < 1 || d.recent < 0 || d.first < 0 || (int64_t)d.first + d.recent > d.budget ||
      check_pages(d) != PKV_OK)
    return PKV_ERR_INVALID_ARG;
  if (d.p_sb < 0 || d.p_sh < 0 || d.w_sb < 0 || d.w_sh < 0 || d.po_sb < 0 || d.po_sh < 0 || d.wo_sb < 0 || d.wo_sh < 0) return PKV_ERR_INVALID_ARG;
  if ((int64_t)d.B * d.Hkv > 1 << 22) return PKV_ERR_UNSUPPORTED;
  return check_cache_limits(d);
}

// Pairs that a head can have.
int64_t most_moves(const pkv_evict_desc& d) {
  const int64_t behind = (int64_t)d.k_cap - d.budget;
  return behind < 0 ? 0 : behind < d.budget ? behind : d.budget;
}

}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

size_t pkv_evict_workspace_bytes(const pkv_evict_desc* desc) {
  if (check_evict_desc(desc) != PKV_OK) return 0;
  return (size_t)desc->B * desc->Hkv * (1 + 2 * (size_t)most_moves(*desc)) * sizeof(int32_t);
}

int pkv_cache_evict(const pkv_evict_desc* desc, void* K_cache, void* V_cache, const int32_t* block_table, const int32_t* count,
                    const int32_t* positions, const float* weights, int32_t* positions_out, float* weights_out, int32_t* count_out,
                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc || !K_cache || !V_cache || !count || !positions || !weights || !positions_out || !weights_out) return PKV_ERR_INVALID_ARG;
  const int rc = check_evict_desc(desc);
  if (rc != PKV_OK) return rc;
  const pkv_evict_desc& d = *desc;
  if (!aligned(K_cache, 16) || !aligned(V_cache, 16) || !aligned(block_table, 4) || !aligned(count, 4) || !aligned(positions, 4) ||
      !aligned(weights, 4) || !aligned(positions_out, 4) || !aligned(weights_out, 4) || !aligned(count_out, 4))
    return PKV_ERR_INVALID_ARG;
  if (d.page_size > 0 && !block_table) return PKV_ERR_INVALID_ARG;
  if (positions_out == positions && (d.po_sb != d.p_sb || d.po_sh != d.p_sh)) return PKV_ERR_INVALID_ARG;
  if (weights_out == weights && (d.wo_sb != d.w_sb || d.wo_sh != d.w_sh)) return PKV_ERR_INVALID_ARG;
  if (count_out == count) return PKV_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < pkv_evict_workspace_bytes(desc)) return PKV_ERR_WORKSPACE;
  EvictArgs a;
  memset(&a, 0, sizeof(a));
  const int units = d.B * d.Hkv;
  a.K = static_cast<char*>(K_cache);
  a.V = static_cast<char*>(V_cache);
  a.table = block_table; a.count = count; a.positions = positions; a.weights = weights;
  a.positions_out = positions_out; a.weights_out = weights_out; a.count_out = count_out;
  a.moves = static_cast<int32_t*>(workspace);
  a.pairs = a.moves + units;
  a.B = d.B; a.Hkv = d.Hkv; a.d = d.d; a.k_cap = d.k_cap; a.page_size = d.page_size; a.num_pages = d.num_pages;
  a.max_pages = d.max_pages; a.budget = d.budget; a.recent = d.recent; a.first = d.first;
  a.most = (int32_t)most_moves(d);
  a.page_magic = magic_of(d.page_size);
  a.c_sb = d.c_sb; a.c_sh = d.c_sh; a.c_st = d.c_st; a.p_sb = d.p_sb; a.p_sh = d.p_sh; a.w_sb = d.w_sb; a.w_sh = d.w_sh;
  a.po_sb = d.po_sb; a.po_sh = d.po_sh; a.wo_sb = d.wo_sb; a.wo_sh = d.wo_sh;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)units), dim3(kThreads), 0, st, a);
  if (hipGetLastError() != hipSuccess) return PKV_ERR_HIP;
  if (a.most == 0) return PKV_OK;
  int64_t chunks = (a.most + kPairs - 1) / kPairs;
  if (chunks > kMaxGrid / units) chunks = kMaxGrid / units;
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(units * chunks)), dim3(256), 0, st, a, (int)chunks);
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
