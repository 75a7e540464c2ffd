// Attention of drafted tokens over a cache (include/pkv.h: pkv_tree_attention).
//
// The T Hq/Hkv query rows of a KV head share its rows of the cache; up to 64 of them are a workgroup of pkv_decode_long.hip's
// kernel, in which only the tiles that hold drafted tokens look at the tree: 32 of its bits are one word, shifted to the tile.
#include "pkv_long.h"

namespace pkv {
namespace {

int check_tree_desc(const pkv_tree_desc* desc) {
  if (!desc) return PKV_ERR_INVALID_ARG;
  const pkv_tree_desc& d = *desc;
  if (check_scores(d) != PKV_OK || check_pages(d) != PKV_OK || d.T < 1 || d.window < 0 || d.reserved != 0 || d.p_sb < 0 || d.p_sh < 0)
    return PKV_ERR_INVALID_ARG;
  if (!good_strides(0, 0, d.q_st) || !good_strides(d.o_sb, d.o_sh, d.o_st)) return PKV_ERR_INVALID_ARG;
  if (d.d != 64 && d.d != 128) return PKV_ERR_UNSUPPORTED;
  if (check_factors(d) != PKV_OK) return PKV_ERR_INVALID_ARG;
  if (d.T > kMostDrafted || d.Hq / d.Hkv > 128 || d.Hq > kMaxGrid || (int64_t)d.B * d.Hq * d.T > kMaxGrid) return PKV_ERR_UNSUPPORTED;
  return check_cache_limits(d);
}

Grid grid_of(const pkv_tree_desc& d) { return grid_of(d.B, d.Hkv, (int64_t)d.T * (d.Hq / d.Hkv), d.k_cap); }

}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

int pkv_tree_bits(int32_t T, const int32_t* parents, int32_t* bits_out) {
  if (T < 1 || T > kMostDrafted || !parents || !bits_out) return PKV_ERR_INVALID_ARG;
  for (int t = 0; t < T; ++t)
    if (parents[t] < -1 || parents[t] >= t) return PKV_ERR_INVALID_ARG;
  const int words = (T + 31) / 32;
  for (int t = 0; t < T; ++t) {
    int32_t* const row = bits_out + (size_t)t * words;
    if (parents[t] >= 0)
      memcpy(row, bits_out + (size_t)parents[t] * words, words * sizeof(int32_t));
    else
      memset(row, 0, words * sizeof(int32_t));
    row[t >> 5] = (int32_t)((uint32_t)row[t >> 5] | 1u << (t & 31));
  }
  return PKV_OK;
}

size_t pkv_tree_workspace_bytes(const pkv_tree_desc* desc) {
  if (check_tree_desc(desc) != PKV_OK) return 0;
  return parts_bytes(grid_of(*desc), desc->T * (desc->Hq / desc->Hkv), desc->d);
}

int pkv_tree_attention(const pkv_tree_desc* desc, const void* q, const void* K_cache, const void* V_cache, const int32_t* block_table,
                       const int32_t* count, const int32_t* new_lens, const int32_t* tree, const int32_t* positions,
                       const int32_t* q_pos, const float* slopes, void* out, float* lse_out, void* workspace, size_t workspace_bytes,
                       void* stream) {
  if (!desc || !q || !K_cache || !V_cache || !count || !out) return PKV_ERR_INVALID_ARG;
  const int rc = check_tree_desc(desc);
  if (rc != PKV_OK) return rc;
  const pkv_tree_desc& d = *desc;
  if (!aligned(q, 16) || !aligned(K_cache, 16) || !aligned(V_cache, 16) || !aligned(out, 16) || !aligned(block_table, 4) ||
      !aligned(count, 4) || !aligned(new_lens, 4) || !aligned(tree, 4) || !aligned(positions, 4) || !aligned(q_pos, 4) ||
      !aligned(slopes, 4) || !aligned(lse_out, 4))
    return PKV_ERR_INVALID_ARG;
  if ((d.page_size > 0 && !block_table) || !positions != !q_pos) return PKV_ERR_INVALID_ARG;
  const size_t need = pkv_tree_workspace_bytes(desc);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return PKV_ERR_WORKSPACE;
  TreeArgs a;
  memset(&a, 0, sizeof(a));
  const Grid grid = grid_of(d);
  fill_long(a, d, grid, d.T * (d.Hq / d.Hkv), q, K_cache, V_cache, out, workspace);
  a.table = block_table; a.count = count; a.positions = positions; a.q_pos = q_pos; a.slopes = slopes;
  a.new_lens = new_lens; a.tree = tree;
  a.lse = lse_out;
  a.window = d.window;
  a.p_sb = d.p_sb; a.p_sh = d.p_sh;
  a.T = d.T; a.words = (d.T + 31) / 32; a.heads = d.Hq / d.Hkv;
  a.q_st = d.q_st; a.o_sb = d.o_sb; a.o_sh = d.o_sh; a.o_st = d.o_st;
  const hipError_t e = launch_long(a, d.dtype, d.d, grid.workgroups, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
