// Attention of one new token per sequence over a cache of any length (include/pkv.h: pkv_decode_attention_long).
//
// HBM-bound: every seen row of K and V is read once (2 d bytes each), for all query heads of its KV head.  128k rows of 8 heads in
// 16-slot pages, d 128: 99 us with the join, 95 of them here (5.65 TB/s; a plain read of as much 6.3); four ragged sequences of up
// to 100k rows: 183 (5.6); 16 of up to 5000 kept rows with positions and biases: 25; 4k rows 12.3; 1000 rows, d 64: 6 and 4.
// Work split: (sequence, KV head, up to 64 of its query heads) x ranges of keys, a workgroup of four waves each; a wave takes
// 16 query heads, so that with up to 16, 32 and 64 heads four, two and one of the waves share the range's 32-key tiles.  Every
// wave works on its own, K tile -> scores -> running softmax -> V tile, the rows of its next tile requested as soon as this
// tile's are used up, and the waves meet once at the end.  Where a sequence has several ranges, they leave un-normalised results
// in a workspace, and a second kernel joins them in order.
// Ranges: as long as fill the device once (512 workgroups), by the sequences' lengths as they are on the device, so that ragged
// batches have ranges of one length too; every wave works out its place among them from all counts (2 to 256 sequences).
//   loads   whole rows, 1 KB at a time, into registers; from there to the wave's own tile in LDS, K first, then V in its place.
//   scores  S^T = K Q^T in v_mfma_f32_16x16x32: 16 keys are the rows of A, 16 heads the columns of B.  Lane (l16, quad) ends with
//           keys 4 quad .. + 3 of head l16, all it needs for its weights.
//   softmax a reference exponent per head and wave, moved only when a score exceeds it by a factor of 2^8 (fp16: 2^2).
//   values  O^T += V^T P^T: the weights are in B's layout already if the 32 keys of a step are taken in the order in which the
//           lanes hold them (4 quad .. + 3 of either half), and V^T is read column-wise.  The weights are given as two numbers of
//           the type, their rounding and what it left (16 bits for bf16; 22 for fp16, down to steps of 2^-37 of the reference):
//           the matrix pipe has time for both products.
// Rows that are not seen (behind the count, outside the window, on a page that does not exist) have weight 0, and their copy of
// V is zero.
#include "pkv_long.h"

namespace pkv {
namespace {

Grid grid_of(const pkv_decode_long_desc& d) { return grid_of(d.B, d.Hkv, d.Hq / d.Hkv, d.k_cap); }

}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

size_t pkv_decode_long_workspace_bytes(const pkv_decode_long_desc* desc) {
  if (check_long_desc(desc) != PKV_OK) return 0;
  return parts_bytes(grid_of(*desc), desc->Hq / desc->Hkv, desc->d);
}

int pkv_decode_attention_long(const pkv_decode_long_desc* desc, const void* q, const void* K_cache, const void* V_cache,
                              const int32_t* block_table, const int32_t* count, const int32_t* positions, const int32_t* q_pos,
                              const float* slopes, void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_long_call(desc, q, K_cache, V_cache, block_table, count, positions, q_pos, slopes, out, lse_out);
  if (rc != PKV_OK) return rc;
  const pkv_decode_long_desc& d = *desc;
  const size_t need = pkv_decode_long_workspace_bytes(desc);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return PKV_ERR_WORKSPACE;
  LongArgs a;
  memset(&a, 0, sizeof(a));
  const Grid grid = grid_of(d);
  fill_long(a, d, grid, d.Hq / d.Hkv, q, K_cache, V_cache, out, workspace);
  a.table = block_table; a.count = count; a.positions = positions; a.q_pos = q_pos; a.slopes = slopes;
  a.lse = lse_out;
  a.window = d.window;
  a.p_sb = d.p_sb; a.p_sh = d.p_sh;
  const hipError_t e = launch_long(a, d.dtype, d.d, grid.workgroups, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
