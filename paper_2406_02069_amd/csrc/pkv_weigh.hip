// Attention of one new token that adds each row's softmax weight to a running sum (include/pkv.h: pkv_decode_attention_accumulate).
//
// HBM-bound like the attention itself (pkv_decode_long.hip), whose kernel leaves the scores behind, 4 bytes a row and query head
// beside the 4 d bytes of the row: a softmax weight is known only once all of the head's scores are.  A last kernel forms the
// weights from them with each head's reference and sum, and adds up those of a KV head's query heads, in order.
#include "pkv_long.h"

namespace pkv {
namespace {

constexpr int kRowsAtATime = 4;  // of a thread
constexpr int kChunk = 256 * kRowsAtATime;

__global__ __launch_bounds__(256) void add_weights_kernel(const WeighArgs a, int chunks, int64_t items) {
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int unit = (int)(item / chunks), chunk = (int)(item % chunks), b = unit / a.Hkv, g = unit % a.Hkv;
    const Tiles tl = tiles_of(a, b);
    const int lo = tl.first * kTile, hi = min(tl.n, (tl.first + tl.count) * kTile), r0 = chunk * kChunk + threadIdx.x;
    if (chunk * kChunk >= hi || (chunk + 1) * kChunk <= lo) continue;
    float sum[kRowsAtATime];
#pragma unroll
    for (int i = 0; i < kRowsAtATime; ++i) sum[i] = 0.0f;
    for (int h = 0; h < a.G; ++h) {
      const float* const mz = a.mz + ((int64_t)b * a.Hq + g * a.G + h) * 2;
      const float* const s = a.scores + ((int64_t)unit * a.G + h) * a.score_row;
      const float ref = mz[0], factor = mz[1];
#pragma unroll
      for (int i = 0; i < kRowsAtATime; ++i) {
        const int r = r0 + 256 * i;
        const float x = r >= lo && r < hi ? s[r] : kNone;
        sum[i] += x == kNone ? 0.0f : exp2_(x - ref) * factor;
      }
    }
    float* const w = a.weights + b * a.w_sb + g * a.w_sh;
#pragma unroll
    for (int i = 0; i < kRowsAtATime; ++i) {
      const int r = r0 + 256 * i;
      if (r >= lo && r < hi) w[r] += sum[i];
    }
  }
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Where the parts of the workspace begin.
struct WeighPlan {
  Grid grid;
  int64_t score_row;
  size_t mz, scores, all;
};
WeighPlan plan_of(const pkv_decode_long_desc& d) {
  WeighPlan p;
  p.grid = grid_of(d.B, d.Hkv, d.Hq / d.Hkv, d.k_cap);
  p.score_row = ((int64_t)d.k_cap + kTile - 1) / kTile * kTile;
  p.mz = up256(parts_bytes(p.grid, d.Hq / d.Hkv, d.d));
  p.scores = p.mz + up256((size_t)d.B * d.Hq * 2 * sizeof(float));
  p.all = p.scores + (size_t)d.B * d.Hq * p.score_row * sizeof(float);
  return p;
}

}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

size_t pkv_decode_accumulate_workspace_bytes(const pkv_decode_long_desc* desc) {
  return check_long_desc(desc) == PKV_OK ? plan_of(*desc).all : 0;
}

int pkv_decode_attention_accumulate(const pkv_decode_long_desc* desc, const void* q, const void* K_cache, const void* V_cache,
                                    const int32_t* block_table, const int32_t* count, const int32_t* positions, const int32_t* q_pos,
                                    const float* slopes, float* weights, int64_t w_sb, int64_t w_sh, void* out, float* lse_out,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!weights || !aligned(weights, 4) || w_sb < 0 || w_sh < 0) return PKV_ERR_INVALID_ARG;
  const int rc = check_long_call(desc, q, K_cache, V_cache, block_table, count, positions, q_pos, slopes, out, lse_out);
  if (rc != PKV_OK) return rc;
  const pkv_decode_long_desc& d = *desc;
  const WeighPlan p = plan_of(d);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < p.all) return PKV_ERR_WORKSPACE;
  WeighArgs a;
  memset(&a, 0, sizeof(a));
  fill_long(a, d, p.grid, d.Hq / d.Hkv, q, K_cache, V_cache, out, workspace);
  a.table = block_table; a.count = count; a.positions = positions; a.q_pos = q_pos; a.slopes = slopes;
  a.lse = lse_out;
  a.window = d.window;
  a.p_sb = d.p_sb; a.p_sh = d.p_sh;
  a.mz = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.mz);
  a.scores = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.scores);
  a.score_row = p.score_row;
  a.weights = weights;
  a.w_sb = w_sb; a.w_sh = w_sh;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (launch_long(a, d.dtype, d.d, p.grid.workgroups, st) != hipSuccess) return PKV_ERR_HIP;
  const int chunks = (int)((p.score_row + kChunk - 1) / kChunk);
  const int64_t items = (int64_t)d.B * d.Hkv * chunks;
  hipLaunchKernelGGL(add_weights_kernel, dim3((unsigned)(items < kMaxGrid ? items : kMaxGrid)), dim3(256), 0, st, a, chunks, items);
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
