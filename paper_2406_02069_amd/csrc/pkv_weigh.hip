// Attention of one new token that adds each row's softmax weight to a running sum (include/pkv.h: pkv_decode_attention_accumulate).
//
//   weights_j += sum_h 2^(s_hj - m_h) / z_h   with m_h, z_h of all ranges: z_h = sum_r 2^(m_hr - m_h) z_hr.
// HBM-bound like the attention itself (pkv_decode_long.hip), whose kernel leaves the scores behind, 4 bytes a row and query head
// beside the 4 d bytes of the row: a softmax weight is known only once all of the head's scores are.  (To read K again instead would be
// 2 d bytes a row, 16 times the score of each of 4 heads at d 128.)  A second kernel joins the ranges' outputs with some of its
// workgroups and forms the weights with the others, which work out each head's reference and sum from the ranges' own: as a launch
// behind the join the weights of 2k rows took 18.5 us, now 15.7.
// 100k and 25k rows of 8 heads with 4 query heads each, d 128: 107 us + 12 (the attention alone 98 in all; 16 MB of scores are written
// and read); 32 sequences of 1500 to 6000 rows of 4 heads, d 64, in pages: 24 + 9.  Many heads on one KV head are bound by the scores: 64 on
// one, d 64, 100k rows 66 us, the attention alone 22 (26 MB of scores written and read beside 26 MB of rows).
#include "pkv_long.h"

namespace pkv {
namespace {

constexpr int kRowsAtATime = 4;  // of a thread
constexpr int kChunk = 256 * kRowsAtATime;
constexpr int kMostHeads = 128;  // of a KV head

// Each head's reference and the factor that makes softmax weights of the 2^(score - reference), from its ranges' references and sums
// (a wave: every fourth head, a lane: every 64th range), or as the attention's kernel has left them.
template <typename T>
__device__ __forceinline__ void heads_of_unit(const WeighArgs& a, int b, int g, float (&mz)[kMostHeads][2]) {
  const int lane = threadIdx.x & 63;
  int ranges = a.ranges, base = b * a.units * a.ranges;
  if (a.by_length) {
    const Place p = a.B <= 64 ? place_of_sequence<1>(a, b, lane) : place_of_sequence<kLaneSequences>(a, b, lane);
    ranges = p.ranges;
    base = p.base;
  }
  const int64_t heads = 16 * a.wave_groups;
  for (int h = this_wave(); h < a.G; h += 4) {
    float m = kNone, z = 0.0f;
    if (ranges > 1) {
      const float* const part = a.part_mz + (((int64_t)base + (g * a.head_groups + h / 64) * ranges) * heads + h % 64) * 2;
      for (int i = lane; i < ranges; i += 64) {
        const float m1 = part[heads * i * 2], z1 = part[heads * i * 2 + 1], top = fmaxf(m, m1), ref = top == kNone ? 0.0f : top;
        z = z * exp2_(m - ref) + z1 * exp2_(m1 - ref);
        m = top;
      }
      float top = m;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
      const float ref = top == kNone ? 0.0f : top;
      z *= exp2_(m - ref);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o);
      m = ref;
      z = z == 0.0f ? 0.0f : (1.0f / Weight<T>::UNIT) / z;
    } else {
      const float* const own = a.mz + ((int64_t)b * a.Hq + g * a.G + h) * 2;
      m = own[0];
      z = own[1];
    }
    if (lane == 0) {
      mz[h][0] = m;
      mz[h][1] = z;
    }
  }
}

// The first `joins` workgroups join ranges, HEADS heads each; the others add weights, kChunk rows of a KV head at a time.
template <typename T, int D, int HEADS>
__global__ __launch_bounds__(256) void join_and_weigh_kernel(const WeighArgs a, int joins, Items items) {
  if ((int)blockIdx.x < joins) {
    join_heads<T, D, HEADS>(a);
    return;
  }
  __shared__ float lds_mz[kMostHeads][2];
  struct Rows {
    int lo, hi;  // visited
  };
  auto rows_of = [&](int b) {
    const Tiles tl = tiles_of(a, b);
    return Rows{tl.first * kTile, min(tl.n, (tl.first + tl.count) * kTile)};
  };
  auto has = [&](int unit, int chunk) {
    const Rows rows = rows_of(unit / a.Hkv);
    return chunk * kChunk < rows.hi && (chunk + 1) * kChunk > rows.lo;
  };
  each_item(items, blockIdx.x - joins, gridDim.x - joins, has, [&](int unit, int chunk) {
    const int b = unit / a.Hkv, g = unit % a.Hkv;
    const Rows rows = rows_of(b);
    const int lo = rows.lo, hi = rows.hi, r0 = chunk * kChunk + threadIdx.x;
    if (chunk * kChunk >= hi || (chunk + 1) * kChunk <= lo) return;
    __syncthreads();  // (the last item's have been read)
    heads_of_unit<T>(a, b, g, lds_mz);
    __syncthreads();
    float sum[kRowsAtATime];
    bool saw[kRowsAtATime];  // (rows that no head sees are not written, not even with what they hold)
#pragma unroll
    for (int i = 0; i < kRowsAtATime; ++i) {
      sum[i] = 0.0f;
      saw[i] = false;
    }
    const float* const s = a.scores + (int64_t)unit * a.G * a.score_row;
#pragma unroll 2
    for (int h = 0; h < a.G; ++h) {
      const float ref = lds_mz[h][0], factor = lds_mz[h][1];
      float x[kRowsAtATime];
#pragma unroll
      for (int i = 0; i < kRowsAtATime; ++i) x[i] = s[h * a.score_row + min(max(r0 + 256 * i, lo), hi - 1)];
#pragma unroll
      for (int i = 0; i < kRowsAtATime; ++i) {
        const bool sees = x[i] != kNone && factor != 0.0f;
        sum[i] += sees ? exp2_(x[i] - ref) * factor : 0.0f;
        saw[i] = saw[i] || sees;
      }
    }
    float* const w = a.weights + b * a.w_sb + g * a.w_sh;
#pragma unroll
    for (int i = 0; i < kRowsAtATime; ++i) {
      const int r = r0 + 256 * i;
      if (r >= lo && r < hi && saw[i]) w[r] += sum[i];
    }
  });
}

template <typename T, int D>
hipError_t launch_weigh(const WeighArgs& a, int64_t workgroups, const Items& items, hipStream_t s) {
  const hipError_t e = launch_long<T, D>(a, workgroups, s);
  if (e != hipSuccess) return e;
  const bool four = a.Hq % 4 == 0 && a.B * a.Hq >= 4 * kWorkgroups;  // (as launch_join)
  const int64_t joins = a.ranges == 0 ? 0 : (int64_t)a.B * a.Hq / (four ? 4 : 1);
  const dim3 grid((unsigned)(joins + workgroups_of(items)));
  if (four)
    hipLaunchKernelGGL((join_and_weigh_kernel<T, D, 4>), grid, dim3(256), 0, s, a, (int)joins, items);
  else
    hipLaunchKernelGGL((join_and_weigh_kernel<T, D, 1>), grid, dim3(256), 0, s, a, (int)joins, items);
  return hipGetLastError();
}

int64_t chunks_of(const pkv_decode_long_desc& d) { return ((int64_t)d.k_cap + kChunk - 1) / kChunk; }

// (joins and weights share a launch; its items are counted in 32 bits)
int check_accumulate_desc(const pkv_decode_long_desc* desc) {
  const int rc = check_long_desc(desc);
  if (rc != PKV_OK) return rc;
  return (int64_t)desc->B * desc->Hq > 1 << 23 || (int64_t)desc->B * desc->Hkv * chunks_of(*desc) > kMostItems ? PKV_ERR_UNSUPPORTED : PKV_OK;
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
  return check_accumulate_desc(desc) == PKV_OK ? plan_of(*desc).all : 0;
}

int pkv_decode_attention_accumulate(const pkv_decode_long_desc* desc, const void* q, const void* K_cache, const void* V_cache,
                                    const int32_t* block_table, const int32_t* count, const int32_t* positions, const int32_t* q_pos,
                                    const float* slopes, float* weights, int64_t w_sb, int64_t w_sh, void* out, float* lse_out,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!weights || !aligned(weights, 4) || w_sb < 0 || w_sh < 0) return PKV_ERR_INVALID_ARG;
  const int rc = check_long_call(desc, q, K_cache, V_cache, block_table, count, positions, q_pos, slopes, out, lse_out);
  if (rc != PKV_OK) return rc;
  if (check_accumulate_desc(desc) != PKV_OK) return PKV_ERR_UNSUPPORTED;
  const pkv_decode_long_desc& d = *desc;
  if (!apart(d.k_cap, {{d.B, w_sb}, {d.Hkv, w_sh}})) return PKV_ERR_INVALID_ARG;
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
  const Items items = items_of((int64_t)d.B * d.Hkv, chunks_of(d));
  hipError_t e;
  if (d.dtype == PKV_BF16)
    e = d.d == 128 ? launch_weigh<__bf16, 128>(a, p.grid.workgroups, items, st) : launch_weigh<__bf16, 64>(a, p.grid.workgroups, items, st);
  else
    e = d.d == 128 ? launch_weigh<_Float16, 128>(a, p.grid.workgroups, items, st) : launch_weigh<_Float16, 64>(a, p.grid.workgroups, items, st);
  return e == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
