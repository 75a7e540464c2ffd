// Attention of one new token per sequence over a cache of any length (include/pkv.h: pkv_decode_attention_long).
//
// HBM-bound: every seen row of K and V is read once (2 d bytes each), for all query heads of its KV head.
// Work split: (sequence, KV head, up to 64 of its query heads) x S ranges of keys, a workgroup of four waves each; a wave takes
// 16 query heads, so that with up to 16, 32 and 64 heads four, two and one of the waves share the range's 32-key tiles.  Every
// wave works on its own, K tile -> scores -> running softmax -> V tile, the rows of its next tile requested as soon as this
// tile's are used up, and the waves meet once at the end.  With S > 1 the ranges leave un-normalised results in a workspace and
// a second kernel joins them in order.
//   scores  S^T = K Q^T in v_mfma_f32_16x16x32: 16 keys are the rows of A, loaded straight into operand layout, 16 heads the
//           columns of B.  Lane (l16, quad) ends with keys 4 quad .. + 3 of head l16, all it needs for its weights.
//   softmax a reference exponent per head and wave, moved only when a score exceeds it by a factor of 2^8.
//   values  O^T += V^T P^T: the weights are in B's layout already if the 32 keys of a step are taken in the order in which the
//           lanes hold them (4 quad .. + 3 of either half), and V^T is read column-wise from the wave's own copy of the tile in
//           LDS.  The weights are given as two numbers of the type, their rounding and what it left (16 bits for bf16, 22 for
//           fp16): the matrix pipe has time for both products.
// Rows that are not seen (behind the count, outside the window, on a page that does not exist) have weight 0, and their copy of
// V is zero.
#include <math.h>
#include <string.h>

#include "pkv_attn.h"

namespace pkv {
namespace {

constexpr int kTile = 32;          // keys per step of a wave
constexpr int kWaves = 4;          // per workgroup
constexpr int kMaxRanges = 512;    // per (sequence, KV head)

struct LongArgs {
  const uint16_t *q, *K, *V;
  const int32_t *table, *count, *positions, *q_pos;
  const float* slopes;
  uint16_t* out;
  float* lse;
  float* part_o;   // [B * Hq][S][d]
  float* part_mz;  // [B * Hq][S][2] reference exponent (log2) and sum
  int32_t B, Hq, Hkv, G, k_cap, page_size, num_pages, max_pages, window, S;
  int32_t head_groups;  // workgroups that share a KV head's rows: ceil(G / 64)
  int32_t wave_groups;  // 16-head groups in a workgroup: 1, 2 or 4
  uint32_t page_magic;  // floor(2^32 / page_size)
  int64_t q_sb, q_sh, c_sb, c_sh, c_st, p_sb, p_sh;
  float scale;          // of the products; with a cap: natural units, without: log2
  float cap2, two_over_cap;  // cap in log2 units (0: none); 2 log2(e) / cap
};

// A row of a tile as its lane knows it: number in the cache (rows of one stride), position, and whether it is seen.
struct Row {
  uint32_t at;
  int32_t pos;
  bool seen;
};

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void decode_long_kernel(const LongArgs a) {
  constexpr int LANES = D / 8, STEPS = D / 32, VLOADS = kTile * LANES / 64, MT = D / 16;
  __shared__ __align__(16) char lds_v[kWaves][kTile * D * 2];
  __shared__ float lds_mz[kWaves][16][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, quad = lane >> 4;
  const int s = blockIdx.x, g = blockIdx.y / a.head_groups, hg = blockIdx.y % a.head_groups, b = blockIdx.z;
  const int wg = wave & (a.wave_groups - 1), share = wave / a.wave_groups, shares = kWaves / a.wave_groups;
  const int h_in = 64 * hg + 16 * wg + l16;  // query head within the group of this KV head
  const bool head = h_in < a.G;
  const int h = g * a.G + (head ? h_in : 0);

  const int n = min(max(a.count[b], 0), a.k_cap);
  const int q_pos = a.q_pos ? a.q_pos[b] : n - 1;
  // Rows that can be seen: all, or with positions of their own numbers those of the window.
  int first = 0, end = n;
  if (!a.positions) {
    end = (int)min((int64_t)n, (int64_t)q_pos + 1);
    if (a.window) first = (int)min((int64_t)n, max((int64_t)0, (int64_t)q_pos - a.window + 1));
  }
  const int tile0 = first / kTile, tiles = end > first ? (end + kTile - 1) / kTile - tile0 : 0;
  const int per = (tiles + a.S - 1) / a.S;
  int t = tile0 + s * per + share;
  const int t_end = min(tile0 + (s + 1) * per, tile0 + tiles);

  u32x4 qf[STEPS];
  {
    const uint16_t* qp = a.q + b * a.q_sb + h * a.q_sh;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) qf[i] = head ? *reinterpret_cast<const u32x4*>(qp + 32 * i + 8 * quad) : (u32x4)(0);
  }
  const float slope = a.slopes ? a.slopes[h] * kLog2e : 0.0f;
  const int64_t row_bytes = (a.page_size ? (int64_t)D : a.c_st) * 2;
  const int64_t base = a.page_size ? 0 : (b * a.c_sb + g * a.c_sh) * 2;
  const char* const Kb = reinterpret_cast<const char*>(a.K) + base + 16 * quad;
  const char* const Vb = reinterpret_cast<const char*>(a.V) + base + 16 * (lane % LANES);
  const int32_t* const table = a.table + (int64_t)b * a.max_pages;
  const int32_t* const pos_b = a.positions + b * a.p_sb + g * a.p_sh;

  // What has to be loaded to know a tile's rows (lane l: row l % 32); rows behind the last one are taken as the last.
  auto look = [&](int tile, int32_t& page, int32_t& pos) {
    const int j = min(tile * kTile + (lane & 31), n - 1);
    page = 0;
    if (a.page_size) {
      uint32_t p = __umulhi((uint32_t)j, a.page_magic);
      if ((uint32_t)j - p * a.page_size >= (uint32_t)a.page_size) ++p;
      page = table[p];
    }
    pos = a.positions ? pos_b[j] : j;
  };
  auto row_of = [&](int tile, int32_t page, int32_t pos) {
    Row r;
    const int j0 = tile * kTile + (lane & 31), j = min(j0, n - 1);
    r.at = (uint32_t)j;
    r.pos = pos;
    r.seen = j0 < n && pos >= 0 && pos <= q_pos && (a.window == 0 || (int64_t)pos > (int64_t)q_pos - a.window);
    if (a.page_size) {
      uint32_t p = __umulhi((uint32_t)j, a.page_magic);
      if ((uint32_t)j - p * a.page_size >= (uint32_t)a.page_size) ++p;
      const bool there = page >= 0 && page < a.num_pages;
      r.seen = r.seen && there;
      r.at = ((uint32_t)(there ? page : 0) * a.Hkv + g) * a.page_size + ((uint32_t)j - p * a.page_size);
    }
    return r;
  };

  u32x4 kf[2][STEPS], vr[VLOADS];
  auto load_k = [&](const Row& r) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const char* p = Kb + (int64_t)(uint32_t)__shfl((int)r.at, 16 * kt + l16) * row_bytes;
#pragma unroll
      for (int i = 0; i < STEPS; ++i) kf[kt][i] = *reinterpret_cast<const u32x4*>(p + 64 * i);
    }
  };
  auto load_v = [&](const Row& r) {
#pragma unroll
    for (int i = 0; i < VLOADS; ++i)
      vr[i] = *reinterpret_cast<const u32x4*>(Vb + (int64_t)(uint32_t)__shfl((int)r.at, i * (64 / LANES) + lane / LANES) * row_bytes);
  };
  // 16-byte piece c of a row of the copy lies at c ^ swizzle(row): 16 rows' pieces of one column block go to all banks.
  auto swizzle = [](int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); };
  char* const copy = lds_v[wave];

  float m = kNone, z = 0.0f;
  f32x4 o[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) o[i] = (f32x4)(0.0f);

  if (t < t_end) {
    int32_t page, pos, page1, pos1;
    look(t, page, pos);
    Row row = row_of(t, page, pos);
    load_k(row);
    load_v(row);
    look(min(t + shares, t_end - 1), page1, pos1);
    for (; t < t_end; t += shares) {
      const bool more = t + shares < t_end;
      const uint32_t seen = (uint32_t)__ballot(row.seen);
      f32x4 sc[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        sc[kt] = (f32x4)(0.0f);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) sc[kt] = Elem<T>::mfma16(kf[kt][i], qf[i], sc[kt]);
      }
      Row next = row;
      if (more) {
        next = row_of(t + shares, page1, pos1);
        load_k(next);
        look(min(t + 2 * shares, t_end - 1), page1, pos1);
      }
      // scores in units of log2
      if (a.cap2 != 0.0f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e >> 2][e & 3] = capped(sc[e >> 2][e & 3] * a.scale, a.two_over_cap, a.cap2);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e >> 2][e & 3] *= a.scale;
      }
      if (a.slopes) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int kp = __shfl(row.pos, 16 * (e >> 2) + 4 * quad + (e & 3));
          sc[e >> 2][e & 3] -= slope * (float)(int)((uint32_t)q_pos - (uint32_t)kp);
        }
      }
      if (seen != 0xFFFFFFFFu) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!((seen >> (16 * (e >> 2) + 4 * quad + (e & 3))) & 1)) sc[e >> 2][e & 3] = kNone;
      }
      float top = sc[0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, sc[e >> 2][e & 3]);
      if (__any(top > m + 8.0f)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m1 = fmaxf(m, top);
        const float f = m1 == kNone ? 1.0f : exp2_(m - m1);
        m = m1;
        z *= f;
#pragma unroll
        for (int i = 0; i < MT; ++i) o[i] *= f;
      }
      const float ref = m == kNone ? 0.0f : m;
      u32x4 hi, lo;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float p0 = exp2_(sc[e >> 2][e & 3] - ref), p1 = exp2_(sc[e >> 2][(e & 3) + 1] - ref);
        z += p0 + p1;
        const uint32_t u = pack2<T>(p0, p1);
        hi[e >> 1] = u;
        lo[e >> 1] = pack2<T>(p0 - unpack<T>(u, 0), p1 - unpack<T>(u, 1));
      }
      // V: registers -> the wave's copy -> columns
#pragma unroll
      for (int i = 0; i < VLOADS; ++i) {
        const int r = i * (64 / LANES) + lane / LANES;
        u32x4 v = vr[i];
        if (seen != 0xFFFFFFFFu && !((seen >> r) & 1)) v = (u32x4)(0);
        *reinterpret_cast<u32x4*>(copy + r * (D * 2) + (((lane % LANES) ^ swizzle(r)) << 4)) = v;
      }
      if (more) load_v(next);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        u32x4 vf;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int r = 16 * half + 4 * quad + (l16 >> 2), c = 2 * mt + ((l16 & 3) >> 1);
          const u32x2 x = read_columns(copy + r * (D * 2) + ((c ^ swizzle(r)) << 4) + 8 * (l16 & 1));
          vf[2 * half] = x[0];
          vf[2 * half + 1] = x[1];
        }
        o[mt] = Elem<T>::mfma16(vf, hi, o[mt]);
        o[mt] = Elem<T>::mfma16(vf, lo, o[mt]);
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
      row = next;
    }
  }
  z += __shfl_xor(z, 16);
  z += __shfl_xor(z, 32);

  // The waves of a head group meet: exponents and sums first, then the outputs, [head][d] in the copies' place.
  if (quad == 0) {
    lds_mz[wave][l16][0] = m;
    lds_mz[wave][l16][1] = z;
  }
  static_assert(16 * D * 4 <= kTile * D * 2, "a wave's outputs fit its copy");
  float* const mine = reinterpret_cast<float*>(copy);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) *reinterpret_cast<f32x4*>(mine + l16 * D + (((4 * mt + quad) ^ (l16 & 7)) << 2)) = o[mt];
  __syncthreads();
  // a thread: four outputs of one head at a time
  const int heads = min(16 * a.wave_groups, a.G - 64 * hg);
  for (int i = threadIdx.x; i < heads * (D / 4); i += 256) {
    const int hh = i / (D / 4), d4 = i % (D / 4), w0 = hh >> 4, hl = hh & 15;
    float top = kNone;
    for (int w = w0; w < kWaves; w += a.wave_groups) top = fmaxf(top, lds_mz[w][hl][0]);
    const float ref = top == kNone ? 0.0f : top;
    float sum = 0.0f;
    f32x4 acc = (f32x4)(0.0f);
    for (int w = w0; w < kWaves; w += a.wave_groups) {
      const float f = exp2_(lds_mz[w][hl][0] - ref);
      sum += f * lds_mz[w][hl][1];
      acc += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(lds_v[w]) + hl * D + ((d4 ^ (hl & 7)) << 2));
    }
    const int64_t row = (int64_t)b * a.Hq + g * a.G + 64 * hg + hh;
    if (a.S > 1) {
      *reinterpret_cast<f32x4*>(a.part_o + (row * a.S + s) * D + 4 * d4) = acc;
      if (d4 == 0) {
        a.part_mz[(row * a.S + s) * 2] = top;
        a.part_mz[(row * a.S + s) * 2 + 1] = sum;
      }
    } else {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      u32x2 w;
      w[0] = pack2<T>(acc[0] * inv, acc[1] * inv);
      w[1] = pack2<T>(acc[2] * inv, acc[3] * inv);
      *reinterpret_cast<u32x2*>(a.out + row * D + 4 * d4) = w;
      if (d4 == 0 && a.lse) a.lse[row] = sum == 0.0f ? kNone : (top + log2_(sum)) * kLn2;
    }
  }
}

// One workgroup per (sequence, query head): the ranges' results in order, 8 threads' shares of them added at the end.
template <typename T, int D>
__global__ __launch_bounds__(256) void decode_long_join_kernel(const LongArgs a) {
  constexpr int PARTS = 256 / (D / 4);
  __shared__ float lds_w[kMaxRanges];
  __shared__ float lds_red[8];
  __shared__ f32x4 lds_o[PARTS][D / 4];
  const int64_t row = blockIdx.x;
  const float* mz = a.part_mz + row * a.S * 2;
  float top = kNone;
  for (int i = threadIdx.x; i < a.S; i += 256) top = fmaxf(top, mz[2 * i]);
  for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
  if ((threadIdx.x & 63) == 0) lds_red[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(lds_red[0], lds_red[1]), fmaxf(lds_red[2], lds_red[3]));
  const float ref = top == kNone ? 0.0f : top;
  float sum = 0.0f;
  for (int i = threadIdx.x; i < a.S; i += 256) {
    const float f = exp2_(mz[2 * i] - ref);
    lds_w[i] = f;
    sum += f * mz[2 * i + 1];
  }
  for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
  if ((threadIdx.x & 63) == 0) lds_red[4 + (threadIdx.x >> 6)] = sum;
  __syncthreads();
  sum = (lds_red[4] + lds_red[5]) + (lds_red[6] + lds_red[7]);
  const int d4 = threadIdx.x % (D / 4), part = threadIdx.x / (D / 4);
  f32x4 acc = (f32x4)(0.0f);
  for (int i = part; i < a.S; i += PARTS) {
    const float f = lds_w[i];
    if (f != 0.0f) acc += f * *reinterpret_cast<const f32x4*>(a.part_o + (row * a.S + i) * D + 4 * d4);
  }
  lds_o[part][d4] = acc;
  __syncthreads();
  if (part == 0) {
    for (int i = 1; i < PARTS; ++i) acc += lds_o[i][d4];
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    u32x2 w;
    w[0] = pack2<T>(acc[0] * inv, acc[1] * inv);
    w[1] = pack2<T>(acc[2] * inv, acc[3] * inv);
    *reinterpret_cast<u32x2*>(a.out + row * D + 4 * d4) = w;
    if (d4 == 0 && a.lse) a.lse[row] = sum == 0.0f ? kNone : (top + log2_(sum)) * kLn2;
  }
}

template <typename T, int D>
hipError_t launch(const LongArgs& a, hipStream_t s) {
  const dim3 grid(a.S, a.Hkv * a.head_groups, a.B), block(256);
  hipLaunchKernelGGL((decode_long_kernel<T, D>), grid, block, 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.S == 1) return e;
  hipLaunchKernelGGL((decode_long_join_kernel<T, D>), dim3((unsigned)(a.B * a.Hq)), block, 0, s, a);
  return hipGetLastError();
}

// Ranges per (sequence, KV head): as many as give 1024 workgroups (two per compute unit at a time, so that a range that starts
// late costs half a turn at most), but none below 256 keys.
int ranges(const pkv_decode_long_desc& d) {
  const int64_t units = (int64_t)d.B * d.Hkv * ((d.Hq / d.Hkv + 63) / 64);
  int64_t S = (1024 + units - 1) / units;
  const int64_t most = ((int64_t)d.k_cap + 255) / 256;
  if (S > most) S = most;
  if (S > kMaxRanges) S = kMaxRanges;
  return (int)(S < 1 ? 1 : S);
}

bool aligned(const void* p, int n) { return ((uintptr_t)p & (n - 1)) == 0; }

int check_long_desc(const pkv_decode_long_desc* desc) {
  if (!desc) return PKV_ERR_INVALID_ARG;
  const pkv_decode_long_desc& d = *desc;
  if (d.B < 1 || d.Hq < 1 || d.Hkv < 1 || d.Hq % d.Hkv != 0 || d.k_cap < 1 || d.page_size < 0 || d.window < 0) return PKV_ERR_INVALID_ARG;
  if (d.dtype != PKV_BF16 && d.dtype != PKV_FP16) return PKV_ERR_INVALID_ARG;
  if (!(d.scale >= 0.0f) || !(d.cap >= 0.0f) || !isfinite(d.scale) || !isfinite(d.cap)) return PKV_ERR_INVALID_ARG;
  if (d.q_sb < 0 || d.q_sb % 8 != 0 || d.q_sh < 0 || d.q_sh % 8 != 0) return PKV_ERR_INVALID_ARG;
  if (d.page_size > 0) {
    if (d.num_pages < 1 || d.max_pages < ((int64_t)d.k_cap + d.page_size - 1) / d.page_size) return PKV_ERR_INVALID_ARG;
  } else {
    const int64_t st[3] = {d.c_sb, d.c_sh, d.c_st};
    for (int i = 0; i < 3; ++i)
      if (st[i] < 0 || st[i] % 8 != 0) return PKV_ERR_INVALID_ARG;
  }
  if (d.p_sb < 0 || d.p_sh < 0) return PKV_ERR_INVALID_ARG;
  if (d.d != 64 && d.d != 128) return PKV_ERR_UNSUPPORTED;
  const int64_t G = d.Hq / d.Hkv;
  if (G > 128 || d.B > 65535 || d.k_cap > (1 << 30) || d.Hkv * ((G + 63) / 64) > 65535 || (int64_t)d.B * d.Hq > 0x7FFFFFFF) return PKV_ERR_UNSUPPORTED;
  // rows of a pool are counted in 32 bits
  if (d.page_size > 0 && (double)d.num_pages * d.Hkv * d.page_size > 4294967295.0) return PKV_ERR_UNSUPPORTED;
  return PKV_OK;
}

}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

size_t pkv_decode_long_workspace_bytes(const pkv_decode_long_desc* desc) {
  if (check_long_desc(desc) != PKV_OK) return 0;
  const int S = ranges(*desc);
  return S == 1 ? 0 : (size_t)desc->B * desc->Hq * S * (desc->d + 2) * sizeof(float);
}

int pkv_decode_attention_long(const pkv_decode_long_desc* desc, const void* q, const void* K_cache, const void* V_cache,
                              const int32_t* block_table, const int32_t* count, const int32_t* positions, const int32_t* q_pos,
                              const float* slopes, void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc || !q || !K_cache || !V_cache || !count || !out) return PKV_ERR_INVALID_ARG;
  const int rc = check_long_desc(desc);
  if (rc != PKV_OK) return rc;
  const pkv_decode_long_desc& d = *desc;
  if (!aligned(q, 16) || !aligned(K_cache, 16) || !aligned(V_cache, 16) || !aligned(out, 16) || !aligned(block_table, 4) ||
      !aligned(count, 4) || !aligned(positions, 4) || !aligned(q_pos, 4) || !aligned(slopes, 4) || !aligned(lse_out, 4))
    return PKV_ERR_INVALID_ARG;
  if (d.page_size > 0 && !block_table) return PKV_ERR_INVALID_ARG;
  const size_t need = pkv_decode_long_workspace_bytes(desc);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return PKV_ERR_WORKSPACE;
  LongArgs a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const uint16_t*>(q);
  a.K = static_cast<const uint16_t*>(K_cache);
  a.V = static_cast<const uint16_t*>(V_cache);
  a.table = block_table; a.count = count; a.positions = positions; a.q_pos = q_pos; a.slopes = slopes;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse_out;
  a.S = ranges(d);
  a.part_o = static_cast<float*>(workspace);
  a.part_mz = a.part_o ? a.part_o + (size_t)d.B * d.Hq * a.S * d.d : nullptr;
  a.B = d.B; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.Hq / d.Hkv; a.k_cap = d.k_cap;
  a.page_size = d.page_size; a.num_pages = d.num_pages; a.max_pages = d.max_pages; a.window = d.window;
  a.head_groups = (a.G + 63) / 64;
  a.wave_groups = a.G <= 16 ? 1 : a.G <= 32 ? 2 : 4;
  a.page_magic = d.page_size > 1 ? (uint32_t)(((uint64_t)1 << 32) / (uint32_t)d.page_size) : 0xFFFFFFFFu;
  a.q_sb = d.q_sb; a.q_sh = d.q_sh; a.c_sb = d.c_sb; a.c_sh = d.c_sh; a.c_st = d.c_st; a.p_sb = d.p_sb; a.p_sh = d.p_sh;
  const double scale = d.scale > 0.0f ? (double)d.scale : 1.0 / sqrt((double)d.d);
  a.scale = (float)(d.cap > 0.0f ? scale : scale * 1.4426950408889634);
  a.cap2 = d.cap * kLog2e;
  a.two_over_cap = d.cap > 0.0f ? 2.0f * kLog2e / d.cap : 0.0f;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (d.dtype == PKV_BF16)
    e = d.d == 128 ? launch<__bf16, 128>(a, st) : launch<__bf16, 64>(a, st);
  else
    e = d.d == 128 ? launch<_Float16, 128>(a, st) : launch<_Float16, 64>(a, st);
  return e == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
