// Rotary positions of new tokens and their append to a cache (include/pkv.h: pkv_rotary_append).
//
// Every element is read once and written once and has a handful of operations; what costs besides is the sine and cosine of
// a (token, pair), in 64 bits up to the fraction of a turn.  Hence one thread per (token, 8 elements of a head), which forms
// its four pairs' sines once and goes over heads of the token with them: 16 neighbouring lanes (8 at d = 64) move one row of a
// head.  A workgroup takes up to 16 tokens, so that what it writes per head lies together, and the heads are dealt out over the
// grid until there are enough workgroups.  Eight ragged prompts of up to 16k tokens (32 / 8 heads, d 128, 2.0 GB moved): 415 us,
// 4.85 TB/s, which is the rate of a large copy; one token: 3.3 us, a launch with a handful of loads behind one another.
#include <math.h>

#include "pkv_hostcheck.h"
#include "pkv_internal.h"

namespace pkv {
namespace {

struct RotaryArgs {
  const uint16_t *q, *k, *v;
  const double* inv_freq;
  const int32_t *positions, *new_lens, *count, *table;
  uint16_t *q_out, *K, *V;
  int32_t *pos_cache, *dropped;
  int32_t B, Hq, Hkv, T, rot, k_cap, page_size, num_pages, max_pages;
  int32_t heads_q, heads;      // query heads given (0 or Hq); they, the key heads and the value heads
  int32_t heads_per_wg;
  float magnitude;
  int64_t q_sb, q_sh, q_st, k_sb, k_sh, k_st, v_sb, v_sh, v_st, o_sb, o_sh, o_st, c_sb, c_sh, c_st, p_sb, p_sh;
};

// Valid new tokens of sequence b, and the row of the first of them.
__device__ __forceinline__ int new_tokens(const RotaryArgs& a, int b) {
  return a.new_lens ? min(max(a.new_lens[b], 0), a.T) : a.T;
}
__device__ __forceinline__ int64_t first_row(const RotaryArgs& a, int b, int n_new) {
  return a.count ? (int64_t)a.count[b] - n_new : 0;
}

// Element offset of head 0 of row r of sequence b, or -1 if there is no such row; *head_stride between heads.
__device__ __forceinline__ int64_t row_offset(const RotaryArgs& a, int b, int64_t r, int d, int64_t* head_stride) {
  if (r < 0 || r >= a.k_cap) return -1;
  if (a.page_size == 0) {
    *head_stride = a.c_sh;
    return b * a.c_sb + r * a.c_st;
  }
  const int page = a.table[(int64_t)b * a.max_pages + r / a.page_size];
  if (page < 0 || page >= a.num_pages) return -1;
  *head_stride = (int64_t)a.page_size * d;
  return ((int64_t)page * a.Hkv * a.page_size + r % a.page_size) * d;
}

// Sine and cosine of p f radians.  In 64 bits: the angle, and its distance from the nearest multiple of pi / 2 (which has two
// words, so that only the angle's own rounding counts); in 32: the Taylor series of both at |y| <= pi / 4 (remainders
// y^11 / 11! < 2e-9 and y^12 / 12! < 2e-10).
__device__ __forceinline__ void sine_cosine(int p, double f, float m, float* s, float* c) {
  const double angle = (double)p * f;
  const double quarter = rint(angle * 0.6366197723675814);
  const float y = (float)fma(-quarter, 6.123233995736766e-17, fma(-quarter, 1.5707963267948966, angle));
  const float y2 = y * y;
  const float sn = y * fmaf(y2, fmaf(y2, fmaf(y2, fmaf(y2, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), 1.0f);
  const float cs = fmaf(y2, fmaf(y2, fmaf(y2, fmaf(y2, fmaf(y2, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
  const int n = (int)(long long)quarter;
  const float s0 = n & 1 ? cs : sn, c0 = n & 1 ? sn : cs;
  *s = m * (n & 2 ? -s0 : s0);
  *c = m * (((n + 1) & 2) ? -c0 : c0);
}

template <typename T>
struct alignas(16) Eight {
  T x[8];
};
template <typename T>
struct alignas(8) Four {
  T x[4];
};

// What a thread does with one head's row: its eight elements from src to dst, turned or copied.
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void move_eight(const T* src, T* dst, int unit, int rot, bool turns, const float (&s)[4], const float (&c)[4]) {
  if (!turns) {
    *reinterpret_cast<Eight<T>*>(dst + 8 * unit) = *reinterpret_cast<const Eight<T>*>(src + 8 * unit);
  } else if constexpr (INTERLEAVED) {
    Eight<T> x = *reinterpret_cast<const Eight<T>*>(src + 8 * unit);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float xa = (float)x.x[2 * i], xb = (float)x.x[2 * i + 1];
      x.x[2 * i] = (T)(xa * c[i] - xb * s[i]);
      x.x[2 * i + 1] = (T)(xb * c[i] + xa * s[i]);
    }
    *reinterpret_cast<Eight<T>*>(dst + 8 * unit) = x;
  } else {
    Four<T> u = *reinterpret_cast<const Four<T>*>(src + 4 * unit), w = *reinterpret_cast<const Four<T>*>(src + rot / 2 + 4 * unit);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float xa = (float)u.x[i], xb = (float)w.x[i];
      u.x[i] = (T)(xa * c[i] - xb * s[i]);
      w.x[i] = (T)(xb * c[i] + xa * s[i]);
    }
    *reinterpret_cast<Four<T>*>(dst + 4 * unit) = u;
    *reinterpret_cast<Four<T>*>(dst + rot / 2 + 4 * unit) = w;
  }
}

// TOKENS tokens of the batch per workgroup (token numbers run over the sequences), the other threads over the heads.
template <typename T, int D, bool INTERLEAVED, int TOKENS>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a) {
  constexpr int LANES = D / 8, HEADS = 256 / LANES / TOKENS;  // lanes of a row; heads the workgroup moves at the same time
  const int unit = threadIdx.x % LANES, row = threadIdx.x / LANES;
  const int64_t token = (int64_t)blockIdx.x * TOKENS + row % TOKENS;
  if (token >= (int64_t)a.B * a.T) return;
  const int b = (int)(token / a.T), t = (int)(token - (int64_t)b * a.T);
  const int n_new = new_tokens(a, b);
  if (t >= n_new) return;
  const int64_t r = first_row(a, b, n_new) + t;
  const int p = a.positions ? a.positions[token] : (int)r;
  const bool turns = 8 * unit < a.rot;
  float s[4] = {0, 0, 0, 0}, c[4] = {0, 0, 0, 0};
  if (turns) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sine_cosine(p, a.inv_freq[4 * unit + i], a.magnitude, &s[i], &c[i]);
  }
  int64_t head_stride = 0;
  const int64_t at = a.K ? row_offset(a, b, r, D, &head_stride) : -1;
  const int h0 = blockIdx.y * a.heads_per_wg, h1 = min(h0 + a.heads_per_wg, a.heads);
  for (int h = h0 + row / TOKENS; h < h1; h += HEADS) {
    if (h < a.heads_q) {
      move_eight<T, INTERLEAVED>(reinterpret_cast<const T*>(a.q) + b * a.q_sb + h * a.q_sh + t * a.q_st,
                                 reinterpret_cast<T*>(a.q_out) + b * a.o_sb + h * a.o_sh + t * a.o_st, unit, a.rot, turns, s, c);
    } else if (at >= 0) {
      const int g = h - a.heads_q;
      if (g < a.Hkv) {
        move_eight<T, INTERLEAVED>(reinterpret_cast<const T*>(a.k) + b * a.k_sb + g * a.k_sh + t * a.k_st,
                                   reinterpret_cast<T*>(a.K) + at + g * head_stride, unit, a.rot, turns, s, c);
        if (a.pos_cache && unit == 0) a.pos_cache[b * a.p_sb + g * a.p_sh + r] = p;
      } else {
        move_eight<T, INTERLEAVED>(reinterpret_cast<const T*>(a.v) + b * a.v_sb + (g - a.Hkv) * a.v_sh + t * a.v_st,
                                   reinterpret_cast<T*>(a.V) + at + (g - a.Hkv) * head_stride, unit, a.rot, false, s, c);
      }
    }
  }
}

// Tokens of a sequence that have no row: one workgroup per sequence.
__global__ __launch_bounds__(256) void rotary_dropped_kernel(const RotaryArgs a, int d) {
  __shared__ int part[4];
  const int b = blockIdx.x;
  const int n_new = new_tokens(a, b);
  const int64_t r0 = first_row(a, b, n_new);
  int n = 0;
  if (a.K) {
    for (int t = threadIdx.x; t < n_new; t += 256) {
      int64_t hs;
      n += row_offset(a, b, r0 + t, d, &hs) < 0;
    }
  }
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) a.dropped[b] = part[0] + part[1] + part[2] + part[3];
}

template <typename T, int D, bool INTERLEAVED>
hipError_t launch(RotaryArgs& a, hipStream_t s) {
  constexpr int LANES = D / 8;
  const int64_t tokens = (int64_t)a.B * a.T;
  const bool few = tokens < 16;  // (then the threads go over the heads of one token)
  const int per = few ? 1 : 16, heads_at_once = 256 / LANES / per;
  const int64_t gx = (tokens + per - 1) / per;
  // As many heads per workgroup as leave four workgroups per compute unit: a thread's sines serve all of them.
  int64_t gy = (a.heads + heads_at_once - 1) / heads_at_once;
  const int64_t enough = (1024 + gx - 1) / gx;
  if (gy > enough) gy = enough;
  a.heads_per_wg = (int)((a.heads + gy - 1) / gy);
  gy = (a.heads + a.heads_per_wg - 1) / a.heads_per_wg;
  if (a.heads > 0) {
    const dim3 grid((unsigned)gx, (unsigned)gy), block(256);
    if (few)
      hipLaunchKernelGGL((rotary_kernel<T, D, INTERLEAVED, 1>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((rotary_kernel<T, D, INTERLEAVED, 16>), grid, block, 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dropped) {
    hipLaunchKernelGGL(rotary_dropped_kernel, dim3(a.B), dim3(256), 0, s, a, D);
    return hipGetLastError();
  }
  return hipSuccess;
}

template <typename T, int D>
hipError_t launch_layout(RotaryArgs& a, int layout, hipStream_t s) {
  return layout == PKV_ROTARY_INTERLEAVED ? launch<T, D, true>(a, s) : launch<T, D, false>(a, s);
}


}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

int pkv_rotary_frequencies(int32_t rot, int32_t scaling, double base, double factor, double trained, double low, double high,
                           double* inv_freq_out, float* magnitude_out) {
  if (!inv_freq_out || !magnitude_out || rot < 2 || rot > 256 || rot % 2 != 0) return PKV_ERR_INVALID_ARG;
  if (scaling < PKV_ROTARY_PLAIN || scaling > PKV_ROTARY_RAMP || !(base > 1.0) || !isfinite(base)) return PKV_ERR_INVALID_ARG;
  if (scaling != PKV_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return PKV_ERR_INVALID_ARG;
  const bool bands = scaling == PKV_ROTARY_BANDS, ramp = scaling == PKV_ROTARY_RAMP;
  if ((bands || ramp) && (!(trained > 0.0) || !(low > 0.0) || !(high > low) || !isfinite(trained) || !isfinite(high)))
    return PKV_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925;
  double from = 0, to = 0;
  if (ramp) {
    from = floor(rot * log(trained / (two_pi * high)) / (2 * log(base)));
    to = ceil(rot * log(trained / (two_pi * low)) / (2 * log(base)));
    from = fmax(from, 0.0);
    to = fmin(to, rot - 1.0);
  }
  for (int32_t i = 0; i < rot / 2; ++i) {
    const double f = pow(base, -2.0 * i / rot);
    double mine = 0;  // share of the frequency that stays as it is
    if (scaling == PKV_ROTARY_PLAIN) mine = 1;
    if (bands) mine = (trained * f / two_pi - low) / (high - low);
    if (ramp) mine = 1 - (i - from) / fmax(to - from, 0.001);
    mine = fmin(fmax(mine, 0.0), 1.0);
    inv_freq_out[i] = scaling == PKV_ROTARY_PLAIN ? f : (1 - mine) * (f / factor) + mine * f;
  }
  *magnitude_out = ramp && factor > 1 ? (float)(0.1 * log(factor) + 1) : 1.0f;
  return PKV_OK;
}

int pkv_rotary_append(const pkv_rotary_desc* desc, const void* q, const void* k, const void* v, const double* inv_freq,
                      const int32_t* positions, const int32_t* new_lens, const int32_t* count, const int32_t* block_table,
                      void* q_out, void* K_cache, void* V_cache, int32_t* pos_cache, int32_t* dropped_out, void* stream) {
  if (!desc || !inv_freq) return PKV_ERR_INVALID_ARG;
  const pkv_rotary_desc& d = *desc;
  if (d.B < 1 || d.Hq < 1 || d.Hkv < 1 || d.T < 1 || d.reserved != 0 || !isfinite(d.magnitude)) return PKV_ERR_INVALID_ARG;
  if (d.layout != PKV_ROTARY_HALF && d.layout != PKV_ROTARY_INTERLEAVED) return PKV_ERR_INVALID_ARG;
  if (d.dtype != PKV_BF16 && d.dtype != PKV_FP16) return PKV_ERR_INVALID_ARG;
  const bool has_q = q || q_out, has_kv = k || v || K_cache || V_cache;
  if ((!has_q && !has_kv) || (has_q && (!q || !q_out)) || (has_kv && (!k || !v || !K_cache || !V_cache))) return PKV_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(q_out, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(K_cache, 16) || !aligned(V_cache, 16) ||
      !aligned(inv_freq, 8) || !aligned(positions, 4) || !aligned(new_lens, 4) || !aligned(count, 4) || !aligned(block_table, 4) ||
      !aligned(pos_cache, 4) || !aligned(dropped_out, 4))
    return PKV_ERR_INVALID_ARG;
  if (has_q && (!good_strides(d.q_sb, d.q_sh, d.q_st) || !good_strides(d.o_sb, d.o_sh, d.o_st))) return PKV_ERR_INVALID_ARG;
  if (has_kv) {
    if (!good_strides(d.k_sb, d.k_sh, d.k_st) || !good_strides(d.v_sb, d.v_sh, d.v_st)) return PKV_ERR_INVALID_ARG;
    if (d.k_cap < 1 || d.page_size < 0) return PKV_ERR_INVALID_ARG;
    if (d.page_size > 0) {
      if (!block_table || d.num_pages < 1 || d.max_pages < ((int64_t)d.k_cap + d.page_size - 1) / d.page_size) return PKV_ERR_INVALID_ARG;
    } else if (!good_strides(d.c_sb, d.c_sh, d.c_st) || d.c_st < d.d) {
      return PKV_ERR_INVALID_ARG;
    }
    if (pos_cache && (d.p_sb < 0 || d.p_sh < 0)) return PKV_ERR_INVALID_ARG;
  } else if (pos_cache) {
    return PKV_ERR_INVALID_ARG;
  }
  if (d.rot < 2 || d.rot > d.d || d.rot % 2 != 0) return PKV_ERR_INVALID_ARG;
  if ((d.d != 64 && d.d != 128) || d.rot % 8 != 0) return PKV_ERR_UNSUPPORTED;
  if ((int64_t)d.B * d.T > 16 * kMaxGrid || d.B > kMaxGrid || (int64_t)d.Hq + 2 * (int64_t)d.Hkv > 65535) return PKV_ERR_UNSUPPORTED;
  RotaryArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.inv_freq = inv_freq;
  a.positions = positions; a.new_lens = new_lens; a.count = count; a.table = block_table;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.K = static_cast<uint16_t*>(K_cache);
  a.V = static_cast<uint16_t*>(V_cache);
  a.pos_cache = pos_cache; a.dropped = dropped_out;
  a.B = d.B; a.Hq = d.Hq; a.Hkv = d.Hkv; a.T = d.T; a.rot = d.rot; a.k_cap = d.k_cap;
  a.page_size = d.page_size; a.num_pages = d.num_pages; a.max_pages = d.max_pages;
  a.heads_q = has_q ? d.Hq : 0;
  a.heads = a.heads_q + (has_kv ? 2 * d.Hkv : 0);
  a.heads_per_wg = 0;
  a.magnitude = d.magnitude;
  a.q_sb = d.q_sb; a.q_sh = d.q_sh; a.q_st = d.q_st; a.k_sb = d.k_sb; a.k_sh = d.k_sh; a.k_st = d.k_st;
  a.v_sb = d.v_sb; a.v_sh = d.v_sh; a.v_st = d.v_st; a.o_sb = d.o_sb; a.o_sh = d.o_sh; a.o_st = d.o_st;
  a.c_sb = d.c_sb; a.c_sh = d.c_sh; a.c_st = d.c_st; a.p_sb = d.p_sb; a.p_sh = d.p_sh;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (d.dtype == PKV_BF16)
    e = d.d == 128 ? launch_layout<__bf16, 128>(a, d.layout, s) : launch_layout<__bf16, 64>(a, d.layout, s);
  else
    e = d.d == 128 ? launch_layout<_Float16, 128>(a, d.layout, s) : launch_layout<_Float16, 64>(a, d.layout, s);
  return e == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
