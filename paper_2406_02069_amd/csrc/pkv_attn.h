// Pieces shared by the attention kernels over whole caches (pkv_prefill.hip, pkv_long.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pkv_internal.h"
#include "pkv_hostcheck.h"

namespace pkv {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -__builtin_inff();

// The two element types: pairs and operands of a matrix instruction.
template <typename T>
struct Elem;
template <>
struct Elem<__bf16> {
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  __device__ static __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  __device__ static __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
};
template <>
struct Elem<_Float16> {
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  __device__ static __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  __device__ static __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
};

// Softmax weights in fp16 are 2^(score - reference + kFp16Shift), and the reference moves once a score exceeds it by more than
// kFp16Slack: 2^15 at most.  The type's steps end at 2^-24, so that weights far below the largest lose their bits and then vanish,
// while their sum in fp32 keeps them; this way the last step is 2^-37 of the reference.  (bf16 has fp32's exponents.)
constexpr float kFp16Shift = 13.0f, kFp16Slack = 2.0f;

// Two floats rounded to the type (to nearest, ties to even), the first one in the low half.
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typename Elem<T>::x2 r;
  r[0] = (T)a;
  r[1] = (T)b;
  return __builtin_bit_cast(uint32_t, r);
}
template <typename T>
__device__ __forceinline__ float unpack(uint32_t u, int i) {
  return (float)__builtin_bit_cast(typename Elem<T>::x2, u)[i];
}

// Of 4 x 16 elements, four 16-bit elements at each of 16 neighbouring lanes' addresses (lanes 4 r .. 4 r + 3 name row r),
// lane i gets column i: the elements of rows 0 .. 3.
__device__ __forceinline__ u32x2 read_columns(const char* lds) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lds)));
}

// Halves of a word whose exponent is all ones (bit 15, bit 31 set).
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t u);
template <>
__device__ __forceinline__ uint32_t not_finite<__bf16>(uint32_t u) {
  return ((u & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
}
template <>
__device__ __forceinline__ uint32_t not_finite<_Float16>(uint32_t u) {
  return ((u & 0x7C007C00u) + 0x04000400u) & 0x80008000u;
}

// (in a scalar register)
__device__ __forceinline__ int wave_max(int x) {
  for (int o = 32; o > 0; o >>= 1) x = max(x, __shfl_xor(x, o));
  return __builtin_amdgcn_readfirstlane(x);
}

// The wave's number in its workgroup, in a scalar register.
__device__ __forceinline__ int this_wave() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// Sum over the wave, up to and including the own lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_from(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int sum_upto(int x) {
  x = add_from<0x111, 0xF>(x);  // row_shr 1, 2, 4, 8: within rows of 16
  x = add_from<0x112, 0xF>(x);
  x = add_from<0x114, 0xF>(x);
  x = add_from<0x118, 0xF>(x);
  x = add_from<0x142, 0xA>(x);  // the rows' sums: row_bcast 15 into rows 1 and 3, row_bcast 31 into rows 2 and 3
  return add_from<0x143, 0xC>(x);
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }

// a f + b g, of results with positive factors, which may be too small for fp32: what is not finite is added as it is.
__device__ __forceinline__ f32x4 weighed(f32x4 a, float f, f32x4 b, float g) {
  f32x4 r = a * f + b * g;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool fa = fabsf(a[i]) < __builtin_inff(), fb = fabsf(b[i]) < __builtin_inff();
    if (!(fa && fb)) r[i] = (fa ? 0.0f : a[i]) + (fb ? 0.0f : b[i]);
  }
  return r;
}

__device__ __forceinline__ bool finite(f32x4 v) {
  return fabsf(v[0]) < __builtin_inff() && fabsf(v[1]) < __builtin_inff() && fabsf(v[2]) < __builtin_inff() && fabsf(v[3]) < __builtin_inff();
}

// Scores capped by a tanh, from products x to log2 units: cap tanh(y) log2(e), y = x scale / cap.
// |y| <= 0.36, where scores lie in earnest: y P(y^2), P of degree 3 (least squares reweighted to even out its relative error,
// 5e-8 at most): a polynomial in x^2, five instructions, exact to a few 2^-24 of the score itself.
// Beyond: cap - 2 cap / (1 + e^(2y)): two transcendental instructions, absolute error about 2^-23 cap (too much for small
// scores), right at both ends (e^... = inf or 0).  This form alone where the polynomial's coefficients leave fp32 (scale / cap above
// a million): products of any size then give the cap itself.
struct Cap {
  float c0, c1, c2, c3;  // coefficients in x^2
  float limit;           // of |x|
  float to_exponent;     // 2 log2(e) scale / cap
  float cap;             // in log2 units; 0: none
};
inline Cap make_cap(double scale, double cap) {
  Cap c = {0, 0, 0, 0, 0, 0, 0};
  if (cap > 0) {
    const double f = scale * 1.4426950408889634, k = scale / cap, k2 = k * k;
    c.c0 = (float)f;
    c.c1 = (float)(-0.33332544 * f * k2);
    c.c2 = (float)(0.13296013 * f * k2 * k2);
    c.c3 = (float)(-0.04888798 * f * k2 * k2 * k2);
    c.limit = (float)(0.36 / k);
    c.to_exponent = (float)(2.0 * 1.4426950408889634 * k);
    c.cap = (float)(cap * 1.4426950408889634);
    if (!(fabsf(c.c1) < __builtin_inff() && fabsf(c.c2) < __builtin_inff() && fabsf(c.c3) < __builtin_inff()))
      c.c1 = c.c2 = c.c3 = c.limit = 0.0f;
  }
  return c;
}
// Whether scale and cap leave factors that fp32 holds.
inline bool finite_factors(double scale, double cap) {
  const Cap c = make_cap(scale, cap);
  const float f[7] = {c.c0, c.c1, c.c2, c.c3, c.limit, c.to_exponent, c.cap};
  for (int i = 0; i < 7; ++i)
    if (!(f[i] - f[i] == 0.0f)) return false;
  const float s = (float)(scale * 1.4426950408889634);
  return s - s == 0.0f;
}
__device__ __forceinline__ float capped_small(float x, const Cap& c) {
  const float x2 = x * x;
  return x * fmaf(fmaf(fmaf(c.c3, x2, c.c2), x2, c.c1), x2, c.c0);
}
__device__ __forceinline__ float capped_any(float x, const Cap& c) {
  const float far = fmaf(-2.0f * c.cap, __builtin_amdgcn_rcpf(1.0f + exp2_(x * c.to_exponent)), c.cap);
  return fabsf(x) <= c.limit ? capped_small(x, c) : far;
}
// N scores of every lane; the second form only where some lane of the wave needs it.
template <int N>
__device__ __forceinline__ void cap_scores(float (&x)[N], const Cap& c) {
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(x[i]));
  if (__any(most > c.limit)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = capped_any(x[i], c);
      __builtin_amdgcn_sched_barrier(0);  // (one after the other: this is rare, and registers are not)
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = capped_small(x[i], c);
  }
}

// ---- kernels that form 32 x 32 tiles of scores, keys and values straight from memory in LDS ----

// References (log2) beyond which a score is rounded before it is compared with them: what one fma of scale and difference finds
// left of a rounded product is as large as a step there, and would be a weight's exponent.
constexpr float kLarge = 0x1p20f;

// 16 bytes per lane from base + at into LDS, lane after lane from byte `to` on.  Asynchronous: wait_loads.  (Written out because
// the compiler lets every later read of LDS wait for such a load, though it goes to another buffer; nothing is returned in
// registers.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is a register that the compiler keeps to itself; nothing else here uses it)
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t at, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(at), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// Waits for the asynchronous loads into LDS, but for the last LATER (below 16) of them: loads end in the order of their requests.
template <int LATER = 0>
__device__ __forceinline__ void wait_loads() {
  static_assert(LATER < 16, "the counter's low bits");
  __builtin_amdgcn_s_waitcnt(0x0F70 | LATER);  // vmcnt
  asm volatile("" : : : "memory");
}

// The first key of register i of a 32 x 32 product, in the lower half of the wave (the upper half: 4 more).
__device__ __forceinline__ constexpr int key_of(int i) { return 8 * (i >> 2) + (i & 3); }

template <int D>
__device__ __forceinline__ int swizzle_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D>
__device__ __forceinline__ int swizzle_v(int row) { return D == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1); }

}  // namespace
}  // namespace pkv
