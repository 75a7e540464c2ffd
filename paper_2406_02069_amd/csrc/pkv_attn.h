// Pieces shared by the attention kernels over whole caches (pkv_prefill.hip, pkv_decode_long.hip).
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

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }

// cap * tanh(s / cap) as cap - 2 cap / (1 + e^(2s / cap)): two transcendental instructions, absolute error about 2^-23 cap, right
// at both ends (e^... = inf or 0).  x * to_exponent is the exponent to base 2, 2 log2(e) s / cap.
__device__ __forceinline__ float capped(float x, float to_exponent, float cap) {
  return fmaf(-2.0f * cap, __builtin_amdgcn_rcpf(1.0f + exp2_(x * to_exponent)), cap);
}

}  // namespace
}  // namespace pkv
