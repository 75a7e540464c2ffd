// What the entry points of pkv_rotary.hip, pkv_prefill.hip and pkv_decode_long.hip ask of their arguments.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace pkv {
namespace {

constexpr int64_t kMaxGrid = 0xFFFFFF;  // workgroups of 256 in one dimension of a launch: 2^32 threads

inline bool aligned(const void* p, int n) { return ((uintptr_t)p & (uintptr_t)(n - 1)) == 0; }

// Element strides that keep rows 16-byte aligned.
inline bool good_strides(int64_t sb, int64_t sh, int64_t st) {
  return sb >= 0 && sh >= 0 && st >= 0 && sb % 8 == 0 && sh % 8 == 0 && st % 8 == 0;
}

}  // namespace
}  // namespace pkv
