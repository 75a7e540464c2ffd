// What csrc/pkv_topk.h takes from csrc/pkv_attn.h, on the CPU.
#pragma once

#include <hip/hip_runtime.h>

namespace pkv {
namespace {

inline int current_device_slot() { return 0; }
inline int this_wave() { return (int)(threadIdx.x >> 6); }

// The DPP forms that sums over lanes use: row_shr 1 .. 15 within rows of 16, row_bcast 15 and 31; ROWS: rows that take part.
template <int CTRL, int ROWS>
inline int add_from(int x) {
  const int lane = threadIdx.x & 63, row = lane >> 4;
  const emulated::Lane& l = emulated::across((uint32_t)x, emulated::kAtOther);
  int from = -1;
  if (CTRL > 0x110 && CTRL < 0x120)
    from = (lane & 15) >= CTRL - 0x110 ? lane - (CTRL - 0x110) : -1;
  else if (CTRL == 0x142)
    from = 16 * row - 1;
  else if (CTRL == 0x143)
    from = row >= 2 ? 31 : -1;
  return (ROWS >> row & 1) && from >= 0 ? x + (int)l.met[from] : x;
}
inline int sum_upto(int x) {
  x = add_from<0x111, 0xF>(x);
  x = add_from<0x112, 0xF>(x);
  x = add_from<0x114, 0xF>(x);
  x = add_from<0x118, 0xF>(x);
  x = add_from<0x142, 0xA>(x);
  return add_from<0x143, 0xC>(x);
}

}  // namespace
}  // namespace pkv
