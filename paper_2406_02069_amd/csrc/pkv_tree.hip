// Attention of drafted tokens over a cache (include/pkv.h: pkv_tree_attention).
//
//   out_t = sum_j 2^(s_tj - m_t) V_j / sum_j 2^(s_tj - m_t)  over the rows j that token t sees, m_t a running reference.
// The T Hq/Hkv query rows of a KV head share its rows of the cache: the more of them, the more products for each byte.  Up to 32 rows
// HBM bounds (decode_long_kernel, which is described in pkv_decode_long.hip: 8 tokens of 32/8 heads, d 128, behind 100k rows 93 us, 4.4
// TB/s); from there on feeding the matrix pipe does (tree_wide_kernel: 16 tokens 88 us, 64 147, 128 258; whole calls, one after the other).
// In both only the steps that hold drafted tokens look at the tree: 32 of its bits are one word, shifted to the step.
//
// tree_wide_kernel: a workgroup is 128 query rows of a KV head x a range of its cache, a wave 32 of the rows against all keys of the
// range, 32 at a time.  What a wave of decode_long_kernel reads for 16 rows serves 128 here: 64 tokens took 439 us there, 209 at once
// with this split.
//   loads   K and V straight into LDS, 8 rows of a step by each wave, two steps ahead in three buffers; a step waits for its own loads
//           only and for the other waves once.  Rows of a page have one base where pages are of 8 k rows (page size 1: 179 us for the
//           64 tokens); page numbers and positions come the same way, for eight steps at a time.
//   scores  S^T = K Q^T in v_mfma_f32_32x32x16: 32 keys are the rows of A, 32 query rows the columns of B, which stay in registers.
//           Lane (col, half) ends with 16 keys of row col.
//   softmax the reference moves when a score exceeds it by 2^6.
//   values  O^T += V^T P^T, V read column-wise.  The weights are rounded to the type once.  decode_long_kernel's second product for what
//           the rounding left would be 24 products a step at d 128 in place of 16, and the vector work that forms its operand: 9, 32, 64 and
//           128 tokens behind 100k rows 86, 97, 147 and 258 us as it is, 94, 112, 184 and 335 with it; 8 sequences of 26 tokens and up to
//           5000 kept rows 53 and 57.  The error of a result, relative to its size, is 2.3e-3 (64 bf16 tokens) and 2.3e-4
//           (26 fp16 tokens), where rounding the result alone makes 1.7e-3 and 2.0e-4.
// What is left at 64 tokens behind 100k rows (139 us at 2.0 GHz; 178 where it is called again and again under a profiler, at 1.6 GHz; 9 in
// the join of 512 ranges' results, 33 MB): vector instructions are issued in 43 % of the cycles, the matrix pipe is busy in 40 %, LDS in
// 20 % without conflicts, and a wave waits for loads, the barrier or a product for 38 % of its time: two waves a SIMD do not fill one
// another's gaps.  With biases and kept positions (8 sequences of 26 tokens: 46 us + 7.6) waves wait 57 % of their time, 31 % is vector issue.
#include <type_traits>

#include "pkv_long.h"
#include "pkv_lds.h"

namespace pkv {
namespace {

// load_to_lds from a lane's own address: rows of a cache in pages lie anywhere.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (as there)
__device__ __forceinline__ void load_to_lds(const char* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(to), "v"(from) : "memory", "m0");
}
// The same of 4 bytes.
__device__ __forceinline__ void word_to_lds(const int32_t* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(to), "v"(from) : "memory", "m0");
}
#pragma clang diagnostic pop

constexpr int kBuffers = 3;  // of a step's keys and values
constexpr int kSlots = 4;    // of what is known of a step: from two steps before it on
constexpr int kAhead = 8;    // steps whose page numbers and positions are requested at a time

// Workgroups of a compute unit.  d 128: three would fit LDS, with 168 registers a lane, and 9 - 32 tokens behind 100k rows take 94 - 111
// us then, 84 - 97 with two (ranges' results are a third fewer); 64 tokens 147 and 150.  d 64: 16 tokens 26.1 with three, 28.0 with two.
template <int D>
constexpr int wide_per_unit() { return D == 128 ? 2 : 3; }
// MODE 1: scores are capped or biased.
template <typename T, int D, int MODE>
__global__ __launch_bounds__(256, (wide_per_unit<D>())) void tree_wide_kernel(const TreeWideArgs a) {
  constexpr int STEPS = D / 16, MB = D / 32, PIECES = D / 8, ROWS_PER_LOAD = 64 / PIECES, ROWS = group_rows<TreeWideArgs>();
  constexpr int OWN = kTile / 4, LOADS = OWN / ROWS_PER_LOAD;  // rows of a step that a wave fetches, loads of K (and of V) for them
  constexpr int ROW = D * 2, BUF = kTile * ROW;
  constexpr float SHIFT = Weight<T>::HALF ? kWideShift : 0.0f;
  __shared__ __align__(1024) char lds[kBuffers * 2 * BUF];  // [buffer][K, V]
  __shared__ int16_t lds_depth[kMostDrafted];
  __shared__ __align__(16) int32_t lds_pos[2][4][kAhead][OWN];  // [step / kAhead % 2][rows' wave][step % kAhead]: given positions
  __shared__ __align__(16) int32_t lds_own_pos[MODE == 1 ? 4 : 1][kTile];  // [wave]: positions that are worked out
  __shared__ int32_t lds_pages[4][2][kAhead * 4];               // [wave][step / kAhead % 2][step % kAhead, rows' wave]: pages of eight rows
  __shared__ int32_t lds_page[4][2][OWN];                       // [wave][step % 2]: of each row that the wave fetches
  __shared__ uint32_t lds_seen[kSlots];                         // [step % kSlots]: rows on pages that exist, a byte of each wave
  __shared__ int32_t lds_span[4][2];
  __shared__ int lds_zeroed;  // whether a value of V that is not finite was put to zero
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const uint32_t pos_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds_pos;
  const uint32_t pages_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds_pages;
  const uint32_t page_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds_page;
  const int lane = threadIdx.x & 63, wave = this_wave(), col = lane & 31, half = lane >> 5;

  // Workgroups that follow one another take different KV heads, then the tiles of rows that read the same keys.
  int b, ranges, per, k;
  Tiles tl;
  if (!a.by_length) {
    ranges = max(a.ranges, 1);
    b = blockIdx.x / (a.units * ranges);
    k = blockIdx.x % (a.units * ranges);
    tl = tiles_of(a, b);
    per = (tl.count + ranges - 1) / ranges;
  } else {
    const Place p = a.B <= 64 ? place_of_workgroup<1>(a, blockIdx.x, lane) : place_of_workgroup<kLaneSequences>(a, blockIdx.x, lane);
    if (p.b < 0) return;
    b = p.b;
    ranges = p.ranges;
    per = p.per;
    k = (int)blockIdx.x - p.base;
    tl = p.tl;
  }
  const int unit = k % a.units, range = k / a.units, g = unit % a.Hkv, tile = unit / a.Hkv;
  const int n = tl.n, past = tl.q_pos;
  int step = tl.first + range * per;
  const int step_end = tl.first + min((range + 1) * per, tl.count);

  const int row = ROWS * tile + 32 * wave + col;  // of those that share the KV head
  const int t = row < a.G ? row / a.heads : 0, h = g * a.heads + (row < a.G ? row % a.heads : 0);
  const int drafted = a.new_lens ? min(max(a.new_lens[b], 0), a.T) : a.T;
  const bool there = row < a.G && t < drafted, wave_there = __any(there);
  const bool placed = a.positions || a.window || (MODE == 1 && a.slopes);  // positions matter
  if (ROWS * tile >= drafted * a.heads) step = step_end;  // no row is there
  const int step_begin = step;

  // What is known of the query rows is requested here, what the first steps' rows are behind it, and waited for together.
  u32x4 qf[STEPS];
  {
    const uint16_t* qp = a.q + b * a.q_sb + h * a.q_sh + t * a.q_st + 8 * half;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) qf[i] = there ? *reinterpret_cast<const u32x4*>(qp + 16 * i) : (u32x4)(0);
  }
  float slope = MODE == 1 && a.slopes ? a.slopes[h] * kLog2e : 0.0f;
  int32_t p_row = placed && a.q_pos ? a.q_pos[(int64_t)b * a.T + t] : 0;

  const uint32_t row_bytes = (uint32_t)(a.page_size ? D : a.c_st) * 2;
  const int64_t base = a.page_size ? 0 : (b * a.c_sb + g * a.c_sh) * 2;
  const char* const Kb = reinterpret_cast<const char*>(a.K) + base;
  const char* const Vb = reinterpret_cast<const char*>(a.V) + base;
  const int32_t* const table = a.table + (int64_t)b * a.max_pages;
  const int32_t* const pos_b = a.positions + b * a.p_sb + g * a.p_sh;

  // Fetching a step: wave w rows 8 w .. 8 w + 7 of K and of V, a row's pieces swapped.  Page numbers, and positions that are given, come
  // through LDS like the rows themselves, for eight steps at a time: were they loaded into registers, their first use would wait for all
  // that has been requested since.  Eight rows in a row of a page, or of a compact cache, have one base; where pages end inside of eight
  // rows, each row is looked up, a step at a time.  Rows behind the last one are taken as the last, those on pages that do not exist as
  // the cache's first.
  const bool odd_pages = a.page_size % OWN != 0;
  auto page_of = [&](int j) {
    uint32_t p = __umulhi((uint32_t)j, a.page_magic);
    if ((uint32_t)j - p * a.page_size >= (uint32_t)a.page_size) ++p;
    return p;
  };
  auto look_ahead = [&](int block) {
    const uint32_t slot = block & 1;
    if (a.positions) {
      const int j = min((block * kAhead + lane / OWN) * kTile + OWN * wave + lane % OWN, n - 1);
      word_to_lds(pos_b + j, pos_base + (slot * 4 + wave) * (64 * 4));
    }
    if (a.page_size && !odd_pages && lane < kAhead * 4) {
      const int j = min((block * kAhead + lane / 4) * kTile + OWN * (lane % 4), n - 1);
      word_to_lds(table + page_of(j), pages_base + (wave * 2 + slot) * (kAhead * 4 * 4));
    }
  };
  auto look = [&](int st) {
    if (odd_pages && lane < OWN) word_to_lds(table + page_of(min(st * kTile + OWN * wave + lane, n - 1)), page_base + (wave * 2 + (st & 1)) * (OWN * 4));
  };
  int32_t pages = 0;       // of the block of steps that is fetched, lane 4 i + w: step i, wave w's rows
  uint32_t pages_are = 0;  // which of them exist
  auto take_pages = [&](int block) {
    if (a.page_size && !odd_pages) {
      pages = lds_pages[wave][block & 1][lane % (kAhead * 4)];
      pages_are = (uint32_t)__ballot((uint32_t)pages < (uint32_t)a.num_pages);
    }
  };
  // (returns which of the step's rows are on pages that exist, where pages do not end inside of eight)
  auto fetch = [&](int st, int buf, auto plain) {
    constexpr bool PLAIN = decltype(plain)::value;  // (known beforehand: neither odd pages nor wide rows)
    const uint32_t to = lds_base + buf * 2 * BUF + OWN * wave * ROW;
    uint32_t is = ~0u;
    int id = lane;
    asm("" : "+v"(id));  // (what follows from it is not kept in registers, which are short)
    if (PLAIN || !odd_pages) {
      const int j0 = min(st * kTile + OWN * wave, (n - 1) / OWN * OWN), most = n - 1 - j0;
      uint64_t row0 = (uint32_t)j0;
      if (a.page_size) {
        const int at = st % kAhead * 4;
        const uint32_t page = (uint32_t)__builtin_amdgcn_readlane(pages, at + wave), own = pages_are >> at & 15;
        is = (own & 1) * 0xFF | (own >> 1 & 1) * 0xFF00 | (own >> 2 & 1) * 0xFF0000 | (own >> 3) * 0xFF000000;
        row0 = own >> wave & 1 ? (page * a.Hkv + g) * a.page_size + ((uint32_t)j0 - page_of(j0) * a.page_size) : 0;
      }
      const char *const Kr = Kb + row0 * row_bytes, *const Vr = Vb + row0 * row_bytes;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int r = i * ROWS_PER_LOAD + id / PIECES, piece = id % PIECES;
        const uint32_t in_k = 16 * (piece ^ swizzle_k<D>(OWN * wave + r)), in_v = 16 * (piece ^ swizzle_v<D>(OWN * wave + r));
        if (PLAIN || row_bytes <= 1u << 26) {
          const uint32_t at = min(r, most) * row_bytes;
          load_to_lds(Kr, at + in_k, to + i * 1024);
          load_to_lds(Vr, at + in_v, to + i * 1024 + BUF);
        } else {
          const uint64_t at = (uint64_t)min(r, most) * row_bytes;
          load_to_lds(Kr + at + in_k, to + i * 1024);
          load_to_lds(Vr + at + in_v, to + i * 1024 + BUF);
        }
      }
    } else {
      const int j0 = st * kTile + OWN * wave;
      uint32_t there8 = 0;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int r = i * ROWS_PER_LOAD + id / PIECES, piece = id % PIECES, j = min(j0 + r, n - 1);
        const uint32_t page = (uint32_t)lds_page[wave][st & 1][r];
        const bool exists = page < (uint32_t)a.num_pages;
        const uint64_t row = exists ? (page * a.Hkv + g) * a.page_size + ((uint32_t)j - page_of(j) * a.page_size) : 0;
        const uint64_t is64 = __ballot(exists);
#pragma unroll
        for (int x = 0; x < ROWS_PER_LOAD; ++x) there8 |= (uint32_t)(is64 >> (x * PIECES) & 1) << (i * ROWS_PER_LOAD + x);
        load_to_lds(Kb + row * row_bytes + 16 * (piece ^ swizzle_k<D>(OWN * wave + r)), to + i * 1024);
        load_to_lds(Vb + row * row_bytes + 16 * (piece ^ swizzle_v<D>(OWN * wave + r)), to + i * 1024 + BUF);
      }
      if (lane == 0) reinterpret_cast<uint8_t*>(&lds_seen[st % kSlots])[wave] = (uint8_t)there8;
    }
    return is;
  };
  // Behind the barrier of the step before (by which all waves have made the step's fetch known): a step's rows that are there, one bit
  // each, and the position of row l % 32.  `is`: what fetch returned.
  auto rows_there = [&](int st, uint32_t is, int32_t& pos) {
    const int left = n - st * kTile;
    if (left < kTile) is &= (1u << left) - 1;
    if (odd_pages) is &= (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_seen[st % kSlots]);
    const int j = st * kTile + col;
    pos = j;
    if (a.positions) {
      pos = lds_pos[st / kAhead & 1][col / OWN][st % kAhead][col % OWN];
      is &= (uint32_t)__ballot(pos >= 0);
    } else if (placed && st * kTile + kTile > past && j >= past) {
      pos = past + lds_depth[min(j - past, a.T - 1)];
    }
    return is;
  };
  // Two steps are on their way while a third is worked on.
  uint32_t is_now = 0, is_next = 0, is_then = 0;
  if (step < step_end) {
    look_ahead(step / kAhead);
    look_ahead(step / kAhead + 1);
    look(step);
    look(step + 1);
  }
  if (placed && !a.q_pos) {
    for (int i = threadIdx.x; i < a.T; i += 256) lds_depth[i] = (int16_t)ancestors(a, b, i, drafted);
    __syncthreads();
    p_row = past + lds_depth[t];
  }
  wait_loads();
#pragma unroll
  for (int i = 0; i < STEPS; ++i) asm volatile("" : "+v"(qf[i]));  // (they are waited for here, and not by every step's products)
  asm volatile("" : "+v"(slope), "+v"(p_row));
  if (step < step_end) {
    take_pages(step / kAhead);
    is_now = fetch(step, 0, std::false_type());
    look(step + 2);
    if (step + 1 < step_end) {
      if ((step + 1) % kAhead == 0) take_pages((step + 1) / kAhead);
      is_next = fetch(step + 1, 1, std::false_type());
    }
  }
  // the least and the greatest position of the wave's rows, and of the workgroup's
  const int32_t w_min = ~wave_max(there ? ~p_row : INT32_MIN), w_max = wave_max(there ? p_row : INT32_MIN);
  if (lane == 0) {
    lds_span[wave][0] = w_min;
    lds_span[wave][1] = w_max;
    if (wave == 0) lds_zeroed = 0;
  }
  lds_barrier();
  const int32_t g_min = min(min(lds_span[0][0], lds_span[1][0]), min(lds_span[2][0], lds_span[3][0]));
  const int32_t g_max = max(max(lds_span[0][1], lds_span[1][1]), max(lds_span[2][1], lds_span[3][1]));
  // Whether rows whose positions are from least to greatest see all rows of a step that are there.
  auto whole = [&](int st, uint32_t now, int32_t pos_now, int32_t least, int32_t greatest) {
    const int off = st * kTile - past;
    if (off + kTile > 0) return false;
    if (!a.positions && !a.window) return true;
    const bool all = pos_now <= least && (!a.window || (int64_t)pos_now > (int64_t)greatest - a.window);
    return (now & ~(uint32_t)__ballot(all)) == 0;
  };
  // Of the rows that are there, those that the own row sees.
  auto visible = [&](int st, uint32_t now, int32_t pos_now) {
    const int off = st * kTile - past;
    uint32_t mine = now;
    if (off + kTile > 0) mine &= drafted_seen(a, b, t, off);
    if (a.positions || a.window) {
      const bool before = off + col < 0;
      const bool all = (!before || pos_now <= w_min) && (!a.window || (int64_t)pos_now > (int64_t)w_max - a.window);
      for (uint32_t left = now & ~(uint32_t)__ballot(all); left != 0; left &= left - 1) {
        const int i = __builtin_ctz(left);
        const int32_t kp = __builtin_amdgcn_readlane(pos_now, i);
        if ((off + i < 0 && kp > p_row) || (a.window && (int64_t)kp <= (int64_t)p_row - a.window)) mine &= ~(1u << i);
      }
    }
    return there ? mine : now;
  };

  float m = kNone, z = 0.0f;
  bool large = false;  // some reference is beyond kLarge
  f32x16 o[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) o[i] = (f32x16)(0.0f);

  // Places in a step's rows, as in pkv_prefill.hip.
  const int k_at = col * ROW + ((half ^ swizzle_k<D>(col)) << 4);
  const int v_row = 4 * half + ((lane & 15) >> 2), v_piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const int v_at = v_row * ROW + ((v_piece ^ swizzle_v<D>(v_row)) << 4) + 8 * (lane & 1);

  // `inner`: the step lies in the past, rows are told apart by pages that do not exist at most, and fetch is plain.
  auto one_step = [&](auto buffer, auto inner) {
    constexpr int buf = decltype(buffer)::value;
    constexpr bool INNER = decltype(inner)::value;
    const char* const Kl = lds + buf * 2 * BUF;
    char* const Vl = lds + buf * 2 * BUF + BUF;
    if (INNER || step + 1 < step_end)  // (the last of the inner steps has one behind it)
      wait_loads<2 * LOADS>();         // (those of the next step)
    else
      wait_loads();
    int32_t pos_now = 0;
    const uint32_t now = INNER ? is_now : rows_there(step, is_now, pos_now);
    const bool all = now == ~0u && (INNER || whole(step, now, pos_now, g_min, g_max));  // every row of the workgroup sees all of the step
    if (!all) {
      // values of V that are not finite would spoil the product with a weight of 0: each wave those that it fetched
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        u32x4* const mine = reinterpret_cast<u32x4*>(Vl + (OWN * wave + i * ROWS_PER_LOAD) * ROW + 16 * lane);
        u32x4 v = *mine;
        uint32_t any = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t nf = not_finite<T>(v[x]);
          any |= nf;
          v[x] &= ~((nf >> 15) * 0xFFFFu);
        }
        if (any) {
          *mine = v;
          lds_zeroed = 1;
        }
      }
    }
    lds_barrier();
    f32x16 sc;
    if (wave_there) {
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const u32x4 kf = *reinterpret_cast<const u32x4*>(Kl + (k_at ^ (i << 5)));
        sc = Elem<T>::mfma32(kf, qf[i], i == 0 ? (f32x16)(0.0f) : sc);
      }
    }
    if (step + 2 < step_end) {  // (beside the products)
      if (step % kAhead == 0 && step != step_begin) look_ahead(step / kAhead + 1);
      if (!INNER) look(step + 3);
      if ((step + 2) % kAhead == 0) take_pages((step + 2) / kAhead);
      is_then = fetch(step + 2, (buf + 2) % kBuffers, inner);
    }
    is_now = is_next;
    is_next = is_then;
    if (!wave_there) return;
    if constexpr (MODE == 1) {
      if (a.cap.cap != 0.0f) {
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = sc[e];
        cap_scores(x, a.cap);
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = x[e];
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] *= a.scale;
      }
      if (INNER && a.slopes) {
        const float far = (float)(p_row - step * kTile - 4 * half);
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = fmaf(-slope, far - (float)key_of(e), sc[e]);
      } else if (a.slopes) {
        if (!a.positions) {
          if (lane < kTile) lds_own_pos[wave][lane] = pos_now;
          own_lds_order();
        }
        const int32_t* const at = a.positions ? lds_pos[step / kAhead & 1][0][step % kAhead] : lds_own_pos[wave];
        const int next = a.positions ? kAhead * OWN : OWN;  // from one wave's rows to the next one's
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const u32x4 kp = *reinterpret_cast<const u32x4*>(&at[x * next + 4 * half]);
          if (all) {  // (positions up to the row's own)
#pragma unroll
            for (int y = 0; y < 4; ++y) sc[4 * x + y] = fmaf(-slope, (float)((uint32_t)p_row - kp[y]), sc[4 * x + y]);
          } else {
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const uint32_t d = (uint32_t)p_row - kp[y];
              sc[4 * x + y] = fmaf(-slope, (float)((int32_t)kp[y] > p_row ? 0u - d : d), sc[4 * x + y]);
            }
          }
        }
        own_lds_order();
      }
    }
    if (!all && (now != ~0u || !whole(step, now, pos_now, w_min, w_max))) {
      const uint32_t mine = (INNER ? now : visible(step, now, pos_now)) >> (4 * half);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!(mine & (1u << key_of(e)))) sc[e] = kNone;
    }
    const float f1 = MODE == 1 ? 1.0f : a.scale;
    float top = sc[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, sc[e]);
    top *= f1;
    if (__any(top - m > 6.0f)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m1 = fmaxf(m, top);
      const float f = m1 == kNone ? 1.0f : exp2_(m - m1);
      m = m1;
      z *= f;
#pragma unroll
      for (int i = 0; i < MB; ++i) o[i] *= f;
      large = __any(m != kNone && fabsf(m) > kLarge);
    }
    float ref = (m == kNone ? 0.0f : m) - SHIFT, factor = f1;
    if (__builtin_expect(large, 0)) {
#pragma clang fp contract(off)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[e] = (sc[e] * f1 - (m == kNone ? 0.0f : m)) + SHIFT;
      ref = 0.0f;
      factor = 1.0f;
    }
    u32x4 pf[2];
    float z0 = 0.0f, z1 = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const float p0 = exp2_(fmaf(sc[e], factor, -ref)), p1 = exp2_(fmaf(sc[e + 1], factor, -ref));
      z0 += p0;
      z1 += p1;
      pf[e >> 3][(e >> 1) & 3] = pack2<T>(p0, p1);
    }
    z += z0 + z1;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        const char* const from = Vl + (v_at ^ (mb << 6)) + 16 * ks * ROW;
        const u32x2 x = read_columns(from), y = read_columns(from + 8 * ROW);
        const u32x4 vf = {x[0], x[1], y[0], y[1]};
        o[mb] = Elem<T>::mfma32(vf, pf[ks], o[mb]);
      }
    }
  };
  // The inner steps three at a time, so that the others begin with the first buffer again.
  const int inner_end = a.positions || a.window || odd_pages || row_bytes > 1u << 26 ? step : min(step_end - 1, past / kTile);
  while (step + 3 <= inner_end) {
    one_step(std::integral_constant<int, 0>(), std::true_type());
    ++step;
    one_step(std::integral_constant<int, 1>(), std::true_type());
    ++step;
    one_step(std::integral_constant<int, 2>(), std::true_type());
    ++step;
  }
  while (step < step_end) {
    one_step(std::integral_constant<int, 0>(), std::false_type());
    if (++step >= step_end) break;
    one_step(std::integral_constant<int, 1>(), std::false_type());
    if (++step >= step_end) break;
    one_step(std::integral_constant<int, 2>(), std::false_type());
    ++step;
  }

  if (!there)  // (0 times what is not finite)
#pragma unroll
    for (int i = 0; i < MB; ++i) o[i] = (f32x16)(0.0f);
  f32x4 naught = (f32x4)(0.0f);  // of what is finite; otherwise NaN
#pragma unroll
  for (int x = 0; x < MB * 16; ++x) naught[x & 3] = fmaf(o[x >> 4][x & 15], 0.0f, naught[x & 3]);
  const bool odd = lds_zeroed != 0 || (naught[0] + naught[1]) + (naught[2] + naught[3]) != 0.0f;
  if (__builtin_expect(__any(odd) && wave_there, 0)) {
    // Values of V that are not finite: where a row sees some, its element is their sum (every weight is positive).
    f32x16 extra[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) extra[i] = (f32x16)(0.0f);
#pragma unroll 1
    for (int st = step_begin; st < step_end; ++st) {
      const int j = min(st * kTile + col, n - 1);
      uint32_t at = (uint32_t)j, left = 0;  // `left`: rows with such values
      int32_t pos = a.positions ? pos_b[j] : placed && j >= past ? past + lds_depth[min(j - past, a.T - 1)] : j;
      bool is = st * kTile + col < n && (!a.positions || pos >= 0);
      if (a.page_size) {
        const uint32_t p = page_of(j), page = (uint32_t)table[p];
        is = is && page < (uint32_t)a.num_pages;
        at = (page * a.Hkv + g) * a.page_size + ((uint32_t)j - p * a.page_size);
      }
      at = is ? at : 0;
      const uint32_t seen = (uint32_t)__ballot(is);
#pragma unroll 1
      for (int r0 = 0; r0 < kTile; r0 += ROWS_PER_LOAD) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(Vb + (uint64_t)(uint32_t)__shfl((int)at, r0 + lane / PIECES) * row_bytes + 16 * (lane % PIECES));
        const uint64_t some = __ballot((not_finite<T>(v[0]) | not_finite<T>(v[1]) | not_finite<T>(v[2]) | not_finite<T>(v[3])) != 0);
#pragma unroll
        for (int r = 0; r < ROWS_PER_LOAD; ++r) left |= (some >> (r * PIECES) & (((uint64_t)1 << PIECES) - 1)) != 0 ? 1u << (r0 + r) : 0u;
      }
      left &= seen;
      if (left == 0) continue;
      const uint32_t mine = there ? visible(st, seen, pos) : 0u;
#pragma unroll 1
      for (; left != 0; left &= left - 1) {
        const int i = __builtin_ctz(left);
        const char* const from = Vb + (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)at, i) * row_bytes + 8 * half;
        const bool sees = mine >> i & 1;
#pragma unroll
        for (int x = 0; x < MB * 4; ++x) {
          const u32x2 u = *reinterpret_cast<const u32x2*>(from + 16 * x);
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float e = unpack<T>(u[y >> 1], y & 1);
            extra[x >> 2][4 * (x & 3) + y] += sees && !(fabsf(e) < __builtin_inff()) ? e : 0.0f;
          }
        }
      }
    }
#pragma unroll
    for (int x = 0; x < MB * 16; ++x) o[x >> 4][x & 15] = extra[x >> 4][x & 15] == 0.0f ? o[x >> 4][x & 15] : extra[x >> 4][x & 15];
  }

  z += __shfl_xor(z, 32);
  int id = threadIdx.x;
  asm("" : "+v"(id));
  const int end_local = 32 * (id >> 6) + (id & 31), end_row = ROWS * tile + end_local, end_half = (id >> 5) & 1;
  if (end_row >= a.G) return;
  if (!there) {
    m = kNone;
    z = 0.0f;
  }
  if (ranges > 1) {
    const int64_t to = (int64_t)blockIdx.x * ROWS + end_local;
    float* const po = a.part_o + to * D + 4 * end_half;
#pragma unroll
    for (int x = 0; x < MB * 4; ++x) {
      f32x4 v;
#pragma unroll
      for (int y = 0; y < 4; ++y) v[y] = o[x >> 2][4 * (x & 3) + y];
      *reinterpret_cast<f32x4*>(po + 8 * x) = v;
    }
    if (end_half == 0) {
      a.part_mz[to * 2] = m;
      a.part_mz[to * 2 + 1] = z;
    }
    return;
  }
  const float inv = z == 0.0f ? 0.0f : 1.0f / z;
  uint16_t* const op = a.out + out_at(a, b, g, end_row, D) + 4 * end_half;
#pragma unroll
  for (int x = 0; x < MB * 4; ++x) {
    u32x2 w;
    w[0] = pack2<T>(o[x >> 2][4 * (x & 3)] * inv, o[x >> 2][4 * (x & 3) + 1] * inv);
    w[1] = pack2<T>(o[x >> 2][4 * (x & 3) + 2] * inv, o[x >> 2][4 * (x & 3) + 3] * inv);
    *reinterpret_cast<u32x2*>(op + 8 * x) = w;
  }
  if (a.lse && end_half == 0) a.lse[lse_at(a, b, g, end_row)] = z == 0.0f ? kNone : (m - SHIFT + log2_(z)) * kLn2;
}

constexpr int kFewJoined = 128;  // workgroups, and below decode_long_join_kernel
// Ranges' results of many rows, joined: a row of them for every D / 4 threads, eight ranges at a time, with nothing to wait for but
// loads.  32/8 heads, d 128, pages: 64 sequences of 16 tokens behind 2000 rows 126 us, by decode_long_join_kernel, whose workgroups share
// out a row's ranges and meet, 151; 8 of 26 behind 5000 (28/4 heads) 36.7 and 41.4.  With fewer workgroups than compute units the many
// ranges of a long cache bound it: behind 100k rows 16 tokens 91 and 87.7, 32 (128 workgroups) 95.7 and 96; behind 4000 rows 22 either way.
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_join_kernel(const TreeWideArgs a, int chunks) {
  constexpr int ROWS = group_rows<TreeWideArgs>(), AT_ONCE = 8;
  constexpr float UNIT = Weight<T>::HALF ? 1.0f / (1 << kWideShift) : 1.0f;
  const int b = blockIdx.x / chunks;
  int ranges = a.ranges, base = b * a.units * a.ranges;
  if (a.by_length) {
    const int lane = threadIdx.x & 63;
    const Place p = a.B <= 64 ? place_of_sequence<1>(a, b, lane) : place_of_sequence<kLaneSequences>(a, b, lane);
    ranges = p.ranges;
    base = p.base;
  }
  const int h = (int)(blockIdx.x % chunks) * (256 / (D / 4)) + threadIdx.x / (D / 4), d4 = threadIdx.x % (D / 4);
  if (ranges == 1 || h >= a.Hq) return;  // (written already)
  const int h_in = h % a.G, g = h / a.G;
  const int64_t at = ((int64_t)base + h_in / ROWS * a.Hkv + g) * ROWS + h_in % ROWS, step = (int64_t)ROWS * a.units;
  float m = kNone, z = 0.0f;
  f32x4 acc = (f32x4)(0.0f);
  for (int i0 = 0; i0 < ranges; i0 += AT_ONCE) {
    float m1[AT_ONCE], z1[AT_ONCE];
    f32x4 v[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {  // (ranges behind the last one: that one, without weight)
      const int64_t from = at + step * min(i0 + k, ranges - 1);
      m1[k] = a.part_mz[from * 2];
      z1[k] = a.part_mz[from * 2 + 1];
      v[k] = *reinterpret_cast<const f32x4*>(a.part_o + from * D + 4 * d4);
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) top = fmaxf(top, m1[k]);
    const float ref = top == kNone ? 0.0f : top, f0 = exp2_(m - ref);
    m = top;
    z *= f0;
    acc *= f0;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const float f1 = i0 + k < ranges ? exp2_(m1[k] - ref) : 0.0f;
      z = fmaf(z1[k], f1, z);
      acc = __builtin_elementwise_fma(v[k], (f32x4)(f1), acc);
    }
  }
  if (__builtin_expect(!finite(acc), 0)) {  // (0 times an infinity is not what it should be)
    acc = (f32x4)(0.0f);
    const float ref = m == kNone ? 0.0f : m;
#pragma unroll 1
    for (int i = 0; i < ranges; ++i)
      acc = weighed(acc, 1.0f, *reinterpret_cast<const f32x4*>(a.part_o + (at + step * i) * D + 4 * d4), exp2_(a.part_mz[(at + step * i) * 2] - ref));
  }
  const float inv = z == 0.0f ? 0.0f : 1.0f / z;
  u32x2 w;
  w[0] = pack2<T>(acc[0] * inv, acc[1] * inv);
  w[1] = pack2<T>(acc[2] * inv, acc[3] * inv);
  *reinterpret_cast<u32x2*>(a.out + out_at(a, b, g, h_in, D) + 4 * d4) = w;
  if (d4 == 0 && a.lse) a.lse[lse_at(a, b, g, h_in)] = z == 0.0f ? kNone : (m + log2_(z * UNIT)) * kLn2;
}

template <typename T, int D>
hipError_t launch_wide(const TreeWideArgs& a, int64_t workgroups, hipStream_t s) {
  if (a.cap.cap != 0.0f || a.slopes)
    hipLaunchKernelGGL((tree_wide_kernel<T, D, 1>), dim3((unsigned)workgroups), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((tree_wide_kernel<T, D, 0>), dim3((unsigned)workgroups), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.ranges == 0) return e;
  const int chunks = (a.Hq + 1024 / D - 1) / (1024 / D);
  if ((int64_t)a.B * chunks < kFewJoined) {
    hipLaunchKernelGGL((decode_long_join_kernel<T, D, 1, TreeWideArgs>), dim3((unsigned)(a.B * a.Hq)), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((tree_join_kernel<T, D>), dim3((unsigned)(a.B * chunks)), dim3(256), 0, s, a, chunks);
  }
  return hipGetLastError();
}

// More than kFewRows query rows a KV head: the kernel above.  32/8 heads, d 128, behind 100k rows: 32 rows 91 us in decode_long_kernel,
// 36 rows 84 here, 64 rows 127 there and 87 here.  Behind 4000 rows the two are 2 us apart.
constexpr int kFewRows = 32;
bool wide(const pkv_tree_desc& d) { return (int64_t)d.T * (d.Hq / d.Hkv) > kFewRows; }

// As grid_of of pkv_long.h, in workgroups of 128 rows, of which the device holds wide_per_unit per compute unit.
int wide_turn(const pkv_tree_desc& d) { return d.d == 128 ? 512 : 768; }
Grid wide_grid(const pkv_tree_desc& d, int turn) {
  constexpr int ROWS = group_rows<TreeWideArgs>();
  const int64_t units = d.Hkv * (((int64_t)d.T * (d.Hq / d.Hkv) + ROWS - 1) / ROWS), all = d.B * units;
  if (d.k_cap <= kLeastWide * kTile) return {all, 0, 0};
  if (d.B > 1 && d.B <= kFlatBatch && (int64_t)d.B * d.k_cap <= (int64_t)1 << 36) {
    const int64_t share = all <= turn / 2 ? turn : 2 * turn;
    return all >= 2 * turn && (d.k_cap <= kWhole || all > kMostUnits) ? Grid{all, 0, 0} : Grid{share + all, (int32_t)share, 1};
  }
  int64_t S = turn / all;
  const int64_t most = ((int64_t)d.k_cap + kLeastWide * kTile - 1) / (kLeastWide * kTile);
  if (S > most) S = most;
  return S <= 1 ? Grid{all, 0, 0} : Grid{all * S, (int32_t)S, 0};
}
size_t wide_bytes(const Grid& g, int d) { return g.ranges == 0 ? 0 : (size_t)g.workgroups * group_rows<TreeWideArgs>() * (d + 2) * sizeof(float); }

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
  if (wide(*desc)) return wide_bytes(wide_grid(*desc, wide_turn(*desc)), desc->d);
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
  if (!apart(d.d, {{d.B, d.o_sb}, {d.Hq, d.o_sh}, {d.T, d.o_st}})) return PKV_ERR_INVALID_ARG;
  const size_t need = pkv_tree_workspace_bytes(desc);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return PKV_ERR_WORKSPACE;
  TreeWideArgs a;
  memset(&a, 0, sizeof(a));
  const bool many = wide(d);
  const Grid grid = many ? wide_grid(d, wide_turn(d)) : grid_of(d);
  fill_long(a, d, grid, d.T * (d.Hq / d.Hkv), q, K_cache, V_cache, out, workspace);
  a.table = block_table; a.count = count; a.positions = positions; a.q_pos = q_pos; a.slopes = slopes;
  a.new_lens = new_lens; a.tree = tree;
  a.lse = lse_out;
  a.window = d.window;
  a.p_sb = d.p_sb; a.p_sh = d.p_sh;
  a.T = d.T; a.words = (d.T + 31) / 32; a.heads = d.Hq / d.Hkv;
  a.q_st = d.q_st; a.o_sb = d.o_sb; a.o_sh = d.o_sh; a.o_st = d.o_st;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (!many) {
    e = launch_long(static_cast<const TreeArgs&>(a), d.dtype, d.d, grid.workgroups, st);
  } else {
    constexpr int ROWS = group_rows<TreeWideArgs>();
    a.turn = wide_turn(d);
    a.head_groups = (a.G + ROWS - 1) / ROWS;
    a.units = a.Hkv * a.head_groups;
    a.part_mz = a.part_o ? a.part_o + (size_t)grid.workgroups * ROWS * d.d : nullptr;
    if (d.dtype == PKV_BF16)
      e = d.d == 128 ? launch_wide<__bf16, 128>(a, grid.workgroups, st) : launch_wide<__bf16, 64>(a, grid.workgroups, st);
    else
      e = d.d == 128 ? launch_wide<_Float16, 128>(a, grid.workgroups, st) : launch_wide<_Float16, 64>(a, grid.workgroups, st);
  }
  return e == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
