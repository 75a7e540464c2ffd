// Attention of a prompt over its keys (include/pkv.h: pkv_prefill_attention).
//
// Bound by power: 4 d products-and-sums per (query row, seen key), for which K and V come from LDS, and an exponential.  A 32k
// prompt (32 / 8 heads, d 128) takes 7.6 - 8.3 ms by card, 1.06 - 1.17 PFLOP/s of what it sees; the clock sinks to 1.6 GHz, at which
// the matrix pipe is busy for 67 % of the cycles.  Forms that need fewer or more cycles took the same time within 3 %.  Capped and
// biased scores and d 64 are bound by vector issue (73 - 82 % of the cycles, 16k prompts).
// Work split: the G T query rows of a KV head (row = token * G + head, so that a tile of rows covers few tokens and hardly more
// keys than its rows see) in tiles of 128, a workgroup of four waves each, 32 rows a wave; the longest tiles first.  Workgroups
// that follow one another take different KV heads: with eight of them each XCD's cache holds the keys of one.  Few rows: the
// keys of a tile are cut into S ranges, whose un-normalised results a second kernel joins in order; with ragged sequences S and a
// workgroup's place go by their lengths, worked out by every wave from all of them.
//   keys    32 at a time, K and V straight from memory into LDS, double-buffered: the next step's are requested when a step
//           begins, one barrier per step.  With 32 keys three workgroups share a compute unit (168 registers), with 64 two: the
//           third is worth more than half the barriers (32k prompt 8.00 against 8.20 ms, 300 rows of 50k keys 0.34 against 0.36).
//           64 rows a wave halve what is read from LDS, but leave one wave per SIMD: 9.1 ms, and 9.3 with the next step's scores
//           formed beside the softmax.  16-byte pieces of a row are swapped (through the lanes' addresses in memory) so that
//           neither way of reading them meets the same bank twice.
//   scores  S^T = K Q^T in v_mfma_f32_32x32x16: a lane ends with 16 keys of one query row (column), the other half of the wave
//           with the other 16, so that maxima and sums stay in the lane.
//   softmax a reference exponent per row, moved only when a score exceeds it by a factor of 2^6.  The weights are rounded to the
//           type (as the result is: the error against 64 bits grows by 2 - 17 %, of packed fp16 documents by a third), their sum
//           is not.  fp16 weights carry a factor of 2^8, so that the type's last step is 2^-32 of the reference; a factor of 2^13
//           and moves at 2^2 would make it 2^-37 and cost 1 - 7 % (1k prompt 31.4 -> 33.7 us).
//   values  O^T += V^T P^T: the weights are in B's layout already if the 16 keys of a step are taken in the order in which the
//           lanes hold them; V^T is read column-wise.
// Masks leave each row an interval of keys.  Steps that no row of a wave sees are skipped, those that all of its rows see whole
// take no comparisons.  In the others hidden keys have the weight 0; a value that is not finite would still spoil their product,
// so the waves look over the rows that they fetched for such a step and put zeros in LDS for such values.  Where that happened, or
// a result is not finite, the rows of V are looked over once more at the end: every weight is positive, so that an element for which
// a row sees values that are not finite is the sum of those, however small their weights are held.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "pkv_attn.h"
#include "pkv_lds.h"

namespace pkv {
namespace {

constexpr int kRows = 128;   // query rows of a workgroup
constexpr int kKeys = 32;    // keys per step
constexpr int kMaxParts = 64;  // ranges of keys
constexpr int kLeastKeys = 768;  // of a range, about
// References (log2) beyond which a score is rounded before it is compared with them: what one fma of scale and difference finds
// left of a rounded product is as large as a step there, and would be a weight's exponent.
constexpr float kLarge = 0x1p20f;

struct PrefillArgs {
  const uint16_t *q, *K, *V;
  const int32_t *seq_lens, *q_start, *doc_start, *prefix_end;
  const float* slopes;
  uint16_t* out;
  float* lse;
  float* part_o;   // [B * Hkv][T * G][S][d]; by length: [slot][128][d], a slot for each workgroup of a tile in several ranges
  float* part_mz;  // the same with 2 instead of d: reference exponent (log2) and sum
  int32_t B, Hq, Hkv, G, T, N, window, S, tiles;
  int32_t by_length;  // 2 .. 64 ragged sequences: ranges and places by their lengths, in up to so many workgroups
  int32_t most_parts, most_slots, turn;  // then: ranges of a tile, slots, workgroups that the device holds at a time
  int64_t q_sb, q_sh, q_st, kv_sb, kv_sh, kv_st, o_sb, o_sh, o_st;
  float scale;  // of the products, to log2 units (without a cap)
  Cap cap;
};

// What the masks leave a query row: keys lo .. hi (none: lo > hi).
struct Seen {
  int32_t lo, hi, p;
};
__device__ __forceinline__ Seen seen_keys(const PrefillArgs& a, int b, int t, int n) {
  Seen s;
  const int64_t p = (int64_t)(a.q_start ? a.q_start[b] : 0) + t;
  s.p = (int32_t)p;
  s.lo = 1;
  s.hi = 0;
  if (p >= 0 && p < n) {
    int lo = 0, hi = s.p;
    if (a.window) lo = max(lo, s.p - a.window + 1);
    if (a.doc_start) lo = max(lo, a.doc_start[(int64_t)b * a.N + p]);
    if (a.prefix_end) hi = max(hi, max(min(a.prefix_end[(int64_t)b * a.N + p], n), 0) - 1);
    if (lo <= hi) {
      s.lo = lo;
      s.hi = hi;
    }
  }
  return s;
}

__device__ __forceinline__ int wave_max(int x) {
  for (int o = 32; o > 0; o >>= 1) x = max(x, __shfl_xor(x, o));
  return __builtin_amdgcn_readfirstlane(x);
}

// The sequences' shares of a call by their lengths, lane b's for sequence b: its tiles first .. first + act - 1 have rows that are
// there, each in S ranges of keys; its workgroups, slots and tiles in several ranges go before `end`, `slots` and `cut`.
// Ranges are as long as make one turn of the device of all work where the tiles alone are half of one at most, else two turns.
struct Shares {
  int first, act, S;
  int all, slots, cut;     // own numbers
  int all_upto, slots_upto, cut_upto;
};
__device__ __forceinline__ int last_of(int upto) { return __builtin_amdgcn_readlane(upto, 63); }
__device__ __forceinline__ Shares shares_of(const PrefillArgs& a, int lane) {
#pragma clang fp contract(off)  // (the join has to come to the same numbers)
  Shares s = {0, 0, 1, 0, 0, 0, 0, 0, 0};
  const int b = min(lane, a.B - 1);
  const int n = a.seq_lens ? min(max(a.seq_lens[b], 0), a.N) : a.N;
  const int64_t start = a.q_start ? a.q_start[b] : 0;
  const int t0 = (int)min(max(-start, (int64_t)0), (int64_t)a.T), t1 = (int)min(max(n - start, (int64_t)t0), (int64_t)a.T);
  float steps = 0.0f;  // of a tile, in the mean (an estimate: documents are not looked at)
  int most = 1;
  if (t1 > t0 && lane < a.B) {
    s.first = t0 * a.G / kRows;
    s.act = (t1 * a.G + kRows - 1) / kRows - s.first;
    int lo = (int)(start + t0) + 1, hi = (int)(start + t1);
    if (a.prefix_end) lo = hi = n;
    else if (a.window) {
      const int span = a.window < a.N ? a.window + kRows / a.G : a.N;
      lo = min(lo, span);
      hi = min(hi, span);
    }
    steps = (float)(((int64_t)lo + hi) / 2 / kKeys + 1);
    most = max(1, min(a.most_parts, hi / kLeastKeys));
  }
  float work = (float)s.act * steps;
  for (int o = 32; o > 0; o >>= 1) work += __shfl_xor(work, o);
  const int active = last_of(sum_upto(s.act * a.Hkv));
  const bool fit = active <= a.turn / 2;
  float per = fmaxf(work * (float)a.Hkv / (float)(fit ? a.turn : 2 * a.turn), 1.0f);
  for (int tries = 0;; ++tries) {
    s.S = min(most, (int)ceilf(steps / per));
    s.S = max(s.S, 1);
    s.all = lane < a.B ? (a.tiles + s.act * (s.S - 1)) * a.Hkv : 0;
    s.cut = s.S > 1 ? s.act * a.Hkv : 0;
    s.slots = s.cut * s.S;
    s.all_upto = sum_upto(s.all);
    s.slots_upto = sum_upto(s.slots);
    const bool room = last_of(s.all_upto) <= a.by_length && last_of(s.slots_upto) <= a.most_slots;  // (S = 1 has room)
    if (room && (!fit || tries >= 6 || last_of(sum_upto(s.act * s.S * a.Hkv)) <= a.turn)) break;
    per *= room ? 1.0625f : 1.5f;
  }
  s.cut_upto = sum_upto(s.cut);
  return s;
}

// 16 bytes per lane from base + at into LDS, lane after lane from byte `to` on.  Asynchronous: wait_loads.  (Written out because
// the compiler lets every later read of LDS wait for such a load, though it goes to another buffer; nothing is returned in
// registers.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is a register that the compiler keeps to itself; nothing else here uses it)
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t at, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(at), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  asm volatile("" : : : "memory");
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

// The first key of register i of a 32 x 32 product, in the lower half of the wave (the upper half: 4 more).
__device__ __forceinline__ constexpr int key_of(int i) { return 8 * (i >> 2) + (i & 3); }

template <int D>
__device__ __forceinline__ int swizzle_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D>
__device__ __forceinline__ int swizzle_v(int row) { return D == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1); }

// MODE 1: scores are capped or biased.
template <typename T, int D, int MODE>
__global__ __launch_bounds__(256, 3) void prefill_kernel(const PrefillArgs a) {
  constexpr int STEPS = D / 16, MB = D / 32, PIECES = D / 8, ROWS_PER_LOAD = 64 / PIECES;
  constexpr int OWN = kKeys / 4, LOADS = OWN / ROWS_PER_LOAD;  // rows of a step that a wave fetches, loads of K (and of V) for them
  constexpr int ROW = D * 2, BUF = kKeys * ROW;
  constexpr float SHIFT = sizeof(T) == 2 && __is_same(T, _Float16) ? 8.0f : 0.0f;  // fp16 weights: away from its subnormals
  __shared__ __align__(1024) char lds[4 * BUF];  // [buffer][K, V]
  __shared__ int lds_range[4][4], lds_place[kRows][2];
  __shared__ int lds_zeroed;  // whether a value of V that is not finite was put to zero
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  int b, g, tile, part, S, slot = 0;
  if (a.by_length) {
    const Shares sh = shares_of(a, lane);
    const int at = (int)blockIdx.x;
    const uint64_t mine = __ballot(at < sh.all_upto && at >= sh.all_upto - sh.all);
    if (mine == 0) return;  // (no work left for this workgroup)
    b = __builtin_ctzll(mine);
    const int k = at - __builtin_amdgcn_readlane(sh.all_upto - sh.all, b), r = k / a.Hkv;
    const int first = __builtin_amdgcn_readlane(sh.first, b), act = __builtin_amdgcn_readlane(sh.act, b);
    g = k % a.Hkv;
    S = __builtin_amdgcn_readlane(sh.S, b);
    part = r % S;
    tile = first + act - 1 - r / S;
    if (r >= act * S) {  // the tiles behind and before those with rows
      part = 0;
      S = 1;
      tile = first + act + (r - act * __builtin_amdgcn_readlane(sh.S, b));
      if (tile >= a.tiles) tile -= a.tiles;
    }
    if (S > 1) slot = __builtin_amdgcn_readlane(sh.slots_upto - sh.slots, b) + k;
  } else {
    const int units = a.B * a.Hkv;
    const int rest = blockIdx.x / units;
    S = a.S;
    part = rest % S;
    tile = a.tiles - 1 - rest / S;
    // Ragged sequences take turns: where a few are long, workgroups at a fixed distance would be, which go to the same part of a die
    // (eight prompts, one of 8192 tokens and seven of 1000, 1525 us, with turns 658).
    const unsigned turn = a.seq_lens || a.q_start ? rest + (rest >> 1) + (rest >> 2) + (rest >> 3) : 0;
    b = (int)((blockIdx.x % units / a.Hkv + turn) % (unsigned)a.B);
    g = blockIdx.x % a.Hkv;
  }
  const int n = a.seq_lens ? min(max(a.seq_lens[b], 0), a.N) : a.N;

  const int64_t rows = (int64_t)a.T * a.G;
  const int64_t row = (int64_t)tile * kRows + 32 * wave + col;
  const bool there = row < rows;
  const int t = there ? (int)(row / a.G) : 0, h = g * a.G + (there ? (int)(row % a.G) : 0);
  lds_place[32 * wave + col][0] = t;  // (both halves of the wave the same)
  lds_place[32 * wave + col][1] = h;
  Seen seen = {1, 0, 0};
  if (there) seen = seen_keys(a, b, t, n);
  const bool some = seen.lo <= seen.hi;

  // Keys of the wave and of the workgroup: the span that some row sees, and the span that all rows see whole.
  const int first_w = -wave_max(some ? -seen.lo : -0x7FFFFFFF), last_w = wave_max(some ? seen.hi : -1);
  const int lo_w = wave_max(some ? seen.lo : 0), hi_w = -wave_max(some ? -seen.hi : -0x7FFFFFFF);
  if (lane == 0) {
    lds_range[wave][0] = first_w;
    lds_range[wave][1] = last_w;
    lds_range[wave][2] = lo_w;
    lds_range[wave][3] = hi_w;
    if (wave == 0) lds_zeroed = 0;
  }
  __syncthreads();
  int first = 0x7FFFFFFF, last = -1, lo_g = 0, hi_g = 0x7FFFFFFF;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    first = min(first, __builtin_amdgcn_readfirstlane(lds_range[w][0]));
    last = max(last, __builtin_amdgcn_readfirstlane(lds_range[w][1]));
    lo_g = max(lo_g, __builtin_amdgcn_readfirstlane(lds_range[w][2]));
    hi_g = min(hi_g, __builtin_amdgcn_readfirstlane(lds_range[w][3]));
  }
  int step = 0, step_end = 0;
  if (last >= 0) {
    step = first / kKeys;
    step_end = last / kKeys + 1;
  }
  if (S > 1) {
    const int per = (step_end - step + S - 1) / S;
    const int s0 = step + part * per;
    step_end = min(step_end, s0 + per);
    step = min(s0, step_end);
  }
  const int step_begin = step;

  // Fetching a step: wave w rows 8 w .. 8 w + 7 of K and of V, a row's pieces swapped.
  const char* const Kb = reinterpret_cast<const char*>(a.K + b * a.kv_sb + g * a.kv_sh);
  const char* const Vb = reinterpret_cast<const char*>(a.V + b * a.kv_sb + g * a.kv_sh);
  const uint32_t stride = (uint32_t)(a.kv_st * 2);
  uint32_t at_k[LOADS], at_v[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = OWN * wave + i * ROWS_PER_LOAD + lane / PIECES, piece = lane % PIECES;
    at_k[i] = r * stride + 16 * (piece ^ swizzle_k<D>(r));
    at_v[i] = r * stride + 16 * (piece ^ swizzle_v<D>(r));
  }
  auto fetch = [&](int st, int buf) {
    const int64_t base = (int64_t)st * kKeys * stride;
    const int most = n - 1 - st * kKeys;  // rows behind the last one are taken as the last
    const uint32_t to = lds_base + buf * 2 * BUF + OWN * wave * ROW;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      uint32_t back = 0;
      if (most < kKeys - 1) {
        const int r = OWN * wave + i * ROWS_PER_LOAD + lane / PIECES;
        back = (uint32_t)max(r - most, 0) * stride;
      }
      load_to_lds(Kb + base, at_k[i] - back, to + i * 1024);
      load_to_lds(Vb + base, at_v[i] - back, to + i * 1024 + BUF);
    }
  };
  if (step < step_end) fetch(step, 0);

  u32x4 qf[STEPS];
  {
    const uint16_t* qp = a.q + b * a.q_sb + h * a.q_sh + t * a.q_st + 8 * half;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) qf[i] = some ? *reinterpret_cast<const u32x4*>(qp + 16 * i) : (u32x4)(0);
  }
  const float slope = MODE == 1 && a.slopes ? a.slopes[h] * kLog2e : 0.0f;

  float m = kNone, z = 0.0f;
  bool large = false;  // some reference is beyond kLarge
  f32x16 o[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) o[i] = (f32x16)(0.0f);

  // Places in a step's rows: for scores this lane's row, for values its place in a block of 8 keys x 32
  // columns.  What is added to them is known at compile time.
  const int k_at = col * ROW + ((half ^ swizzle_k<D>(col)) << 4);
  const int v_row = 4 * half + ((lane & 15) >> 2), v_piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const int v_at = v_row * ROW + ((v_piece ^ swizzle_v<D>(v_row)) << 4) + 8 * (lane & 1);

  auto one_step = [&](auto buffer) {
    constexpr int buf = decltype(buffer)::value;
    const char* const Kl = lds + buf * 2 * BUF;
    char* const Vl = lds + buf * 2 * BUF + BUF;
    const int key0 = step * kKeys;
    const bool cut = key0 < lo_g || key0 + kKeys - 1 > hi_g;  // some row of the workgroup does not see all of the step
    wait_loads();
    if (cut) {  // the rows of V that this wave fetched
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        u32x4* const at = reinterpret_cast<u32x4*>(Vl + (OWN * wave + i * ROWS_PER_LOAD) * ROW + 16 * lane);
        u32x4 v = *at;
        uint32_t any = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t nf = not_finite<T>(v[x]);
          any |= nf;
          v[x] &= ~((nf >> 15) * 0xFFFFu);
        }
        if (any) {
          *at = v;
          lds_zeroed = 1;
        }
      }
    }
    lds_barrier();
    if (step + 1 < step_end) fetch(step + 1, buf ^ 1);
    if (key0 > last_w || key0 + kKeys - 1 < first_w) return;
    f32x16 sc;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const u32x4 kf = *reinterpret_cast<const u32x4*>(Kl + (k_at ^ (i << 5)));
      sc = Elem<T>::mfma32(kf, qf[i], i == 0 ? (f32x16)(0.0f) : sc);
    }
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
      if (a.slopes) {
        const float far = (float)(seen.p - key0 - 4 * half);
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = fmaf(-slope, fabsf(far - (float)key_of(e)), sc[e]);
      }
    }
    if (key0 < lo_w || key0 + kKeys - 1 > hi_w) {
      asm volatile("");  // (a branch, not 32 comparisons in every step)
      const uint32_t from = (uint32_t)(seen.lo - key0 - 4 * half), width = (uint32_t)(seen.hi - seen.lo);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!some | ((uint32_t)key_of(e) - from > width)) sc[e] = kNone;
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
        const char* const at = Vl + (v_at ^ (mb << 6)) + 16 * ks * ROW;
        const u32x2 x = read_columns(at), y = read_columns(at + 8 * ROW);
        const u32x4 vf = {x[0], x[1], y[0], y[1]};
        o[mb] = Elem<T>::mfma32(vf, pf[ks], o[mb]);
      }
    }
  };
  while (step < step_end) {
    one_step(std::integral_constant<int, 0>());
    if (++step >= step_end) break;
    one_step(std::integral_constant<int, 1>());
    ++step;
  }

  f32x4 naught = (f32x4)(0.0f);  // of what is finite; otherwise NaN
#pragma unroll
  for (int x = 0; x < MB * 16; ++x) naught[x & 3] = fmaf(o[x >> 4][x & 15], 0.0f, naught[x & 3]);
  const bool odd = lds_zeroed != 0 || (naught[0] + naught[1]) + (naught[2] + naught[3]) != 0.0f;
  if (__builtin_expect(__any(odd), 0)) {
    // Sums of what is not finite: first of the steps that all rows see whole, by column, eight columns a lane; then of the others,
    // which have left nothing in the results, row by row.
    int id = threadIdx.x;
    asm("" : "+v"(id));  // (nothing of this is kept in registers during the loop)
    const int in_load = (id & 63) / PIECES, piece_at = 16 * (id % PIECES), upper_half = (id >> 5) & 1;
    auto odd_part = [](float value) { return fabsf(value) < __builtin_inff() ? 0.0f : value; };
    auto rows_of = [&](int k0) { return *reinterpret_cast<const u32x4*>(Vb + (int64_t)min(k0 + in_load, n - 1) * stride + piece_at); };
    auto any_odd = [](u32x4 v) { return __ballot((not_finite<T>(v[0]) | not_finite<T>(v[1]) | not_finite<T>(v[2]) | not_finite<T>(v[3])) != 0); };
    auto cut = [&](int st) { return st * kKeys < lo_g || st * kKeys + kKeys - 1 > hi_g; };
    float all[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) all[x] = 0.0f;
#pragma unroll 1
    for (int st = step_begin; st < step_end; ++st) {
      if (cut(st)) continue;
      u32x4 v[4];
#pragma unroll 1
      for (int k0 = st * kKeys; k0 < st * kKeys + kKeys; k0 += 4 * ROWS_PER_LOAD) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = rows_of(k0 + i * ROWS_PER_LOAD);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (any_odd(v[i]))
#pragma unroll
            for (int x = 0; x < 8; ++x) all[x] += odd_part(unpack<T>(v[i][x >> 1], x & 1));
      }
    }
#pragma unroll
    for (int x = 0; x < 8; ++x)
      for (int across = PIECES; across < 64; across <<= 1) all[x] += __shfl_xor(all[x], across);
#pragma unroll
    for (int x = 0; x < MB * 4; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float lower = __shfl(all[y], x), upper = __shfl(all[4 + y], x), e = upper_half ? upper : lower;
        o[x >> 2][4 * (x & 3) + y] = e == 0.0f ? o[x >> 2][4 * (x & 3) + y] : e;
      }
#pragma unroll 1
    for (int k0 = max(first_w, step_begin * kKeys) / ROWS_PER_LOAD * ROWS_PER_LOAD; k0 < min(last_w + 1, step_end * kKeys); k0 += ROWS_PER_LOAD) {
      if (!cut(k0 / kKeys)) continue;
      uint64_t left = any_odd(rows_of(k0));
#pragma unroll 1
      while (left != 0) {
        const int in = __builtin_ctzll(left) / PIECES, k = k0 + in;
        left &= ~(((1ull << PIECES) - 1) << (in * PIECES));
        if (k >= n) break;  // (the last row once more)
        const bool sees = some && k >= seen.lo && k <= seen.hi;
        const char* const from = Vb + (int64_t)k * stride + 8 * upper_half;
#pragma unroll
        for (int x = 0; x < MB * 4; ++x) {
          const u32x2 u = *reinterpret_cast<const u32x2*>(from + 16 * x);
#pragma unroll
          for (int y = 0; y < 4; ++y) o[x >> 2][4 * (x & 3) + y] += sees ? odd_part(unpack<T>(u[y >> 1], y & 1)) : 0.0f;
        }
      }
    }
  }

  z += __shfl_xor(z, 32);
  // (a row's place is not kept in registers, which are short in the loop)
  int id = threadIdx.x;
  asm("" : "+v"(id));
  const int local = 32 * (id >> 6) + (id & 31), end_half = (id >> 5) & 1;
  const uint32_t end_row = (uint32_t)tile * kRows + local;
  if (end_row >= (uint32_t)rows) return;
  const int t_out = lds_place[local][0], h_out = lds_place[local][1];
  const int64_t out_row = ((int64_t)b * a.Hq + h_out) * a.T + t_out;
  if (S > 1) {
    const int64_t at = a.by_length ? (int64_t)slot * kRows + local : ((int64_t)(b * a.Hkv + g) * rows + end_row) * S + part;
    float* po = a.part_o + at * D + 4 * end_half;
    if (!some) m = kNone, z = 0.0f;
#pragma unroll
    for (int x = 0; x < MB * 4; ++x) {
      f32x4 v;
#pragma unroll
      for (int y = 0; y < 4; ++y) v[y] = some ? o[x >> 2][4 * (x & 3) + y] : 0.0f;
      *reinterpret_cast<f32x4*>(po + 8 * x) = v;
    }
    if (end_half == 0) {
      a.part_mz[at * 2] = m;
      a.part_mz[at * 2 + 1] = z;
    }
    return;
  }
  const bool none = !some || z == 0.0f;
  const float inv = none ? 0.0f : 1.0f / z;
  uint16_t* op = a.out + b * a.o_sb + h_out * a.o_sh + t_out * a.o_st + 4 * end_half;
#pragma unroll
  for (int x = 0; x < MB * 4; ++x) {
    u32x2 w;
    w[0] = none ? 0 : pack2<T>(o[x >> 2][4 * (x & 3)] * inv, o[x >> 2][4 * (x & 3) + 1] * inv);
    w[1] = none ? 0 : pack2<T>(o[x >> 2][4 * (x & 3) + 2] * inv, o[x >> 2][4 * (x & 3) + 3] * inv);
    *reinterpret_cast<u32x2*>(op + 8 * x) = w;
  }
  if (a.lse && end_half == 0) a.lse[out_row] = none ? kNone : (m - SHIFT + log2_(z)) * kLn2;
}

// The ranges' results of a query row, d / 4 x SHARES threads each: the shares take every SHARES-th range, in order, and are added
// at the end.
template <typename T, int D, int SHARES>
__global__ __launch_bounds__(256) void prefill_join_kernel(const PrefillArgs a) {
  constexpr int LANES = D / 4, ROWS = 256 / LANES / SHARES;
  constexpr float SHIFT = __is_same(T, _Float16) ? 8.0f : 0.0f;
  __shared__ float lds_sum[SHARES > 1 ? 256 / LANES : 1];
  __shared__ f32x4 lds_o[SHARES > 1 ? 256 : 1];
  const int d4 = threadIdx.x % LANES, share = threadIdx.x / LANES % SHARES;
  const int64_t rows = (int64_t)a.T * a.G, all = rows * a.B * a.Hkv;
  const int64_t mine = (int64_t)blockIdx.x * ROWS + threadIdx.x / (LANES * SHARES), at = min(mine, all - 1);
  const float* mz = a.part_mz + at * a.S * 2;
  float top = kNone;
  for (int i = 0; i < a.S; ++i) top = fmaxf(top, mz[2 * i]);
  const float ref = top == kNone ? 0.0f : top;
  float sum = 0.0f;
  f32x4 acc = (f32x4)(0.0f);
  const float* po = a.part_o + at * a.S * D + 4 * d4;
#pragma unroll 4
  for (int i = share; i < a.S; i += SHARES) {
    const float f = exp2_(mz[2 * i] - ref);
    sum += f * mz[2 * i + 1];
    acc += f * *reinterpret_cast<const f32x4*>(po + (int64_t)i * D);
  }
  if (__builtin_expect(!finite(acc), 0)) {  // (0 times an infinity is not what it should be)
    acc = (f32x4)(0.0f);
#pragma unroll 1
    for (int i = share; i < a.S; i += SHARES)
      acc = weighed(acc, 1.0f, *reinterpret_cast<const f32x4*>(po + (int64_t)i * D), exp2_(mz[2 * i] - ref));
  }
  if constexpr (SHARES > 1) {
    lds_o[threadIdx.x] = acc;
    if (d4 == 0) lds_sum[threadIdx.x / LANES] = sum;  // (the same in all threads of a share)
    __syncthreads();
    if (share > 0) return;
    for (int i = 1; i < SHARES; ++i) {
      acc += lds_o[threadIdx.x + i * LANES];
      sum += lds_sum[threadIdx.x / LANES + i];
    }
  }
  if (mine >= all) return;
  const int unit = (int)(at / rows);
  const int64_t row = at - unit * rows;
  const int b = unit / a.Hkv, g = unit % a.Hkv, t = (int)(row / a.G), h = g * a.G + (int)(row % a.G);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  u32x2 w;
  w[0] = pack2<T>(acc[0] * inv, acc[1] * inv);
  w[1] = pack2<T>(acc[2] * inv, acc[3] * inv);
  *reinterpret_cast<u32x2*>(a.out + b * a.o_sb + h * a.o_sh + t * a.o_st + 4 * d4) = w;
  if (d4 == 0 && a.lse) a.lse[((int64_t)b * a.Hq + h) * a.T + t] = sum == 0.0f ? kNone : (top - SHIFT + log2_(sum)) * kLn2;
}

// The same by length: a quarter of a tile in several ranges, four rows at a time for d / 4 threads, running maxima.
constexpr int kJoinRows = 32;
template <typename T, int D>
__global__ __launch_bounds__(256) void prefill_join_by_length_kernel(const PrefillArgs a) {
  constexpr int LANES = D / 4, GROUPS = 256 / LANES, R = kJoinRows / GROUPS;
  constexpr float SHIFT = __is_same(T, _Float16) ? 8.0f : 0.0f;
  const int at = (int)blockIdx.x / (kRows / kJoinRows);
  const Shares sh = shares_of(a, threadIdx.x & 63);
  const uint64_t mine = __ballot(at < sh.cut_upto && at >= sh.cut_upto - sh.cut);
  if (mine == 0) return;
  const int b = __builtin_ctzll(mine), S = __builtin_amdgcn_readlane(sh.S, b);
  const int k = at - __builtin_amdgcn_readlane(sh.cut_upto - sh.cut, b), g = k % a.Hkv;
  const int tile = __builtin_amdgcn_readlane(sh.first + sh.act, b) - 1 - k / a.Hkv;
  const int slot = __builtin_amdgcn_readlane(sh.slots_upto - sh.slots, b) + k / a.Hkv * S * a.Hkv + g;
  const int d4 = threadIdx.x % LANES, first = (int)(blockIdx.x % (kRows / kJoinRows)) * kJoinRows + threadIdx.x / LANES;
  const int64_t rows = (int64_t)a.T * a.G, row0 = (int64_t)tile * kRows + first;
  if (row0 >= rows) return;
  float m[R], z[R];
  f32x4 acc[R];
  auto join = [&](int j, auto careful) {
    const int64_t from = (int64_t)(slot + j * a.Hkv) * kRows + first;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t r = row0 + i * GROUPS < rows ? from + i * GROUPS : from;  // (rows that are not there leave nothing)
      const float m1 = a.part_mz[2 * r], z1 = a.part_mz[2 * r + 1];
      const f32x4 v = *reinterpret_cast<const f32x4*>(a.part_o + r * D + 4 * d4);
      const float top = fmaxf(m[i], m1), ref = top == kNone ? 0.0f : top;
      const float f0 = exp2_(m[i] - ref), f1 = exp2_(m1 - ref);
      m[i] = top;
      z[i] = z[i] * f0 + z1 * f1;
      if constexpr (decltype(careful)::value)
        acc[i] = weighed(acc[i], f0, v, f1);
      else
        acc[i] = __builtin_elementwise_fma(acc[i], (f32x4)(f0), v * f1);
    }
  };
  auto nothing = [&]() {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      m[i] = kNone;
      z[i] = 0.0f;
      acc[i] = (f32x4)(0.0f);
    }
  };
  nothing();
#pragma unroll 2
  for (int j = 0; j < S; ++j) join(j, std::false_type());
  bool odd = false;
#pragma unroll
  for (int i = 0; i < R; ++i) odd = odd || !finite(acc[i]);
  if (__builtin_expect(odd, 0)) {  // (0 times an infinity is not what it should be)
    nothing();
#pragma unroll 1
    for (int j = 0; j < S; ++j) join(j, std::true_type());
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t row = row0 + i * GROUPS;
    if (row >= rows) break;
    const int t = (int)(row / a.G), h = g * a.G + (int)(row % a.G);
    const float inv = z[i] == 0.0f ? 0.0f : 1.0f / z[i];
    u32x2 w;
    w[0] = pack2<T>(acc[i][0] * inv, acc[i][1] * inv);
    w[1] = pack2<T>(acc[i][2] * inv, acc[i][3] * inv);
    *reinterpret_cast<u32x2*>(a.out + b * a.o_sb + h * a.o_sh + t * a.o_st + 4 * d4) = w;
    if (d4 == 0 && a.lse) a.lse[((int64_t)b * a.Hq + h) * a.T + t] = z[i] == 0.0f ? kNone : (m[i] - SHIFT + log2_(z[i])) * kLn2;
  }
}

template <typename T, int D>
hipError_t launch(const PrefillArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.by_length ? a.by_length : (int64_t)a.tiles * a.S * a.B * a.Hkv)), block(256);
  if (a.cap.cap != 0.0f || a.slopes)
    hipLaunchKernelGGL((prefill_kernel<T, D, 1>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((prefill_kernel<T, D, 0>), grid, block, 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (!a.by_length && a.S == 1)) return e;
  if (a.by_length) {  // (a tile in several ranges has two slots at least)
    hipLaunchKernelGGL((prefill_join_by_length_kernel<T, D>), dim3((unsigned)(a.most_slots / 2 * (kRows / kJoinRows))), block, 0, s, a);
    return hipGetLastError();
  }
  const int64_t rows = (int64_t)a.T * a.G * a.B * a.Hkv;
  constexpr int PER = 256 / (D / 4);  // rows of a workgroup with one share
  if (a.S <= 16)  // (8400 rows of 11 ranges: 11.8 us, with eight shares 20.8)
    hipLaunchKernelGGL((prefill_join_kernel<T, D, 1>), dim3((unsigned)((rows + PER - 1) / PER)), block, 0, s, a);
  else
    hipLaunchKernelGGL((prefill_join_kernel<T, D, 8>), dim3((unsigned)((rows + PER / 8 - 1) / (PER / 8))), block, 0, s, a);
  return hipGetLastError();
}

int64_t row_tiles(const pkv_prefill_desc& d) { return ((int64_t)d.T * (d.Hq / d.Hkv) + kRows - 1) / kRows; }

int turn_of(const pkv_prefill_desc& d) { return d.d == 64 ? 1024 : 768; }  // workgroups that the device holds at a time

// Ranges of keys per tile of rows, where all sequences are as long.  The device holds 768 workgroups at a time (1024 with d = 64):
// one range where the tiles alone are as many, otherwise the fewest that fill (nearly) the largest share of one or two turns (300
// rows of 50k keys, 28 heads: 309 us in 11 ranges, 346 in 8, 361 in 12; 2048 rows of 64k keys, 512 tiles: 2.10 ms in 3, 2.20
// undivided).  A range's result is written and read again, 64 KB for 128 rows, so that none has fewer than 768 keys (4 x 64 rows of
// 3000 keys, 32 heads: 36 us with 1000 keys a range, 48 with 256).  By N, not by what is seen: with a window the ranges are shorter.
int parts(const pkv_prefill_desc& d) {
  const int64_t wgs = row_tiles(d) * d.B * d.Hkv, slots = turn_of(d);
  if (wgs >= slots) return 1;
  int64_t most = d.N / kLeastKeys;
  if (most > kMaxParts) most = kMaxParts;
  if (most > 2 * slots / wgs) most = 2 * slots / wgs;
  int best = 1;
  double share = 0.0;
  for (int64_t S = 1; S <= most; ++S) {
    const double full = (double)(wgs * S) / (double)((wgs * S + slots - 1) / slots * slots);
    if (full > 1.03 * share) {
      best = (int)S;
      share = full;
    }
  }
  return best;
}

// Ragged sequences: PrefillArgs' numbers for shares by length; workgroups 0 where there are none: where a sequence's rows alone
// fill the device (eight prompts of 200 - 4096 tokens 293 us, by length 313), and for few keys, where it is not worth the second
// kernel.  32 / 8 heads, d 128, us without and with: 24 x 96 rows of 400 - 8000 keys 229 and 146, of 800 - 16 000 452 and 310, all
// of 8000 370 and 368; 4 x 1024 rows of 400 - 8000 keys 270 and 232, all of 8000 483 and 502, all of 4000 232 and 263; 8 x 256
// rows, one sequence of 60 000 keys and seven of 1000, 741 and 351.
constexpr int kLeastRagged = 8 * kLeastKeys;
struct ByLength {
  int32_t workgroups, parts, slots;
};
ByLength by_length(const pkv_prefill_desc& d) {
  const int64_t unit = row_tiles(d) * d.Hkv, wgs = unit * d.B, turn = turn_of(d);
  if (d.B < 2 || d.B > 64 || d.N < kLeastRagged || unit >= turn) return {0, 1, 0};
  const int64_t extra = wgs <= turn / 2 ? turn : 2 * turn, most = d.N / kLeastKeys < kMaxParts ? d.N / kLeastKeys : kMaxParts;
  return {(int32_t)(wgs + extra), (int32_t)most, (int32_t)(wgs * most < 2 * extra ? wgs * most : 2 * extra)};
}

// Bytes of the ranges' results of a call with (ragged) or without lengths or starts.
size_t workspace_bytes_of(const pkv_prefill_desc& d, bool ragged) {
  const size_t row = (d.d + 2) * sizeof(float);
  const ByLength shares = by_length(d);
  if (ragged && shares.workgroups > 0) return (size_t)shares.slots * kRows * row;
  const int S = parts(d);
  return S == 1 ? 0 : (size_t)d.B * d.Hq * d.T * S * row;
}

double scale_of(const pkv_prefill_desc& d) { return d.scale > 0.0f ? (double)d.scale : 1.0 / sqrt((double)d.d); }

int check_prefill_desc(const pkv_prefill_desc* desc) {
  if (!desc) return PKV_ERR_INVALID_ARG;
  const pkv_prefill_desc& d = *desc;
  if (d.B < 1 || d.Hq < 1 || d.Hkv < 1 || d.Hq % d.Hkv != 0 || d.T < 1 || d.N < 1 || d.window < 0) return PKV_ERR_INVALID_ARG;
  if (d.dtype != PKV_BF16 && d.dtype != PKV_FP16) return PKV_ERR_INVALID_ARG;
  if (!(d.scale >= 0.0f) || !(d.cap >= 0.0f) || !isfinite(d.scale) || !isfinite(d.cap)) return PKV_ERR_INVALID_ARG;
  if (!good_strides(d.q_sb, d.q_sh, d.q_st) || !good_strides(d.kv_sb, d.kv_sh, d.kv_st) || !good_strides(d.o_sb, d.o_sh, d.o_st))
    return PKV_ERR_INVALID_ARG;
  if (d.d != 64 && d.d != 128) return PKV_ERR_UNSUPPORTED;
  if (!finite_factors(scale_of(d), d.cap)) return PKV_ERR_INVALID_ARG;
  if (d.Hq / d.Hkv > 128 || d.B > 65535 || d.N > (1 << 30) || d.T > (1 << 30)) return PKV_ERR_UNSUPPORTED;
  if ((int64_t)d.T * (d.Hq / d.Hkv) > 0x7FFFFF00ll) return PKV_ERR_UNSUPPORTED;
  if (d.kv_st > (1 << 23)) return PKV_ERR_UNSUPPORTED;  // (offsets inside a step: 32 bits)
  if ((int64_t)d.B * d.Hkv > kMaxGrid || row_tiles(d) > kMaxGrid / ((int64_t)d.B * d.Hkv)) return PKV_ERR_UNSUPPORTED;
  return PKV_OK;
}

}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

size_t pkv_prefill_even_workspace_bytes(const pkv_prefill_desc* desc) {
  if (check_prefill_desc(desc) != PKV_OK) return 0;
  return workspace_bytes_of(*desc, false);
}

size_t pkv_prefill_workspace_bytes(const pkv_prefill_desc* desc) {
  if (check_prefill_desc(desc) != PKV_OK) return 0;
  const size_t even = workspace_bytes_of(*desc, false), ragged = workspace_bytes_of(*desc, true);
  return even > ragged ? even : ragged;
}

int pkv_prefill_attention(const pkv_prefill_desc* desc, const void* q, const void* K, const void* V, const int32_t* seq_lens,
                          const int32_t* q_start, const int32_t* doc_start, const int32_t* prefix_end, const float* slopes,
                          void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc || !q || !K || !V || !out) return PKV_ERR_INVALID_ARG;
  const int rc = check_prefill_desc(desc);
  if (rc != PKV_OK) return rc;
  const pkv_prefill_desc& d = *desc;
  if (!aligned(q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(seq_lens, 4) || !aligned(q_start, 4) ||
      !aligned(doc_start, 4) || !aligned(prefix_end, 4) || !aligned(slopes, 4) || !aligned(lse_out, 4))
    return PKV_ERR_INVALID_ARG;
  const size_t need = workspace_bytes_of(d, seq_lens || q_start);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return PKV_ERR_WORKSPACE;
  PrefillArgs a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const uint16_t*>(q);
  a.K = static_cast<const uint16_t*>(K);
  a.V = static_cast<const uint16_t*>(V);
  a.seq_lens = seq_lens; a.q_start = q_start; a.doc_start = doc_start; a.prefix_end = prefix_end; a.slopes = slopes;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse_out;
  a.B = d.B; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.Hq / d.Hkv; a.T = d.T; a.N = d.N; a.window = d.window;
  a.S = parts(d);
  a.tiles = (int32_t)row_tiles(d);
  a.turn = turn_of(d);
  a.part_o = static_cast<float*>(workspace);
  const ByLength ragged = by_length(d);
  if ((seq_lens || q_start) && ragged.workgroups > 0) {
    a.by_length = ragged.workgroups;
    a.most_parts = ragged.parts;
    a.most_slots = ragged.slots;
    a.part_mz = a.part_o ? a.part_o + (size_t)ragged.slots * kRows * d.d : nullptr;
  } else {
    a.part_mz = a.part_o ? a.part_o + (size_t)d.B * d.Hq * d.T * a.S * d.d : nullptr;
  }
  a.q_sb = d.q_sb; a.q_sh = d.q_sh; a.q_st = d.q_st; a.kv_sb = d.kv_sb; a.kv_sh = d.kv_sh; a.kv_st = d.kv_st;
  a.o_sb = d.o_sb; a.o_sh = d.o_sh; a.o_st = d.o_st;
  a.scale = (float)(scale_of(d) * 1.4426950408889634);
  a.cap = make_cap(scale_of(d), d.cap);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (d.dtype == PKV_BF16)
    e = d.d == 128 ? launch<__bf16, 128>(a, st) : launch<__bf16, 64>(a, st);
  else
    e = d.d == 128 ? launch<_Float16, 128>(a, st) : launch<_Float16, 64>(a, st);
  return e == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
