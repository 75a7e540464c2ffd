// Attention of one new token per sequence over a cache of any length (include/pkv.h: pkv_decode_attention_long).
//
// HBM-bound: every seen row of K and V is read once (2 d bytes each), for all query heads of its KV head.  128k rows of 8 heads in
// 16-slot pages, d 128: 99 us with the join, 95 of them here (5.65 TB/s; a plain read of as much 6.3); four ragged sequences of up
// to 100k rows: 183 (5.6); 16 of up to 5000 kept rows with positions and biases: 25; 4k rows 12.3; 1000 rows, d 64: 6 and 4.
// Work split: (sequence, KV head, up to 64 of its query heads) x ranges of keys, a workgroup of four waves each; a wave takes
// 16 query heads, so that with up to 16, 32 and 64 heads four, two and one of the waves share the range's 32-key tiles.  Every
// wave works on its own, K tile -> scores -> running softmax -> V tile, the rows of its next tile requested as soon as this
// tile's are used up, and the waves meet once at the end.  Where a sequence has several ranges, they leave un-normalised results
// in a workspace, and a second kernel joins them in order.
// Ranges: as long as fill the device once (512 workgroups), by the sequences' lengths as they are on the device, so that ragged
// batches have ranges of one length too; every wave works out its place among them from all counts (2 to 256 sequences).
//   loads   whole rows, 1 KB at a time, into registers; from there to the wave's own tile in LDS, K first, then V in its place.
//   scores  S^T = K Q^T in v_mfma_f32_16x16x32: 16 keys are the rows of A, 16 heads the columns of B.  Lane (l16, quad) ends with
//           keys 4 quad .. + 3 of head l16, all it needs for its weights.
//   softmax a reference exponent per head and wave, moved only when a score exceeds it by a factor of 2^8 (fp16: 2^2).
//   values  O^T += V^T P^T: the weights are in B's layout already if the 32 keys of a step are taken in the order in which the
//           lanes hold them (4 quad .. + 3 of either half), and V^T is read column-wise.  The weights are given as two numbers of
//           the type, their rounding and what it left (16 bits for bf16; 22 for fp16, down to steps of 2^-37 of the reference):
//           the matrix pipe has time for both products.
// Rows that are not seen (behind the count, outside the window, on a page that does not exist) have weight 0, and their copy of
// V is zero.
#include <math.h>
#include <string.h>

#include "pkv_attn.h"

namespace pkv {
namespace {

constexpr int kTile = 32;          // keys per step of a wave
constexpr int kWaves = 4;          // per workgroup
constexpr int kWorkgroups = 512;   // at a time on the device: two per compute unit
constexpr int kLaneSequences = 4;  // sequences a lane looks after where ranges go by lengths,
constexpr int kFlatBatch = 64 * kLaneSequences;  // and so many at most in all
constexpr int kLeastTiles = 8;     // of a range

struct LongArgs {
  const uint16_t *q, *K, *V;
  const int32_t *table, *count, *positions, *q_pos;
  const float* slopes;
  uint16_t* out;
  float* lse;
  float* part_o;   // [workgroup][head of its group][d]
  float* part_mz;  // [workgroup][head of its group][2] reference exponent (log2) and sum
  int32_t B, Hq, Hkv, G, k_cap, page_size, num_pages, max_pages, window;
  int32_t ranges;       // 0: every sequence whole; by_length: workgroups to share out; otherwise ranges of each sequence
  int32_t by_length;    // (2 .. kFlatBatch sequences)
  int32_t units;        // of a sequence: Hkv * head_groups
  int32_t head_groups;  // workgroups that share a KV head's rows: ceil(G / 64)
  int32_t wave_groups;  // 16-head groups in a workgroup: 1, 2 or 4
  uint32_t page_magic;  // floor(2^32 / page_size)
  int64_t q_sb, q_sh, c_sb, c_sh, c_st, p_sb, p_sh;
  float scale;          // of the products, to log2 units (without a cap)
  Cap cap;
};

// The factor of the softmax weights, and how far a score may exceed the reference (log2).
template <typename T>
struct Weight {
  static constexpr bool HALF = __is_same(T, _Float16);
  static constexpr float SHIFT = HALF ? kFp16Shift : 0.0f, SLACK = HALF ? kFp16Slack : 8.0f;
  static constexpr float UNIT = HALF ? 1.0f / (1 << (int)kFp16Shift) : 1.0f;  // 2^-SHIFT
};

// A wave's reads and writes of its own part of LDS keep their order.
__device__ __forceinline__ void own_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// The tiles of sequence b that can hold a seen row: all, or with positions of their own numbers those of the window.
struct Tiles {
  int n, q_pos, first, count;
};
__device__ __forceinline__ Tiles tiles_of(const LongArgs& a, int b) {
  Tiles r;
  r.n = min(max(a.count[b], 0), a.k_cap);
  r.q_pos = a.q_pos ? a.q_pos[b] : r.n - 1;
  int first = 0, end = r.n;
  if (!a.positions) {
    end = (int)min((int64_t)r.n, (int64_t)r.q_pos + 1);
    if (a.window) first = (int)min((int64_t)r.n, max((int64_t)0, (int64_t)r.q_pos - a.window + 1));
  }
  r.first = first / kTile;
  r.count = end > first ? (end + kTile - 1) / kTile - r.first : 0;
  return r;
}

// How the sequences are cut, for 2 .. 64 E of them: lane i looks after sequences i E .. i E + E - 1, whose numbers of ranges and
// first workgroup it works out; all ranges but a sequence's last have `per` tiles.  Ranges as long as make `ranges` workgroups of
// all tiles, then, of one turn of the device, longer (a few tries) until the last, shorter ones of the sequences fit among them
// too; never more than ranges + B * units.
template <int E>
struct Cut {
  Tiles tl[E];
  int ranges[E], per, base, end;
};
template <int E>
__device__ __forceinline__ Cut<E> flat_cut(const LongArgs& a, int lane) {
  Cut<E> c;
  int sum = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    c.tl[e] = tiles_of(a, min(lane * E + e, a.B - 1));
    sum += lane * E + e < a.B ? c.tl[e].count : 0;
  }
  const uint64_t all = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(sum_upto(sum), 63) * (uint32_t)a.units;
  const int shares = kWaves / a.wave_groups, shift = a.ranges == kWorkgroups ? 9 : 10;
  c.per = max((int)((all + a.ranges - 1) >> shift), kLeastTiles);
  c.per = (c.per + shares - 1) / shares * shares;
  for (int tries = 0;; ++tries) {
    sum = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      c.ranges[e] = lane * E + e < a.B ? max(1, (int)((uint32_t)(c.tl[e].count + c.per - 1) / (uint32_t)c.per)) : 0;
      sum += c.ranges[e] * a.units;
    }
    c.end = sum_upto(sum);
    if (shift != 9 || tries == 6 || __builtin_amdgcn_readlane(c.end, 63) <= kWorkgroups) break;
    c.per += max(shares, c.per / 16 / shares * shares);
  }
  c.base = c.end - sum;
  return c;
}

// A workgroup's sequence, that one's ranges and its first workgroup; no sequence (-1): no work is left for it.
struct Place {
  int b, ranges, per, base;
  Tiles tl;
};
__device__ __forceinline__ Tiles tiles_from(const Tiles& t, int lane) {
  return {__builtin_amdgcn_readlane(t.n, lane), __builtin_amdgcn_readlane(t.q_pos, lane), __builtin_amdgcn_readlane(t.first, lane),
          __builtin_amdgcn_readlane(t.count, lane)};
}
template <int E>
__device__ __forceinline__ Place place_of_workgroup(const LongArgs& a, int workgroup, int lane) {
  const Cut<E> c = flat_cut<E>(a, lane);
  const uint64_t mine = __ballot(workgroup >= c.base && workgroup < c.end);
  if (mine == 0) return {-1, 0, 0, 0, {0, 0, 0, 0}};
  const int at = __builtin_ctzll(mine);
  Place p = {at * E, __builtin_amdgcn_readlane(c.ranges[0], at), c.per, __builtin_amdgcn_readlane(c.base, at), tiles_from(c.tl[0], at)};
#pragma unroll
  for (int e = 1; e < E; ++e) {
    if (workgroup >= p.base + p.ranges * a.units) {
      p.base += p.ranges * a.units;
      p.ranges = __builtin_amdgcn_readlane(c.ranges[e], at);
      p.b = at * E + e;
      p.tl = tiles_from(c.tl[e], at);
    }
  }
  return p;
}
template <int E>
__device__ __forceinline__ Place place_of_sequence(const LongArgs& a, int b, int lane) {
  const Cut<E> c = flat_cut<E>(a, lane);
  const int at = b / E;
  Place p = {b, __builtin_amdgcn_readlane(c.ranges[0], at), c.per, __builtin_amdgcn_readlane(c.base, at), c.tl[0]};
#pragma unroll
  for (int e = 1; e < E; ++e) {
    if (e <= b % E) {
      p.base += p.ranges * a.units;
      p.ranges = __builtin_amdgcn_readlane(c.ranges[e], at);
    }
  }
  return p;
}

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void decode_long_kernel(const LongArgs a) {
  constexpr int LANES = D / 8, STEPS = D / 32, VLOADS = kTile * LANES / 64, MT = D / 16;
  __shared__ __align__(16) char lds_v[kWaves][kTile * D * 2];
  __shared__ float lds_mz[kWaves][16][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, quad = lane >> 4;
  int b, s, ranges, unit;
  Tiles tl;
  int per;
  if (!a.by_length) {
    ranges = max(a.ranges, 1);
    s = blockIdx.x % ranges;
    b = blockIdx.x / ranges / a.units;
    unit = blockIdx.x / ranges % a.units;
    tl = tiles_of(a, b);
    per = (tl.count + ranges - 1) / ranges;
  } else {
    const Place p = a.B <= 64 ? place_of_workgroup<1>(a, blockIdx.x, lane) : place_of_workgroup<kLaneSequences>(a, blockIdx.x, lane);
    if (p.b < 0) return;
    b = p.b;
    ranges = p.ranges;
    per = p.per;
    unit = ((int)blockIdx.x - p.base) / ranges;
    s = ((int)blockIdx.x - p.base) % ranges;
    tl = p.tl;
  }
  const int g = unit / a.head_groups, hg = unit % a.head_groups;
  const int wg = wave & (a.wave_groups - 1), share = wave / a.wave_groups, shares = kWaves / a.wave_groups;
  const int h_in = 64 * hg + 16 * wg + l16;  // query head within the group of this KV head
  const bool head = h_in < a.G;
  const int h = g * a.G + (head ? h_in : 0);

  const int n = tl.n, q_pos = tl.q_pos;
  int t = tl.first + s * per + share;
  const int t_end = tl.first + min((s + 1) * per, tl.count);

  u32x4 qf[STEPS];
  {
    const uint16_t* qp = a.q + b * a.q_sb + h * a.q_sh;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) qf[i] = head ? *reinterpret_cast<const u32x4*>(qp + 32 * i + 8 * quad) : (u32x4)(0);
  }
  const float slope = a.slopes ? a.slopes[h] * kLog2e : 0.0f;
  const uint32_t row_bytes = (uint32_t)(a.page_size ? D : a.c_st) * 2;
  const int64_t base = a.page_size ? 0 : (b * a.c_sb + g * a.c_sh) * 2;
  const char* const Kb = reinterpret_cast<const char*>(a.K) + base + 16 * (lane % LANES);
  const char* const Vb = reinterpret_cast<const char*>(a.V) + base + 16 * (lane % LANES);
  const int32_t* const table = a.table + (int64_t)b * a.max_pages;
  const int32_t* const pos_b = a.positions + b * a.p_sb + g * a.p_sh;
  const int least = a.window ? (int)max((int64_t)q_pos - a.window + 1, (int64_t)0) : 0;  // of the seen positions
  if (q_pos < least) t = t_end;

  // What has to be loaded to know a tile's rows: lane l looks after row l % 32.
  int32_t page = 0, slot = 0, pos_next = 0;
  auto look = [&](int tile) {
    const int j = min(tile * kTile + (lane & 31), n - 1);
    slot = j;
    if (a.page_size) {
      uint32_t p = __umulhi((uint32_t)j, a.page_magic);
      if ((uint32_t)j - p * a.page_size >= (uint32_t)a.page_size) ++p;
      slot = j - p * a.page_size;
      page = table[p];
    }
    pos_next = a.positions ? pos_b[j] : j;
  };
  // The rows that are seen, one bit each, their positions, and where the rows lie (in rows of one stride).  Where a row is not
  // seen, the cache's first is loaded: nothing that is far, or not there.
  uint32_t seen = 0, at = 0;
  int32_t pos = 0;
  auto resolve = [&](int tile) {
    pos = pos_next;
    bool is = tile < t_end && tile * kTile + (lane & 31) < n && (uint32_t)pos - (uint32_t)least <= (uint32_t)q_pos - (uint32_t)least;
    at = slot;
    if (a.page_size) {
      is = is && (uint32_t)page < (uint32_t)a.num_pages;
      at = ((uint32_t)page * a.Hkv + g) * a.page_size + slot;
    }
    at = is ? at : 0;
    seen = (uint32_t)__ballot(is);
  };

  // Rows of a tile, 1 KB of neighbouring rows at a time: load i holds rows i 64 / LANES .. of the tile.
  u32x4 kr[VLOADS], vr[VLOADS];
  uint32_t at_row[VLOADS];
  auto load = [&](const char* from, u32x4 (&to)[VLOADS]) {
#pragma unroll
    for (int i = 0; i < VLOADS; ++i) to[i] = *reinterpret_cast<const u32x4*>(from + (uint64_t)at_row[i] * row_bytes);
  };
  auto place = [&]() {
#pragma unroll
    for (int i = 0; i < VLOADS; ++i) at_row[i] = (uint32_t)__shfl((int)at, i * (64 / LANES) + lane / LANES);
  };
  // 16-byte piece c of a row of the copies lies at c ^ swizzle(row): 16 rows' pieces of one column block go to all banks, whether
  // whole pieces of K or column blocks of V are read.
  auto swizzle_k = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
  auto swizzle = [](int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); };
  char* const copy = lds_v[wave];

  float m = kNone, z = 0.0f;
  f32x4 o[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) o[i] = (f32x4)(0.0f);

  if (t < t_end) {
    const int t_first = t;
    look(t);
    resolve(t);
    place();
    look(min(t + shares, t_end - 1));
    load(Kb, kr);
    load(Vb, vr);
    for (; t < t_end; t += shares) {
      const uint32_t now = seen;
      const int32_t pos_now = pos;
#pragma unroll
      for (int i = 0; i < VLOADS; ++i) {
        const int r = i * (64 / LANES) + lane / LANES;
        *reinterpret_cast<u32x4*>(copy + r * (D * 2) + (((lane % LANES) ^ swizzle_k(r)) << 4)) = kr[i];
      }
      resolve(t + shares);
      place();
      look(min(t + 2 * shares, t_end - 1));
      load(Kb, kr);
      own_lds_order();
      f32x4 sc[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        sc[kt] = (f32x4)(0.0f);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const int r = 16 * kt + l16;
          const u32x4 kf = *reinterpret_cast<const u32x4*>(copy + r * (D * 2) + (((4 * i + quad) ^ swizzle_k(r)) << 4));
          sc[kt] = Elem<T>::mfma16(kf, qf[i], sc[kt]);
        }
      }
      own_lds_order();
      // scores in units of log2
      if (__builtin_expect(a.cap.cap != 0.0f, 0)) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = sc[e >> 2][e & 3];
        cap_scores(x, a.cap);
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e >> 2][e & 3] = x[e];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e >> 2][e & 3] *= a.scale;
      }
      if (__builtin_expect(a.slopes != nullptr, 0)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int kp = __shfl(pos_now, 16 * (e >> 2) + 4 * quad + (e & 3));
          sc[e >> 2][e & 3] -= slope * (float)(int)((uint32_t)q_pos - (uint32_t)kp);
        }
      }
      if (__builtin_expect(now != 0xFFFFFFFFu, 0)) {
        const uint32_t mine = now >> (4 * quad);
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e >> 2][e & 3] = mine & (1u << (16 * (e >> 2) + (e & 3))) ? sc[e >> 2][e & 3] : kNone;
      }
      float top = sc[0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, sc[e >> 2][e & 3]);
      if (__any(top - m > Weight<T>::SLACK)) {  // (top - m, since m + SLACK is rounded where scores are large)
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
      auto weight = [&](float x) {
        const float below = x - ref;
        return exp2_(Weight<T>::HALF ? below + Weight<T>::SHIFT : below);
      };
      u32x4 hi, lo;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float p0 = weight(sc[e >> 2][e & 3]), p1 = weight(sc[e >> 2][(e & 3) + 1]);
        z += p0 + p1;
        const uint32_t u = pack2<T>(p0, p1);
        hi[e >> 1] = u;
        lo[e >> 1] = pack2<T>(p0 - unpack<T>(u, 0), p1 - unpack<T>(u, 1));
      }
      // V: registers -> the wave's copy -> columns
#pragma unroll
      for (int i = 0; i < VLOADS; ++i) {
        const int r = i * (64 / LANES) + lane / LANES;
        *reinterpret_cast<u32x4*>(copy + r * (D * 2) + (((lane % LANES) ^ swizzle(r)) << 4)) = vr[i];
      }
      load(Vb, vr);
      if (__builtin_expect(now != 0xFFFFFFFFu, 0)) {
        own_lds_order();
        if (!((now >> (lane & 31)) & 1)) {  // two lanes a row
#pragma unroll 1
          for (int c = lane >> 5; c < LANES; c += 2) *reinterpret_cast<u32x4*>(copy + (lane & 31) * (D * 2) + (c << 4)) = (u32x4)(0);
        }
      }
      own_lds_order();
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
      own_lds_order();
    }
    // A value that is not finite in a seen row: its column is what the sum of those is (every weight is positive), and not what
    // 0 or less, where a weight's second part is that, makes of an infinity.
    bool odd = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < 4; ++e) odd = odd || !(fabsf(o[mt][e]) < __builtin_inff());
    if (__builtin_expect(__any(odd), 0)) {
      f32x4 extra[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) extra[mt] = (f32x4)(0.0f);
      const char* const Vq = reinterpret_cast<const char*>(a.V) + base + 8 * quad;
      for (t = t_first; t < t_end; t += shares) {
        look(t);
        resolve(t);
        for (uint32_t left = seen; left != 0; left &= left - 1) {
          const char* const row = Vq + (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)at, __builtin_ctz(left)) * row_bytes;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const u32x2 v = *reinterpret_cast<const u32x2*>(row + 32 * mt);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = unpack<T>(v[e >> 1], e & 1);
              extra[mt][e] += fabsf(x) < __builtin_inff() ? 0.0f : x;
            }
          }
        }
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[mt][e] = extra[mt][e] == 0.0f ? o[mt][e] : extra[mt][e];
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
    auto outputs = [&](int w) { return *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(lds_v[w]) + hl * D + ((d4 ^ (hl & 7)) << 2)); };
    for (int w = w0; w < kWaves; w += a.wave_groups) {
      const float f = exp2_(lds_mz[w][hl][0] - ref);
      sum += f * lds_mz[w][hl][1];
      acc += f * outputs(w);
    }
    if (__builtin_expect(!finite(acc), 0)) {
      acc = (f32x4)(0.0f);
#pragma unroll 1
      for (int w = w0; w < kWaves; w += a.wave_groups) acc = weighed(acc, 1.0f, outputs(w), exp2_(lds_mz[w][hl][0] - ref));
    }
    const int64_t row = (int64_t)b * a.Hq + g * a.G + 64 * hg + hh;
    if (ranges > 1) {
      const int64_t at = (int64_t)blockIdx.x * (16 * a.wave_groups) + hh;
      *reinterpret_cast<f32x4*>(a.part_o + at * D + 4 * d4) = acc;
      if (d4 == 0) {
        a.part_mz[at * 2] = top;
        a.part_mz[at * 2 + 1] = sum;
      }
    } else {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      u32x2 w;
      w[0] = pack2<T>(acc[0] * inv, acc[1] * inv);
      w[1] = pack2<T>(acc[2] * inv, acc[3] * inv);
      *reinterpret_cast<u32x2*>(a.out + row * D + 4 * d4) = w;
      if (d4 == 0 && a.lse) a.lse[row] = sum == 0.0f ? kNone : (top + log2_(sum * Weight<T>::UNIT)) * kLn2;
    }
  }
}

// One workgroup per (sequence, HEADS query heads one after the other): the ranges' results, every PARTS-th of them by one part of
// the threads, in order, each with a running maximum of its own (so that a range's exponent and its values are requested together),
// then the parts.
template <typename T, int D, int HEADS>
__global__ __launch_bounds__(256) void decode_long_join_kernel(const LongArgs a) {
  constexpr int PARTS = 256 / (D / 4);
  __shared__ float lds_m[PARTS], lds_z[PARTS];
  __shared__ f32x4 lds_o[PARTS][D / 4];
  const int b = (int)((int64_t)blockIdx.x * HEADS / a.Hq);
  int ranges = a.ranges, base = b * a.units * a.ranges;
  if (a.by_length) {
    const int lane = threadIdx.x & 63;
    const Place p = a.B <= 64 ? place_of_sequence<1>(a, b, lane) : place_of_sequence<kLaneSequences>(a, b, lane);
    ranges = p.ranges;
    base = p.base;
  }
  if (ranges == 1) return;  // (written already)
  const int64_t heads = 16 * a.wave_groups;
  const int d4 = threadIdx.x % (D / 4), part = threadIdx.x / (D / 4);
  float m, z;
  f32x4 acc;
  auto join = [&](float m1, float z1, f32x4 v, bool careful = false) {
    const float top = fmaxf(m, m1), ref = top == kNone ? 0.0f : top;
    const float f0 = exp2_(m - ref), f1 = exp2_(m1 - ref);
    m = top;
    z = z * f0 + z1 * f1;
    if (careful)
      acc = weighed(acc, f0, v, f1);
    else
      acc = __builtin_elementwise_fma(acc, (f32x4)(f0), v * f1);
  };
  auto nothing = [&]() {
    m = kNone;
    z = 0.0f;
    acc = (f32x4)(0.0f);
  };
#pragma unroll 1
  for (int k = 0; k < HEADS; ++k) {
    const int64_t row = (int64_t)blockIdx.x * HEADS + k;
    const int h = (int)(row % a.Hq), h_in = h % a.G, unit = h / a.G * a.head_groups + h_in / 64;
    const int64_t at = ((int64_t)base + unit * ranges) * heads + h_in % 64;
    nothing();
#pragma unroll 4
    for (int i = part; i < ranges; i += PARTS) {
      const float* const mz = a.part_mz + (at + heads * i) * 2;
      join(mz[0], mz[1], *reinterpret_cast<const f32x4*>(a.part_o + (at + heads * i) * D + 4 * d4));
    }
    if (__builtin_expect(!finite(acc), 0)) {  // (0 times an infinity is not what it should be)
      nothing();
#pragma unroll 1
      for (int i = part; i < ranges; i += PARTS) {
        const float* const mz = a.part_mz + (at + heads * i) * 2;
        join(mz[0], mz[1], *reinterpret_cast<const f32x4*>(a.part_o + (at + heads * i) * D + 4 * d4), true);
      }
    }
    if (k > 0) __syncthreads();  // (the last head's parts have been read)
    lds_o[part][d4] = acc;
    if (d4 == 0) {
      lds_m[part] = m;
      lds_z[part] = z;
    }
    __syncthreads();
    if (part == 0) {
#pragma unroll
      for (int i = 1; i < PARTS; ++i) join(lds_m[i], lds_z[i], lds_o[i][d4]);
      if (__builtin_expect(!finite(acc), 0)) {
        nothing();
#pragma unroll 1
        for (int i = 0; i < PARTS; ++i) join(lds_m[i], lds_z[i], lds_o[i][d4], true);
      }
      const float inv = z == 0.0f ? 0.0f : 1.0f / z;
      u32x2 w;
      w[0] = pack2<T>(acc[0] * inv, acc[1] * inv);
      w[1] = pack2<T>(acc[2] * inv, acc[3] * inv);
      *reinterpret_cast<u32x2*>(a.out + row * D + 4 * d4) = w;
      if (d4 == 0 && a.lse) a.lse[row] = z == 0.0f ? kNone : (m + log2_(z * Weight<T>::UNIT)) * kLn2;
    }
  }
}

// Query heads that a workgroup's results have room for.
int heads_of(int G) { return G <= 16 ? 16 : G <= 32 ? 32 : 64; }

// Two turns of workgroups without ranges: they are not cut where a sequence is short, or where there are so many that the longest
// matters little (and the workspace would be large).  128 sequences of 8 heads, d 128: 127 of 1000 rows and one of 100 000 take
// 1085 us uncut, 181 cut (floor 148); 128 of 1000 rows 94 and 100, of 8000 rows 688 and 693, of 100 rows 17 and 25.
constexpr int kWhole = 4096, kMostUnits = 8192;

// Workgroups of a call, and what LongArgs::ranges and by_length are for it.
struct Grid {
  int64_t workgroups;
  int32_t ranges, by_length;
};
Grid grid_of(const pkv_decode_long_desc& d) {
  const int64_t units = (int64_t)d.Hkv * ((d.Hq / d.Hkv + 63) / 64), all = d.B * units;
  if (d.k_cap <= kLeastTiles * kTile) return {all, 0, 0};
  // (tiles of all sequences are added in 32 bits)
  if (d.B > 1 && d.B <= kFlatBatch && (int64_t)d.B * d.k_cap <= (int64_t)1 << 36) {
    const int64_t share = all <= kWorkgroups / 2 ? kWorkgroups : 2 * kWorkgroups;
    return all >= 2 * kWorkgroups && (d.k_cap <= kWhole || all > kMostUnits) ? Grid{all, 0, 0} : Grid{share + all, (int32_t)share, 1};
  }
  int64_t S = kWorkgroups / all;
  const int64_t most = ((int64_t)d.k_cap + kLeastTiles * kTile - 1) / (kLeastTiles * kTile);
  if (S > most) S = most;
  return S <= 1 ? Grid{all, 0, 0} : Grid{all * S, (int32_t)S, 0};
}

template <typename T, int D>
hipError_t launch(const LongArgs& a, int64_t workgroups, hipStream_t s) {
  hipLaunchKernelGGL((decode_long_kernel<T, D>), dim3((unsigned)workgroups), dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.ranges == 0) return e;
  // Many heads: four a workgroup (128 sequences of 32 heads, 100 rows each: 25 us, one by one 30; 64 of 16 are faster one by one).
  if (a.Hq % 4 == 0 && a.B * a.Hq >= 4 * kWorkgroups)
    hipLaunchKernelGGL((decode_long_join_kernel<T, D, 4>), dim3((unsigned)(a.B * a.Hq / 4)), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((decode_long_join_kernel<T, D, 1>), dim3((unsigned)(a.B * a.Hq)), dim3(256), 0, s, a);
  return hipGetLastError();
}

double scale_of(const pkv_decode_long_desc& d) { return d.scale > 0.0f ? (double)d.scale : 1.0 / sqrt((double)d.d); }

int check_long_desc(const pkv_decode_long_desc* desc) {
  if (!desc) return PKV_ERR_INVALID_ARG;
  const pkv_decode_long_desc& d = *desc;
  if (d.B < 1 || d.Hq < 1 || d.Hkv < 1 || d.Hq % d.Hkv != 0 || d.k_cap < 1 || d.page_size < 0 || d.window < 0) return PKV_ERR_INVALID_ARG;
  if (d.dtype != PKV_BF16 && d.dtype != PKV_FP16) return PKV_ERR_INVALID_ARG;
  if (!(d.scale >= 0.0f) || !(d.cap >= 0.0f) || !isfinite(d.scale) || !isfinite(d.cap)) return PKV_ERR_INVALID_ARG;
  if (!good_strides(d.q_sb, d.q_sh, 0)) return PKV_ERR_INVALID_ARG;
  if (d.page_size > 0) {
    if (d.num_pages < 1 || d.max_pages < ((int64_t)d.k_cap + d.page_size - 1) / d.page_size) return PKV_ERR_INVALID_ARG;
  } else {
    if (!good_strides(d.c_sb, d.c_sh, d.c_st)) return PKV_ERR_INVALID_ARG;
  }
  if (d.p_sb < 0 || d.p_sh < 0) return PKV_ERR_INVALID_ARG;
  if (d.d != 64 && d.d != 128) return PKV_ERR_UNSUPPORTED;
  if (!finite_factors(scale_of(d), d.cap)) return PKV_ERR_INVALID_ARG;
  const int64_t G = d.Hq / d.Hkv;
  if (G > 128 || d.B > 65535 || d.k_cap > (1 << 30) || d.Hkv > 65535 || (int64_t)d.B * d.Hq > kMaxGrid) return PKV_ERR_UNSUPPORTED;
  if (d.page_size == 0 && d.c_st > (1 << 30)) return PKV_ERR_UNSUPPORTED;  // (a row's bytes: 32 bits)
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
  const Grid g = grid_of(*desc);
  return g.ranges == 0 ? 0 : (size_t)g.workgroups * heads_of(desc->Hq / desc->Hkv) * (desc->d + 2) * sizeof(float);
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
  const Grid grid = grid_of(d);
  a.ranges = grid.ranges;
  a.by_length = grid.by_length;
  a.part_o = static_cast<float*>(workspace);
  a.part_mz = a.part_o ? a.part_o + (size_t)grid.workgroups * heads_of(d.Hq / d.Hkv) * d.d : nullptr;
  a.B = d.B; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.Hq / d.Hkv; a.k_cap = d.k_cap;
  a.page_size = d.page_size; a.num_pages = d.num_pages; a.max_pages = d.max_pages; a.window = d.window;
  a.head_groups = (a.G + 63) / 64;
  a.units = a.Hkv * a.head_groups;
  a.wave_groups = heads_of(a.G) / 16;
  a.page_magic = d.page_size > 1 ? (uint32_t)(((uint64_t)1 << 32) / (uint32_t)d.page_size) : 0xFFFFFFFFu;
  a.q_sb = d.q_sb; a.q_sh = d.q_sh; a.c_sb = d.c_sb; a.c_sh = d.c_sh; a.c_st = d.c_st; a.p_sb = d.p_sb; a.p_sh = d.p_sh;
  a.scale = (float)(scale_of(d) * 1.4426950408889634);
  a.cap = make_cap(scale_of(d), d.cap);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (d.dtype == PKV_BF16)
    e = d.d == 128 ? launch<__bf16, 128>(a, grid.workgroups, st) : launch<__bf16, 64>(a, grid.workgroups, st);
  else
    e = d.d == 128 ? launch<_Float16, 128>(a, grid.workgroups, st) : launch<_Float16, 64>(a, grid.workgroups, st);
  return e == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
