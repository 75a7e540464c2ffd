// Attention of few query rows per KV head over caches of any length: the kernel and the join of its ranges, as pkv_decode_long.hip (one
// token, where the kernel is described), pkv_weigh.hip (the same, handing its scores on), pkv_tree.hip (drafted tokens) and
// pkv_blocks.hip (listed blocks of rows) build them.
#pragma once

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
constexpr int kLeastTiles = 8;     // of a range,
// and of many query rows, whose results are more to join (32/8 heads, d 128: 64 tokens behind 4000 rows with 8, 12, 16 26.2, 27.6, 29.3 us,
// 4 sequences of 32 tokens behind 3000 rows 28.5, 27.5, 29.1).
constexpr int kLeastWide = 12;

// What the kernel is built for: one token over all rows; the same, handing its scores on; drafted tokens; listed blocks of rows.
// (kTreeWide: drafted tokens whose query rows are many, in pkv_tree.hip's own kernel.)
enum { kOneToken = 0, kWeigh = 1, kTree = 2, kBlocks = 3, kTreeWide = 4 };

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
  static constexpr int MODE = kOneToken;
};
// Adding up weights: the scores are kept for the kernel behind, which also joins ranges.
struct WeighArgs : LongArgs {
  float* scores;      // [B * Hkv][G][score_row], in log2 units, -inf where a row is not seen; rows of the visited tiles
  float* mz;          // [B * Hq][2] reference exponent and factor of heads that are not cut into ranges
  float* weights;
  int64_t score_row, w_sb, w_sh;
  static constexpr int MODE = kWeigh;
};
// Drafted tokens: G is the number of query rows that share a KV head, T * heads, row t * heads + h.  Hq is Hkv * G.
struct TreeArgs : LongArgs {
  const int32_t *tree, *new_lens;
  int32_t T, words, heads;  // words of 32 drafted tokens in a row of tree
  int64_t q_st, o_sb, o_sh, o_st;
  static constexpr int MODE = kTree;
};
struct TreeWideArgs : TreeArgs {
  int32_t turn;  // workgroups that the device holds at a time
  static constexpr int MODE = kTreeWide;
};
template <typename A>
constexpr bool drafted_mode() { return A::MODE == kTree || A::MODE == kTreeWide; }
// Query rows of a workgroup.
template <typename A>
constexpr int group_rows() { return A::MODE == kTreeWide ? 128 : 64; }
// Listed blocks: place x of the list's rows is row list[x >> shift] << shift | (x & (block - 1)).
struct BlocksArgs : LongArgs {
  const int32_t* blocks;  // [B][Hkv][most]
  int32_t most, shift;
  static constexpr int MODE = kBlocks;
};

// The factor of the softmax weights, and how far a score may exceed the reference (log2).
template <typename T>
struct Weight {
  static constexpr bool HALF = __is_same(T, _Float16);
  static constexpr float SHIFT = HALF ? kFp16Shift : 0.0f, SLACK = HALF ? kFp16Slack : 8.0f;
  static constexpr float UNIT = HALF ? 1.0f / (1 << (int)kFp16Shift) : 1.0f;  // 2^-SHIFT
};

constexpr int kWideShift = 8;  // kTreeWide, fp16: as pkv_prefill.hip has it

// As many workgroups as a launch whose items follow the room of a cache starts at most: two turns of the device, eight of 256 threads per
// compute unit.  Most of a large cache's room holds no rows yet, and a workgroup that finds nothing to do still has to be started: one row
// too many in 64 sequences of 8 heads, room for 4096 rows, 30 us with a workgroup for each item, 16 with these.  A prime, so that the items
// of one head spread over all of them (one sequence of 64 evicted from 16k rows to 2k: 37 us, with 2048 workgroups 56).  With 2039 and 8191:
// 15 and 18, 33 and 41; 64 sequences evicted from 4096 rows to 2048 157 and 146, with these 148.
constexpr int kMostWorkgroups = 4093;
// The items: `chunks` chunks of each of `units` heads.  Where there are no more than workgroups, neighbours have neighbouring chunks of a head
// (weights of 100k and 25k rows 121 us, 125 the other way round); otherwise the heads' first chunks come first, which spreads what there is
// where heads have few (weights of 64 sequences of 2000 rows with room for 16k 83 us, head by head 99).
struct Items {
  uint32_t all;           // units * chunks, below 2^31
  uint32_t minor, magic;  // chunks, or units; magic_of(minor)
  bool by_head;
};
// A workgroup's items, every stride-th from its first one on: work(unit, chunk).  A lane looks whether one of 64 has something to do, so that
// those that have not cost one look together; all waves of the workgroup come to the same.
template <typename Has, typename Work>
__device__ __forceinline__ void each_item(const Items& items, uint32_t first, uint32_t stride, Has has, Work work) {
  auto major_of = [&](uint32_t item) {
    const uint32_t m = __umulhi(item, items.magic);
    return m + (item - m * items.minor >= items.minor);
  };
  if (items.by_head) {
    const uint32_t unit = major_of(first);
    work((int)unit, (int)(first - unit * items.minor));
    return;
  }
  const uint32_t lane = threadIdx.x & 63;
  for (uint32_t i0 = first; i0 < items.all; i0 += 64 * stride) {
    const uint32_t own = min(i0 + lane * stride, items.all - 1), chunk = major_of(own), unit = own - chunk * items.minor;
    for (uint64_t left = __ballot(i0 + lane * stride < items.all && has((int)unit, (int)chunk)); left != 0; left &= left - 1) {
      const int l = __builtin_ctzll(left);
      work(__builtin_amdgcn_readlane((int)unit, l), __builtin_amdgcn_readlane((int)chunk, l));
    }
  }
}

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
// (Drafted tokens: q_pos is the first one's row.)
template <typename A>
__device__ __forceinline__ Tiles tiles_of(const A& a, int b) {
  Tiles r;
  r.n = min(max(a.count[b], 0), a.k_cap);
  int first = 0, end = r.n;
  if constexpr (A::MODE == kBlocks) {
    r.q_pos = r.n - 1;
    r.first = 0;
    r.count = ((min(a.most, (r.n + (1 << a.shift) - 1) >> a.shift) << a.shift) + kTile - 1) / kTile;
    return r;
  }
  if constexpr (drafted_mode<A>()) {
    r.q_pos = max(a.count[b], 0) - (a.new_lens ? min(max(a.new_lens[b], 0), a.T) : a.T);
    if (!a.positions && a.window) first = (int)min((int64_t)r.n, max((int64_t)0, (int64_t)r.q_pos - a.window + 1));
    r.first = first / kTile;
    r.count = end > first ? (end + kTile - 1) / kTile - r.first : 0;
    return r;
  }
  r.q_pos = a.q_pos ? a.q_pos[b] : r.n - 1;
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
template <int E, typename A>
__device__ __forceinline__ Cut<E> flat_cut(const A& a, int lane) {
  Cut<E> c;
  int sum = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    c.tl[e] = tiles_of(a, min(lane * E + e, a.B - 1));
    sum += lane * E + e < a.B ? c.tl[e].count : 0;
  }
  const uint64_t all = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(sum_upto(sum), 63) * (uint32_t)a.units;
  const int shares = A::MODE == kTreeWide ? 1 : kWaves / a.wave_groups, shift = a.ranges == kWorkgroups ? 9 : 10;
  c.per = A::MODE == kTreeWide ? max((int)((all + a.ranges - 1) / (uint32_t)a.ranges), kLeastWide) : max((int)((all + a.ranges - 1) >> shift), kLeastTiles);
  c.per = (c.per + shares - 1) / shares * shares;
  for (int tries = 0;; ++tries) {
    sum = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      c.ranges[e] = lane * E + e < a.B ? max(1, (int)((uint32_t)(c.tl[e].count + c.per - 1) / (uint32_t)c.per)) : 0;
      sum += c.ranges[e] * a.units;
    }
    c.end = sum_upto(sum);
    if constexpr (A::MODE == kTreeWide) {
      if (a.ranges != a.turn || tries == 6 || __builtin_amdgcn_readlane(c.end, 63) <= a.turn) break;
    }
    if (A::MODE != kTreeWide && (shift != 9 || tries == 6 || __builtin_amdgcn_readlane(c.end, 63) <= kWorkgroups)) break;
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
template <int E, typename A>
__device__ __forceinline__ Place place_of_workgroup(const A& a, int workgroup, int lane) {
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
template <int E, typename A>
__device__ __forceinline__ Place place_of_sequence(const A& a, int b, int lane) {
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

// A head's reference and the factor that makes softmax weights of the 2^(score - reference).
__device__ __forceinline__ void keep_mz(const WeighArgs& a, int b, int g, int h_in, float ref, float factor) {
  float* const mz = a.mz + ((int64_t)b * a.Hq + g * a.G + h_in) * 2;
  mz[0] = ref;
  mz[1] = factor;
}

constexpr int kMostDrafted = 256;
// How many of the drafted tokens token t sees besides itself.
__device__ __forceinline__ int ancestors(const TreeArgs& a, int b, int t, int drafted) {
  if (!a.tree) return min(t, drafted);
  const int32_t* const row = a.tree + ((int64_t)b * a.T + t) * a.words;
  int n = 0;
  for (int w = 0; w < a.words; ++w) {
    const int there = min(max(drafted - 32 * w, 0), 32);
    const uint32_t own = w == t >> 5 ? 1u << (t & 31) : 0u, all = there == 32 ? ~0u : (1u << there) - 1;
    n += __popc((uint32_t)row[w] & ~own & all);
  }
  return n;
}
// Which of the 32 tokens from off on (those before 0: the past) token t sees.
__device__ __forceinline__ uint32_t drafted_seen(const TreeArgs& a, int b, int t, int off) {
  if (!a.tree) {
    const int k = t - off + 1;
    return k <= 0 ? 0u : k >= 32 ? ~0u : (1u << k) - 1;
  }
  const int32_t* const row = a.tree + ((int64_t)b * a.T + t) * a.words;
  if (off < 0) return (uint32_t)row[0] << -off | ((1u << -off) - 1);
  const int w = off >> 5;
  const uint64_t lo = w < a.words ? (uint32_t)row[w] : 0u, hi = w + 1 < a.words ? (uint32_t)row[w + 1] : 0u;
  return (uint32_t)((hi << 32 | lo) >> (off & 31));
}

// A row's place in out: row h_in of those that share KV head g.
template <typename A>
__device__ __forceinline__ int64_t out_at(const A& a, int b, int g, int h_in, int D) {
  if constexpr (drafted_mode<A>())
    return b * a.o_sb + (g * a.heads + h_in % a.heads) * a.o_sh + (h_in / a.heads) * a.o_st;
  else
    return ((int64_t)b * a.Hq + g * a.G + h_in) * D;
}
template <typename A>
__device__ __forceinline__ int64_t lse_at(const A& a, int b, int g, int h_in) {
  if constexpr (drafted_mode<A>())
    return ((int64_t)b * (a.Hkv * a.heads) + g * a.heads + h_in % a.heads) * a.T + h_in / a.heads;
  else
    return (int64_t)b * a.Hq + g * a.G + h_in;
}

template <typename T, int D, typename A>
__global__ __launch_bounds__(256, 2) void decode_long_kernel(const A a) {
  constexpr bool TREE = A::MODE == kTree, BLOCKS = A::MODE == kBlocks;
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
  int h, t_row = 0;  // (t_row: the drafted token)
  if constexpr (TREE) {
    t_row = head ? h_in / a.heads : 0;
    h = g * a.heads + (head ? h_in % a.heads : 0);
  } else {
    h = g * a.G + (head ? h_in : 0);
  }

  const int n = tl.n, q_pos = tl.q_pos;
  int t = tl.first + s * per + share;
  const int t_end = tl.first + min((s + 1) * per, tl.count);

  u32x4 qf[STEPS];
  {
    const uint16_t* qp = a.q + b * a.q_sb + h * a.q_sh;
    if constexpr (TREE) qp += t_row * a.q_st;
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
  const int least = !TREE && a.window ? (int)max((int64_t)q_pos - a.window + 1, (int64_t)0) : 0;  // of the seen positions
  if (!TREE && q_pos < least) t = t_end;

  // Drafted tokens: the own row's position, which rows of a tile it sees (one bit each) of those that are there for some row, and
  // the least and the greatest position of the wave's rows.
  [[maybe_unused]] int32_t p_row = 0, p_min = 0, p_max = 0;
  [[maybe_unused]] int drafted = 0;  // tokens, and whether the own row is one of them
  [[maybe_unused]] bool row_there = false;
  __shared__ int32_t lds_depth[TREE ? kMostDrafted : 1];
  if constexpr (TREE) {
    drafted = a.new_lens ? min(max(a.new_lens[b], 0), a.T) : a.T;
    row_there = head && t_row < drafted;
    if (a.q_pos) {
      p_row = a.q_pos[(int64_t)b * a.T + t_row];
    } else if (a.window || a.slopes) {  // (behind the past as far as ancestors lie between)
      for (int i = threadIdx.x; i < a.T; i += 256) lds_depth[i] = ancestors(a, b, i, drafted);
      __syncthreads();
      p_row = q_pos + lds_depth[t_row];
    }
    p_min = ~wave_max(row_there ? ~p_row : INT32_MIN);
    p_max = wave_max(row_there ? p_row : INT32_MIN);
  }

  // What has to be loaded to know a tile's rows: lane l looks after row l % 32.
  int32_t page = 0, slot = 0, pos_next = 0;
  // Listed blocks: the list is looked up a tile before that.
  [[maybe_unused]] int32_t block_next = 0, row_next = 0;
  auto peek = [&](int tile) {
    if constexpr (BLOCKS) {
      const int entries = min(a.most, (n + (1 << a.shift) - 1) >> a.shift);
      block_next = a.blocks[((int64_t)b * a.Hkv + g) * a.most + min((tile * kTile + (lane & 31)) >> a.shift, entries - 1)];
    }
  };
  auto look = [&](int tile) {
    int j = min(tile * kTile + (lane & 31), n - 1);
    if constexpr (BLOCKS) {
      const int x = tile * kTile + (lane & 31);
      const bool is = (uint32_t)block_next <= (uint32_t)((n - 1) >> a.shift) && x < min(a.most, (n + (1 << a.shift) - 1) >> a.shift) << a.shift;
      row_next = is ? (block_next << a.shift) + (x & ((1 << a.shift) - 1)) : n;
      j = min(row_next, n - 1);
    }
    slot = j;
    if (a.page_size) {
      uint32_t p = __umulhi((uint32_t)j, a.page_magic);
      if ((uint32_t)j - p * a.page_size >= (uint32_t)a.page_size) ++p;
      slot = j - p * a.page_size;
      page = table[p];
    }
    pos_next = a.positions ? pos_b[j] : j;
    if constexpr (TREE) {
      if (!a.positions) pos_next = j < q_pos || !(a.window || a.slopes) ? j : q_pos + lds_depth[min(j - q_pos, a.T - 1)];
    }
  };
  // Of the rows `now` that are there, those that the own row sees.
  auto visible = [&](int tile, uint32_t now, int32_t pos_now) {
    uint32_t mine = now;
    if constexpr (TREE) {
      if (!row_there) mine = 0;
      const int off = tile * kTile - q_pos;  // the drafted token of the tile's first row
      if (off + kTile > 0) mine &= drafted_seen(a, b, t_row, off);
      if (a.positions || a.window) {
        const bool past = off + (lane & 31) < 0;
        const bool all = (!past || pos_now <= p_min) && (!a.window || (int64_t)pos_now > (int64_t)p_max - a.window);
        for (uint32_t left = now & ~(uint32_t)__ballot(all); left != 0; left &= left - 1) {
          const int i = __builtin_ctz(left);
          const int32_t kp = __builtin_amdgcn_readlane(pos_now, i);
          if ((off + i < 0 && kp > p_row) || (a.window && (int64_t)kp <= (int64_t)p_row - a.window)) mine &= ~(1u << i);
        }
      }
    }
    return mine;
  };
  // The rows that are seen, one bit each, their positions, and where the rows lie (in rows of one stride).  Where a row is not
  // seen, the cache's first is loaded: nothing that is far, or not there.
  uint32_t seen = 0, at = 0;
  int32_t pos = 0;
  auto resolve = [&](int tile) {
    pos = pos_next;
    bool is = tile < t_end;
    if constexpr (BLOCKS)
      is = is && row_next < n;
    else if constexpr (TREE)
      is = is && tile * kTile + (lane & 31) < n && (!a.positions || pos >= 0);
    else
      is = is && tile * kTile + (lane & 31) < n && (uint32_t)pos - (uint32_t)least <= (uint32_t)q_pos - (uint32_t)least;
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
  [[maybe_unused]] bool zeroed = false;  // whether a value of V that is not finite was put to zero

  if (t < t_end) {
    const int t_first = t;
    peek(t);
    look(t);
    peek(min(t + shares, t_end - 1));
    resolve(t);
    place();
    look(min(t + shares, t_end - 1));
    peek(min(t + 2 * shares, t_end - 1));
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
      peek(min(t + 3 * shares, t_end - 1));
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
          if constexpr (TREE)
            sc[e >> 2][e & 3] -= slope * (float)(kp > p_row ? (uint32_t)kp - (uint32_t)p_row : (uint32_t)p_row - (uint32_t)kp);
          else
            sc[e >> 2][e & 3] -= slope * (float)(int)((uint32_t)q_pos - (uint32_t)kp);
        }
      }
      [[maybe_unused]] bool hidden = false;  // some row of the wave does not see a row that is there
      uint32_t vis = now;
      if constexpr (TREE) {
        vis = visible(t, now, pos_now);
        hidden = __any(row_there && vis != now);
      }
      if (__builtin_expect(TREE ? __any(vis != 0xFFFFFFFFu) : now != 0xFFFFFFFFu, 0)) {
        const uint32_t mine = vis >> (4 * quad);
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e >> 2][e & 3] = mine & (1u << (16 * (e >> 2) + (e & 3))) ? sc[e >> 2][e & 3] : kNone;
      }
      if constexpr (A::MODE == kWeigh) {
        if (head) {
          float* const to = a.scores + (((int64_t)b * a.Hkv + g) * a.G + h_in) * a.score_row + (int64_t)t * kTile + 4 * quad;
          *reinterpret_cast<f32x4*>(to) = sc[0];
          *reinterpret_cast<f32x4*>(to + 16) = sc[1];
        }
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
      if constexpr (TREE) {
        if (hidden) {  // a value that is not finite would spoil the product with a weight of 0
          uint32_t any = 0;
#pragma unroll
          for (int i = 0; i < VLOADS; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const uint32_t nf = not_finite<T>(vr[i][x]);
              any |= nf;
              vr[i][x] &= ~((nf >> 15) * 0xFFFFu);
            }
          zeroed = zeroed || __any(any != 0);
        }
      }
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
    if constexpr (TREE) {
      if (!row_there)  // (0 times what is not finite)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) o[mt] = (f32x4)(0.0f);
    }
    bool odd = zeroed;
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
        peek(t);
        look(t);
        resolve(t);
        [[maybe_unused]] const uint32_t vis = visible(t, seen, pos);
        for (uint32_t left = seen; left != 0; left &= left - 1) {
          const char* const row = Vq + (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)at, __builtin_ctz(left)) * row_bytes;
          [[maybe_unused]] const bool sees = !TREE || (vis >> __builtin_ctz(left) & 1);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const u32x2 v = *reinterpret_cast<const u32x2*>(row + 32 * mt);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = unpack<T>(v[e >> 1], e & 1);
              extra[mt][e] += fabsf(x) < __builtin_inff() || !sees ? 0.0f : x;
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
      *reinterpret_cast<u32x2*>(a.out + out_at(a, b, g, 64 * hg + hh, D) + 4 * d4) = w;
      if (d4 == 0 && a.lse) a.lse[lse_at(a, b, g, 64 * hg + hh)] = sum == 0.0f ? kNone : (top + log2_(sum * Weight<T>::UNIT)) * kLn2;
      if constexpr (A::MODE == kWeigh) {
        if (d4 == 0) keep_mz(a, b, g, 64 * hg + hh, ref, inv * (1.0f / Weight<T>::UNIT));
      }
    }
  }
}

// One workgroup per (sequence, HEADS query heads one after the other): the ranges' results, every PARTS-th of them by one part of
// the threads, in order, each with a running maximum of its own (so that a range's exponent and its values are requested together),
// then the parts.
template <typename T, int D, int HEADS, typename A>
__device__ __forceinline__ void join_heads(const A& a) {
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
  constexpr bool WIDE = A::MODE == kTreeWide;
  constexpr float UNIT = WIDE && Weight<T>::HALF ? 1.0f / (1 << kWideShift) : Weight<T>::UNIT;
  const int64_t heads = WIDE ? 128 : 16 * a.wave_groups, step = WIDE ? heads * a.units : heads;  // between a row's ranges
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
    const int h = (int)(row % a.Hq), h_in = h % a.G, group = h_in / group_rows<A>();
    const int unit = WIDE ? group * a.Hkv + h / a.G : h / a.G * a.head_groups + group;
    const int64_t at = ((int64_t)base + (WIDE ? unit : unit * ranges)) * heads + h_in % group_rows<A>();
    nothing();
#pragma unroll 4
    for (int i = part; i < ranges; i += PARTS) {
      const float* const mz = a.part_mz + (at + step * i) * 2;
      join(mz[0], mz[1], *reinterpret_cast<const f32x4*>(a.part_o + (at + step * i) * D + 4 * d4));
    }
    if (__builtin_expect(!finite(acc), 0)) {  // (0 times an infinity is not what it should be)
      nothing();
#pragma unroll 1
      for (int i = part; i < ranges; i += PARTS) {
        const float* const mz = a.part_mz + (at + step * i) * 2;
        join(mz[0], mz[1], *reinterpret_cast<const f32x4*>(a.part_o + (at + step * i) * D + 4 * d4), true);
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
      *reinterpret_cast<u32x2*>(a.out + out_at(a, b, h / a.G, h_in, D) + 4 * d4) = w;
      if (d4 == 0 && a.lse) a.lse[lse_at(a, b, h / a.G, h_in)] = z == 0.0f ? kNone : (m + log2_(z * UNIT)) * kLn2;
    }
  }
}
template <typename T, int D, int HEADS, typename A>
__global__ __launch_bounds__(256) void decode_long_join_kernel(const A a) {
  join_heads<T, D, HEADS>(a);
}

// Query heads that a workgroup's results have room for.
inline int heads_of(int G) { return G <= 16 ? 16 : G <= 32 ? 32 : 64; }

// Two turns of workgroups without ranges: they are not cut where a sequence is short, or where there are so many that the longest
// matters little (and the workspace would be large).  128 sequences of 8 heads, d 128: 127 of 1000 rows and one of 100 000 take
// 1085 us uncut, 181 cut (floor 148); 128 of 1000 rows 94 and 100, of 8000 rows 688 and 693, of 100 rows 17 and 25.
constexpr int kWhole = 4096, kMostUnits = 8192;

// Workgroups of a call of B sequences with `rows` query rows on each of Hkv heads and up to k_cap keys, and what LongArgs::ranges and
// by_length are for it.
struct Grid {
  int64_t workgroups;
  int32_t ranges, by_length;
};
inline Grid grid_of(int64_t B, int64_t Hkv, int64_t rows, int64_t k_cap) {
  const int64_t units = Hkv * ((rows + 63) / 64), all = B * units;
  if (k_cap <= kLeastTiles * kTile) return {all, 0, 0};
  // (tiles of all sequences are added in 32 bits)
  if (B > 1 && B <= kFlatBatch && B * k_cap <= (int64_t)1 << 36) {
    const int64_t share = all <= kWorkgroups / 2 ? kWorkgroups : 2 * kWorkgroups;
    return all >= 2 * kWorkgroups && (k_cap <= kWhole || all > kMostUnits) ? Grid{all, 0, 0} : Grid{share + all, (int32_t)share, 1};
  }
  int64_t S = kWorkgroups / all;
  const int64_t most = (k_cap + kLeastTiles * kTile - 1) / (kLeastTiles * kTile);
  if (S > most) S = most;
  return S <= 1 ? Grid{all, 0, 0} : Grid{all * S, (int32_t)S, 0};
}
// Bytes of the ranges' results.
inline size_t parts_bytes(const Grid& g, int rows, int d) {
  return g.ranges == 0 ? 0 : (size_t)g.workgroups * heads_of(rows) * (d + 2) * sizeof(float);
}

template <typename T, int D, typename A>
hipError_t launch_join(const A& a, hipStream_t s) {
  // Many heads: four a workgroup (128 sequences of 32 heads, 100 rows each: 25 us, one by one 30; 64 of 16 are faster one by one).
  if (a.Hq % 4 == 0 && a.B * a.Hq >= 4 * kWorkgroups)
    hipLaunchKernelGGL((decode_long_join_kernel<T, D, 4, A>), dim3((unsigned)(a.B * a.Hq / 4)), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((decode_long_join_kernel<T, D, 1, A>), dim3((unsigned)(a.B * a.Hq)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int D, typename A>
hipError_t launch_long(const A& a, int64_t workgroups, hipStream_t s) {
  hipLaunchKernelGGL((decode_long_kernel<T, D, A>), dim3((unsigned)workgroups), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.ranges == 0 || A::MODE == kWeigh ? e : launch_join<T, D>(a, s);  // (kWeigh has a join of its own)
}
template <typename A>
hipError_t launch_long(const A& a, int dtype, int d, int64_t workgroups, hipStream_t s) {
  if (dtype == PKV_BF16)
    return d == 128 ? launch_long<__bf16, 128>(a, workgroups, s) : launch_long<__bf16, 64>(a, workgroups, s);
  return d == 128 ? launch_long<_Float16, 128>(a, workgroups, s) : launch_long<_Float16, 64>(a, workgroups, s);
}

// What all descriptors of such calls have in common: the arguments' fields, and whether they hold together.
template <typename Desc>
double scale_of(const Desc& d) { return d.scale > 0.0f ? (double)d.scale : 1.0 / sqrt((double)d.d); }

template <typename Desc>
int check_pages(const Desc& d) {
  if (d.k_cap < 1 || d.page_size < 0) return PKV_ERR_INVALID_ARG;
  if (d.page_size > 0) {
    if (d.num_pages < 1 || d.max_pages < ((int64_t)d.k_cap + d.page_size - 1) / d.page_size) return PKV_ERR_INVALID_ARG;
  } else {
    if (!good_strides(d.c_sb, d.c_sh, d.c_st)) return PKV_ERR_INVALID_ARG;
  }
  return PKV_OK;
}
template <typename Desc>
int check_cache_limits(const Desc& d) {
  if (d.d != 64 && d.d != 128) return PKV_ERR_UNSUPPORTED;
  if (d.B > 65535 || d.k_cap > (1 << 30) || d.Hkv > 65535) return PKV_ERR_UNSUPPORTED;
  if (d.page_size == 0 && d.c_st > (1 << 30)) return PKV_ERR_UNSUPPORTED;  // (a row's bytes: 32 bits)
  // rows of a pool are counted in 32 bits
  if (d.page_size > 0 && (double)d.num_pages * d.Hkv * d.page_size > 4294967295.0) return PKV_ERR_UNSUPPORTED;
  return PKV_OK;
}
template <typename Desc>
int check_scores(const Desc& d) {
  if (d.B < 1 || d.Hq < 1 || d.Hkv < 1 || d.Hq % d.Hkv != 0) return PKV_ERR_INVALID_ARG;
  if (d.dtype != PKV_BF16 && d.dtype != PKV_FP16) return PKV_ERR_INVALID_ARG;
  if (!(d.scale >= 0.0f) || !(d.cap >= 0.0f) || !isfinite(d.scale) || !isfinite(d.cap)) return PKV_ERR_INVALID_ARG;
  if (!good_strides(d.q_sb, d.q_sh, 0)) return PKV_ERR_INVALID_ARG;
  return PKV_OK;
}
template <typename Desc>
int check_factors(const Desc& d) { return finite_factors(scale_of(d), d.cap) ? PKV_OK : PKV_ERR_INVALID_ARG; }

inline int check_long_desc(const pkv_decode_long_desc* desc) {
  if (!desc) return PKV_ERR_INVALID_ARG;
  const pkv_decode_long_desc& d = *desc;
  if (check_scores(d) != PKV_OK || check_pages(d) != PKV_OK || d.window < 0 || d.p_sb < 0 || d.p_sh < 0) return PKV_ERR_INVALID_ARG;
  if (d.d != 64 && d.d != 128) return PKV_ERR_UNSUPPORTED;
  if (check_factors(d) != PKV_OK) return PKV_ERR_INVALID_ARG;
  if (d.Hq / d.Hkv > 128 || (int64_t)d.B * d.Hq > kMaxGrid) return PKV_ERR_UNSUPPORTED;
  return check_cache_limits(d);
}

inline int check_long_call(const pkv_decode_long_desc* desc, const void* q, const void* K_cache, const void* V_cache, const int32_t* block_table,
                           const int32_t* count, const int32_t* positions, const int32_t* q_pos, const float* slopes, const void* out,
                           const float* lse_out) {
  if (!desc || !q || !K_cache || !V_cache || !count || !out) return PKV_ERR_INVALID_ARG;
  const int rc = check_long_desc(desc);
  if (rc != PKV_OK) return rc;
  if (!aligned(q, 16) || !aligned(K_cache, 16) || !aligned(V_cache, 16) || !aligned(out, 16) || !aligned(block_table, 4) ||
      !aligned(count, 4) || !aligned(positions, 4) || !aligned(q_pos, 4) || !aligned(slopes, 4) || !aligned(lse_out, 4))
    return PKV_ERR_INVALID_ARG;
  if (desc->page_size > 0 && !block_table) return PKV_ERR_INVALID_ARG;
  return PKV_OK;
}

// Whether places of a tensor are distinct, as what a call writes must be: `inner` neighbours, and dimensions of `size` places that lie
// `stride` apart, in any order.  Of those with several places each stride has to reach behind all that the smaller ones span.  (Enough
// for it; slices and transposes of a contiguous tensor are like that.)
struct Dim {
  int64_t size, stride;
};
template <int N>
bool apart(int64_t inner, Dim (&&dims)[N]) {
  int64_t span = inner;
  for (int i = 0; i < N; ++i) {
    for (int k = i + 1; k < N; ++k) {
      if (dims[k].stride < dims[i].stride) {
        const Dim d = dims[i];
        dims[i] = dims[k];
        dims[k] = d;
      }
    }
    if (dims[i].size <= 1) continue;
    if (dims[i].stride < span) return false;
    const int64_t steps = dims[i].size - 1;
    span = dims[i].stride > (INT64_MAX - span) / steps ? INT64_MAX : span + dims[i].stride * steps;
  }
  return true;
}

inline uint32_t magic_of(int page_size) { return page_size > 1 ? (uint32_t)(((uint64_t)1 << 32) / (uint32_t)page_size) : 0xFFFFFFFFu; }

inline Items items_of(int64_t units, int64_t chunks) {
  const bool by_head = units * chunks <= kMostWorkgroups;
  const int minor = (int)(by_head ? chunks : units);
  return {(uint32_t)(units * chunks), (uint32_t)minor, magic_of(minor), by_head};
}
inline int64_t workgroups_of(const Items& items) { return items.all < kMostWorkgroups ? items.all : kMostWorkgroups; }
constexpr int64_t kMostItems = ((int64_t)1 << 31) - 1;

// The fields that a descriptor gives; rows: query rows that share a KV head.
template <typename Desc>
void fill_long(LongArgs& a, const Desc& d, const Grid& grid, int rows, const void* q, const void* K, const void* V, void* out, void* parts) {
  a.q = static_cast<const uint16_t*>(q);
  a.K = static_cast<const uint16_t*>(K);
  a.V = static_cast<const uint16_t*>(V);
  a.out = static_cast<uint16_t*>(out);
  a.ranges = grid.ranges;
  a.by_length = grid.by_length;
  a.part_o = static_cast<float*>(parts);
  a.part_mz = a.part_o ? a.part_o + (size_t)grid.workgroups * heads_of(rows) * d.d : nullptr;
  a.B = d.B; a.Hq = d.Hkv * rows; a.Hkv = d.Hkv; a.G = rows; a.k_cap = d.k_cap;
  a.page_size = d.page_size; a.num_pages = d.num_pages; a.max_pages = d.max_pages;
  a.head_groups = (rows + 63) / 64;
  a.units = a.Hkv * a.head_groups;
  a.wave_groups = heads_of(rows) / 16;
  a.page_magic = magic_of(d.page_size);
  a.q_sb = d.q_sb; a.q_sh = d.q_sh; a.c_sb = d.c_sb; a.c_sh = d.c_sh; a.c_st = d.c_st;
  a.scale = (float)(scale_of(d) * 1.4426950408889634);
  a.cap = make_cap(scale_of(d), d.cap);
}

}  // namespace
}  // namespace pkv
