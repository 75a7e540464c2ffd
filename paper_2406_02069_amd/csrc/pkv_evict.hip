// Eviction by accumulated weights, in place (include/pkv.h: pkv_cache_evict).
//
// Two launches.  The first, a workgroup per (sequence, KV head), finds the smallest weight that stays and pairs the rows behind the
// budget that stay with the holes before it, the i-th with the i-th by counting both (a prefix sum over waves): sources lie behind all
// destinations, so that the second can copy the pairs' rows in any order, in place, by two turns of workgroups at most.
// Up to 64 rows are moved by the first already, which is the only one where there can be no more.
// What bounds it: the first launch is one compute unit's time for a head, a few passes over 4-byte keys (pkv_topk.h) which stand in LDS
// for up to 32k rows and in L2, through the workspace, beyond; the second the copy.  d 128, 8 heads: one row too many of 2049 in 8
// sequences 6.7 us where the cache has room for no more, 10 in room for 4096 (the second launch finds nothing to do); 4 sequences of up to
// 32k rows to 2k 33 + 12 (keys formed again in each pass: 121), 131072 to 2048 122 (312 with keys formed again), four times that at once 136,
// 64 sequences of 4096 to 2048 145 (0.5 GB moved).
#include <string.h>

#include "pkv_long.h"
#include "pkv_topk.h"

namespace pkv {
namespace {

constexpr int kMovedHere = 64;  // rows that the first launch moves by itself
constexpr int kPairs = 32;      // of an item of the second launch

struct EvictArgs {
  char *K, *V;
  const int32_t *table, *count, *positions;
  const float* weights;
  int32_t* positions_out;
  float* weights_out;
  int32_t* count_out;
  int32_t* moves;  // [unit]
  int32_t* pairs;  // [unit][2][most]: destinations, sources
  uint32_t* keys;  // [unit][key_room], for more rows than LDS holds
  int64_t key_room;
  int32_t B, Hkv, d, k_cap, page_size, num_pages, max_pages, budget, recent, first, most;
  int32_t in_lds;  // keys that the launch has room for
  int32_t second;  // whether there is a second launch
  uint32_t page_magic;
  int64_t c_sb, c_sh, c_st, p_sb, p_sh, w_sb, w_sh, po_sb, po_sh, wo_sb, wo_sh;
};

// Where row j of a sequence and head lies, in bytes; -1: on a page that does not exist.
__device__ __forceinline__ int64_t row_at(const EvictArgs& a, int b, int g, int j) {
  if (a.page_size == 0) return (b * a.c_sb + g * a.c_sh + j * a.c_st) * 2;
  uint32_t p = __umulhi((uint32_t)j, a.page_magic);
  if ((uint32_t)j - p * a.page_size >= (uint32_t)a.page_size) ++p;
  const int32_t page = a.table[(int64_t)b * a.max_pages + p];
  if ((uint32_t)page >= (uint32_t)a.num_pages) return -1;
  return (((int64_t)page * a.Hkv + g) * a.page_size + (j - p * a.page_size)) * a.d * 2;
}

// A pair's rows of K and V, a 16-byte piece of each; left out where a page does not exist.
__device__ __forceinline__ void move_piece(const EvictArgs& a, int b, int g, int to, int from, int piece) {
  const int64_t dst = row_at(a, b, g, to), src = row_at(a, b, g, from);
  if (dst < 0 || src < 0) return;
  const u32x4 k = *reinterpret_cast<const u32x4*>(a.K + src + 16 * piece), v = *reinterpret_cast<const u32x4*>(a.V + src + 16 * piece);
  *reinterpret_cast<u32x4*>(a.K + dst + 16 * piece) = k;
  *reinterpret_cast<u32x4*>(a.V + dst + 16 * piece) = v;
}

// What a workgroup looks after: a sequence and KV head.
struct Unit {
  int unit, b, g, n;
  const int32_t* pos;
  const float* weight;
  int32_t* pos_out;
  float* weight_out;
};

// What becomes of a row that is not moved into: before the budget it stays (holes are filled later), behind it it is emptied.  Where the
// outputs are the inputs, the former is there already, and the latter waits until the moved rows have been read; where there is a second
// launch, its many workgroups empty the rows (32k rows to 2k, 4 sequences: 33.9 us instead of 32.8 for the first if it does that itself).
__device__ __forceinline__ void keep_row(const EvictArgs& a, const Unit& u, int r, int32_t p, float w) {
  const bool stays = r < a.budget;
  if (!stays && a.second) return;
  if (u.pos_out != u.pos) u.pos_out[r] = stays ? p : -1;
  if (u.weight_out != u.weight) u.weight_out[r] = stays ? w : 0.0f;
}

// Pairs are known: the rows' positions and weights follow, and few rows of K and V are moved here.
__device__ __forceinline__ void finish(const EvictArgs& a, const Unit& u, int late) {
  const int32_t *const to = a.pairs + (int64_t)u.unit * 2 * a.most, *const from = to + a.most;
  __threadfence_block();
  __syncthreads();
  for (int i = threadIdx.x; i < late; i += kThreads) {
    const int dst = to[i], src = from[i];
    const bool there = row_at(a, u.b, u.g, dst) >= 0 && row_at(a, u.b, u.g, src) >= 0;
    u.pos_out[dst] = there ? u.pos[src] : -1;
    u.weight_out[dst] = u.weight[src];
  }
  const bool here = late <= kMovedHere;
  if (threadIdx.x == 0) a.moves[u.unit] = here ? 0 : late;
  if (here) {
    const int lanes = a.d / 8;
    for (int i = threadIdx.x; i < late * lanes; i += kThreads) move_piece(a, u.b, u.g, to[i / lanes], from[i / lanes], i % lanes);
  }
  if (a.second || (u.pos_out != u.pos && u.weight_out != u.weight)) return;
  __syncthreads();
  for (int r = a.budget + threadIdx.x; r < u.n; r += kThreads) {
    if (u.pos_out == u.pos) u.pos_out[r] = -1;
    if (u.weight_out == u.weight) u.weight_out[r] = 0.0f;
  }
}

// A row's key: rows that are not there 1, weights that are NaN 2, protected rows the greatest (0: no row).
__device__ __forceinline__ uint32_t row_key(const EvictArgs& a, int32_t p, float w, int newest) {
  return p < 0 ? 1u : p < a.first || p > newest - a.recent ? kTop : w == w ? key_of_float(w) : 2u;
}
__device__ __forceinline__ int newest_of_all(int newest, SelectLds& lds) {
  newest = wave_max(newest);
  if ((threadIdx.x & 63) == 0) lds.sums[threadIdx.x >> 6][0] = newest;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWavesOf; ++w) newest = max(newest, lds.sums[w][0]);
  return newest;
}

// The pairs of a head, by the keys that key_at looks up.
template <typename KeyAt>
__device__ __forceinline__ void pair_rows(const EvictArgs& a, const Unit& u, KeyAt key_at, const Met& met, SelectLds& lds) {
  const Keys<KeyAt> keys(u.n, key_at);
  const Cutoff cut = cutoff_of(keys, met, a.budget, lds);
  const int equal0 = equal_before(keys, cut, lds);
  int equal = equal0, holes = 0, late = 0;
  const int lane = threadIdx.x & 63;
  keys.each([&](int r, const uint32_t(&key)[kBatch]) {
    bool in[kBatch];
    among_largest(key, cut, equal, in);
    const int r0 = __builtin_amdgcn_readfirstlane(r - lane);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int before = min(max(a.budget - r0 - 64 * i, 0), 64);  // of the 64 rows, in front of the budget
      const uint64_t stay = __ballot(in[i]), front = before == 64 ? ~(uint64_t)0 : ((uint64_t)1 << before) - 1;
      holes += before - __popcll(stay & front);
      late += __popcll(stay & ~front);
    }
  });
  lds.sums[this_wave()][1] = holes;
  lds.sums[this_wave()][2] = late;
  __syncthreads();
  const Before h = before_wave(lds, 1), l = before_wave(lds, 2);
  holes = h.mine;
  late = l.mine;
  equal = equal0;
  int32_t *const to = a.pairs + (int64_t)u.unit * 2 * a.most, *const from = to + a.most;
  keys.each([&](int r, const uint32_t(&key)[kBatch]) {
    bool in[kBatch];
    among_largest(key, cut, equal, in);
    const int r0 = __builtin_amdgcn_readfirstlane(r - lane);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int before = min(max(a.budget - r0 - 64 * i, 0), 64);
      const uint64_t stay = __ballot(in[i]), front = before == 64 ? ~(uint64_t)0 : ((uint64_t)1 << before) - 1;
      const uint64_t hs = ~stay & front, ls = stay & ~front;
      if (hs != 0) {
        if (hs >> lane & 1) to[holes + below_me(hs)] = r + 64 * i;
        holes += __popcll(hs);
      }
      if (ls != 0) {
        if (ls >> lane & 1) from[late + below_me(ls)] = r + 64 * i;
        late += __popcll(ls);
      }
    }
  });
  finish(a, u, l.all);  // (as many holes as late rows)
}

// Keys in LDS, from rows' positions and weights that are all requested together.
__device__ __forceinline__ void evict_rows(const EvictArgs& a, const Unit& u, uint32_t* kept, SelectLds& lds) {
  constexpr int MOST = kKeysInLds / kThreads;
  int32_t p[MOST];
  float w[MOST];
  int newest = -1;
#pragma unroll
  for (int i0 = 0; i0 < MOST; i0 += kBatch) {
    if (i0 * kThreads < u.n) {
#pragma unroll
      for (int i = i0; i < i0 + kBatch; ++i) p[i] = u.pos[min((int)threadIdx.x + i * kThreads, u.n - 1)];
#pragma unroll
      for (int i = i0; i < i0 + kBatch; ++i) w[i] = u.weight[min((int)threadIdx.x + i * kThreads, u.n - 1)];
    }
  }
#pragma unroll
  for (int i0 = 0; i0 < MOST; i0 += kBatch) {
    if (i0 * kThreads < u.n) {
#pragma unroll
      for (int i = i0; i < i0 + kBatch; ++i) newest = max(newest, p[i]);
    }
  }
  newest = newest_of_all(newest, lds);
  Met met;
#pragma unroll
  for (int i0 = 0; i0 < MOST; i0 += kBatch) {
    if (i0 * kThreads < u.n) {
#pragma unroll
      for (int i = i0; i < i0 + kBatch; ++i) {
        const int r = (int)threadIdx.x + i * kThreads;
        const uint32_t key = r < u.n ? row_key(a, p[i], w[i], newest) : 0u;
        met.meet(key);
        kept[r] = key;
        if (r < u.n) keep_row(a, u, r, p[i], w[i]);
      }
    }
  }
  pair_rows(a, u, [&](int r) { return kept[r]; }, met, lds);  // (its first barrier comes before the first look-up)
}
// Keys in memory, for more rows than LDS holds: once more than there, each pass goes over them in L2.
__device__ __forceinline__ void evict_many_rows(const EvictArgs& a, const Unit& u, SelectLds& lds) {
  uint32_t* const kept = a.keys + (int64_t)u.unit * a.key_room;
  int newest = -1;
  for (int r0 = threadIdx.x; r0 < u.n; r0 += kRun) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) newest = max(newest, u.pos[min(r0 + i * kThreads, u.n - 1)]);
  }
  newest = newest_of_all(newest, lds);
  Met met;
  for (int r0 = 0; r0 < u.n; r0 += kRun) {
    int32_t p[kBatch];
    float w[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int r = min(r0 + (int)threadIdx.x + i * kThreads, u.n - 1);
      p[i] = u.pos[r];
      w[i] = u.weight[r];
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int r = r0 + (int)threadIdx.x + i * kThreads;
      const uint32_t key = r < u.n ? row_key(a, p[i], w[i], newest) : 0u;
      met.meet(key);
      kept[r] = key;
      if (r < u.n) keep_row(a, u, r, p[i], w[i]);
    }
  }
  pair_rows(a, u, [&](int r) { return kept[r]; }, met, lds);  // (its first barrier comes before the first look-up)
}

// One row too many, as in a step of decoding: the row with the least key goes, the last of those that have it.  The last row, which
// takes its place, is requested before that is known.
__device__ __forceinline__ void evict_one(const EvictArgs& a, const Unit& u, SelectLds& lds) {
  const int lanes = a.d / 8, last = u.n - 1;
  const int64_t src = row_at(a, u.b, u.g, last);
  u32x4 k = (u32x4)(0), v = (u32x4)(0);
  if (src >= 0 && (int)threadIdx.x < lanes) {
    k = *reinterpret_cast<const u32x4*>(a.K + src + 16 * threadIdx.x);
    v = *reinterpret_cast<const u32x4*>(a.V + src + 16 * threadIdx.x);
  }
  const int32_t last_pos = u.pos[last];
  const float last_weight = u.weight[last];
  int newest = -1;
  for (int r0 = threadIdx.x; r0 < u.n; r0 += 4 * kThreads) {
#pragma unroll
    for (int i = 0; i < 4; ++i) newest = max(newest, u.pos[min(r0 + i * kThreads, last)]);
  }
  newest = newest_of_all(newest, lds);
  uint64_t least = ~(uint64_t)0;  // key and, descending, row
  const bool copy = u.pos_out != u.pos || u.weight_out != u.weight;
  for (int r0 = threadIdx.x; r0 < u.n; r0 += 4 * kThreads) {
    int32_t p[4];
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[i] = u.pos[min(r0 + i * kThreads, last)];
      w[i] = u.weight[min(r0 + i * kThreads, last)];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = min(r0 + i * kThreads, last);
      least = min(least, (uint64_t)row_key(a, p[i], w[i], newest) << 32 | (uint32_t)~r);
      if (copy && r < last) {
        u.pos_out[r] = p[i];
        u.weight_out[r] = w[i];
      }
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o));
  if ((threadIdx.x & 63) == 0) lds.keys[threadIdx.x >> 6] = least;
  __syncthreads();  // (also: what is copied has been)
#pragma unroll
  for (int w = 0; w < kWavesOf; ++w) least = min(least, lds.keys[w]);
  const int hole = (int)~(uint32_t)least;
  const int64_t dst = hole < last ? row_at(a, u.b, u.g, hole) : -1;
  const bool moved = src >= 0 && dst >= 0;
  if (moved && (int)threadIdx.x < lanes) {
    *reinterpret_cast<u32x4*>(a.K + dst + 16 * threadIdx.x) = k;
    *reinterpret_cast<u32x4*>(a.V + dst + 16 * threadIdx.x) = v;
  }
  if (threadIdx.x == 0) {
    if (hole < last) {
      u.pos_out[hole] = moved ? last_pos : -1;
      u.weight_out[hole] = last_weight;
    }
    u.pos_out[last] = -1;
    u.weight_out[last] = 0.0f;
    a.moves[u.unit] = 0;
  }
}

__global__ __launch_bounds__(kThreads) void evict_select_kernel(const EvictArgs a) {
  __shared__ SelectLds lds;
  extern __shared__ uint32_t kept[];
  Unit u;
  u.unit = blockIdx.x;
  u.b = u.unit / a.Hkv;
  u.g = u.unit % a.Hkv;
  u.n = min(max(a.count[u.b], 0), a.k_cap);
  u.pos = a.positions + u.b * a.p_sb + u.g * a.p_sh;
  u.weight = a.weights + u.b * a.w_sb + u.g * a.w_sh;
  u.pos_out = a.positions_out + u.b * a.po_sb + u.g * a.po_sh;
  u.weight_out = a.weights_out + u.b * a.wo_sb + u.g * a.wo_sh;
  if (u.g == 0 && threadIdx.x == 0 && a.count_out) a.count_out[u.b] = min(u.n, a.budget);
  if (u.n <= a.budget) {
    if (u.pos_out != u.pos || u.weight_out != u.weight) {
      for (int r = threadIdx.x; r < u.n; r += kThreads) {
        u.pos_out[r] = u.pos[r];
        u.weight_out[r] = u.weight[r];
      }
    }
    if (threadIdx.x == 0) a.moves[u.unit] = 0;
  } else if (u.n == a.budget + 1) {
    evict_one(a, u, lds);
  } else if (u.n <= a.in_lds) {
    evict_rows(a, u, kept, lds);
  } else {
    evict_many_rows(a, u, lds);
  }
}

// An item: `share` rows of K and of V of a head, 16 bytes a thread at a time, and its share of the rows that are emptied.
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs a, int chunks, int share, Items items) {
  const int lanes = a.d / 8;
  auto rows_of = [&](int b) { return min(max(a.count[b], 0), a.k_cap); };
  auto has = [&](int unit, int chunk) {
    const int moves = a.moves[unit], n = rows_of(unit / a.Hkv);
    return (int64_t)chunk * share < moves || a.budget + (int64_t)chunk * 256 < n;
  };
  each_item(items, blockIdx.x, gridDim.x, has, [&](int unit, int chunk) {
    const int b = unit / a.Hkv, g = unit % a.Hkv, moves = a.moves[unit], n = rows_of(b);
    int32_t* const pos_out = a.positions_out + b * a.po_sb + g * a.po_sh;
    float* const weight_out = a.weights_out + b * a.wo_sb + g * a.wo_sh;
    for (int64_t r = a.budget + (int64_t)chunk * 256 + threadIdx.x; r < n; r += (int64_t)chunks * 256) {
      pos_out[r] = -1;
      weight_out[r] = 0.0f;
    }
    const int32_t *const to = a.pairs + (int64_t)unit * 2 * a.most, *const from = to + a.most;
    for (int i = threadIdx.x; i < share * lanes; i += 256) {
      const int p = chunk * share + i / lanes;
      if (p >= moves) break;
      move_piece(a, b, g, to[p], from[p], i % lanes);
    }
  });
}

int check_evict_desc(const pkv_evict_desc* desc) {
  if (!desc) return PKV_ERR_INVALID_ARG;
  const pkv_evict_desc& d = *desc;
  if (d.B < 1 || d.Hkv < 1 || d.budget < 1 || d.recent < 0 || d.first < 0 || (int64_t)d.first + d.recent > d.budget ||
      check_pages(d) != PKV_OK)
    return PKV_ERR_INVALID_ARG;
  if (d.p_sb < 0 || d.p_sh < 0 || d.w_sb < 0 || d.w_sh < 0 || d.po_sb < 0 || d.po_sh < 0 || d.wo_sb < 0 || d.wo_sh < 0) return PKV_ERR_INVALID_ARG;
  if ((int64_t)d.B * d.Hkv >= 1 << 22) return PKV_ERR_UNSUPPORTED;  // (workgroups of 1024: 2^32 threads)
  return check_cache_limits(d);
}

// Pairs that a head can have.
int64_t most_moves(const pkv_evict_desc& d) {
  const int64_t behind = (int64_t)d.k_cap - d.budget;
  return behind < 0 ? 0 : behind < d.budget ? behind : d.budget;
}

// Keys of a head that wait in memory.
int64_t room_of_keys(const pkv_evict_desc& d) { return d.k_cap <= kKeysInLds ? 0 : ((int64_t)d.k_cap + kRun - 1) / kRun * kRun; }

}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

size_t pkv_evict_workspace_bytes(const pkv_evict_desc* desc) {
  if (check_evict_desc(desc) != PKV_OK) return 0;
  return (size_t)desc->B * desc->Hkv * (1 + 2 * (size_t)most_moves(*desc) + (size_t)room_of_keys(*desc)) * sizeof(int32_t);
}

int pkv_cache_evict(const pkv_evict_desc* desc, void* K_cache, void* V_cache, const int32_t* block_table, const int32_t* count,
                    const int32_t* positions, const float* weights, int32_t* positions_out, float* weights_out, int32_t* count_out,
                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc || !K_cache || !V_cache || !count || !positions || !weights || !positions_out || !weights_out) return PKV_ERR_INVALID_ARG;
  const int rc = check_evict_desc(desc);
  if (rc != PKV_OK) return rc;
  const pkv_evict_desc& d = *desc;
  if (!aligned(K_cache, 16) || !aligned(V_cache, 16) || !aligned(block_table, 4) || !aligned(count, 4) || !aligned(positions, 4) ||
      !aligned(weights, 4) || !aligned(positions_out, 4) || !aligned(weights_out, 4) || !aligned(count_out, 4))
    return PKV_ERR_INVALID_ARG;
  if (d.page_size > 0 && !block_table) return PKV_ERR_INVALID_ARG;
  if (!apart(d.k_cap, {{d.B, d.po_sb}, {d.Hkv, d.po_sh}}) || !apart(d.k_cap, {{d.B, d.wo_sb}, {d.Hkv, d.wo_sh}})) return PKV_ERR_INVALID_ARG;
  if (d.page_size == 0 && !apart(d.d, {{d.B, d.c_sb}, {d.Hkv, d.c_sh}, {d.k_cap, d.c_st}})) return PKV_ERR_INVALID_ARG;
  if (positions_out == positions && (d.po_sb != d.p_sb || d.po_sh != d.p_sh)) return PKV_ERR_INVALID_ARG;
  if (weights_out == weights && (d.wo_sb != d.w_sb || d.wo_sh != d.w_sh)) return PKV_ERR_INVALID_ARG;
  if (count_out == count) return PKV_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < pkv_evict_workspace_bytes(desc)) return PKV_ERR_WORKSPACE;
  EvictArgs a;
  memset(&a, 0, sizeof(a));
  const int units = d.B * d.Hkv;
  a.K = static_cast<char*>(K_cache);
  a.V = static_cast<char*>(V_cache);
  a.table = block_table; a.count = count; a.positions = positions; a.weights = weights;
  a.positions_out = positions_out; a.weights_out = weights_out; a.count_out = count_out;
  a.moves = static_cast<int32_t*>(workspace);
  a.pairs = a.moves + units;
  a.B = d.B; a.Hkv = d.Hkv; a.d = d.d; a.k_cap = d.k_cap; a.page_size = d.page_size; a.num_pages = d.num_pages;
  a.max_pages = d.max_pages; a.budget = d.budget; a.recent = d.recent; a.first = d.first;
  a.most = (int32_t)most_moves(d);
  a.key_room = room_of_keys(d);
  a.keys = reinterpret_cast<uint32_t*>(a.pairs + (size_t)units * 2 * a.most);
  a.page_magic = magic_of(d.page_size);
  a.c_sb = d.c_sb; a.c_sh = d.c_sh; a.c_st = d.c_st; a.p_sb = d.p_sb; a.p_sh = d.p_sh; a.w_sb = d.w_sb; a.w_sh = d.w_sh;
  a.po_sb = d.po_sb; a.po_sh = d.po_sh; a.wo_sb = d.wo_sb; a.wo_sh = d.wo_sh;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  a.in_lds = keys_in_lds(d.k_cap);
  a.second = a.most > kMovedHere;
  static bool granted[kMaxDevices];
  if (grant_keys(reinterpret_cast<const void*>(evict_select_kernel), granted) != hipSuccess) return PKV_ERR_HIP;
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)units), dim3(kThreads), (size_t)a.in_lds * sizeof(uint32_t), st, a);
  if (hipGetLastError() != hipSuccess) return PKV_ERR_HIP;
  if (!a.second) return PKV_OK;
  int64_t share = kPairs;
  while (units * ((a.most + share - 1) / share) > kMostItems) share *= 2;
  const int chunks = (int)((a.most + share - 1) / share);
  const Items items = items_of(units, chunks);
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)workgroups_of(items)), dim3(256), 0, st, a, chunks, (int)share, items);
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_HIP;
}

}  // extern "C"
