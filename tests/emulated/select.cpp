// The selection of csrc/pkv_topk.h by an emulated workgroup whose waves run in one order after another, against a sort.
//   select N K TOPS LEVELS SEED: N keys of LEVELS different values (0: any), TOPS of them protected, of which K are taken.
#include "pkv_topk.h"

#include <algorithm>
#include <numeric>
#include <random>

int main(int argc, char** argv) {
  if (argc != 6) return 2;
  const int n = atoi(argv[1]), k = atoi(argv[2]), tops = atoi(argv[3]), levels = atoi(argv[4]);
  std::mt19937 rng((unsigned)atoi(argv[5]));
  const int room = (n + pkv::kRun - 1) / pkv::kRun * pkv::kRun;
  std::vector<uint32_t> keys(room, 0u);
  for (int i = 0; i < n; ++i) keys[i] = levels ? 0x80000000u + rng() % levels : 1 + rng() % 0xFFFFFFFEu;
  std::vector<int> rows(n);
  std::iota(rows.begin(), rows.end(), 0);
  std::shuffle(rows.begin(), rows.end(), rng);
  for (int i = 0; i < tops; ++i) keys[rows[i]] = pkv::kTop;
  std::vector<int> want(n);
  std::iota(want.begin(), want.end(), 0);
  std::stable_sort(want.begin(), want.end(), [&](int a, int b) { return keys[a] > keys[b]; });
  want.resize(k);
  std::sort(want.begin(), want.end());

  for (int order = 0; order < 4; ++order) {
    std::vector<int> rank(16);
    std::iota(rank.begin(), rank.end(), 0);
    if (order == 1) std::reverse(rank.begin(), rank.end());
    if (order > 1) std::shuffle(rank.begin(), rank.end(), rng);
    pkv::SelectLds lds;
    memset(&lds, 0xFF, sizeof(lds));
    std::vector<int> got(k, -1);
    bool inside = true;
    const bool ended = emulated::run(rank, 200, [&]() {
      pkv::Met met;
      for (int i = threadIdx.x; i < room; i += pkv::kThreads) met.meet(keys[i]);
      auto key_at = [&](int i) { return keys[i]; };
      const pkv::Keys<decltype(key_at)> all(n, key_at);
      const pkv::Cutoff cut = pkv::cutoff_of(all, met, k, lds);
      const int equal0 = pkv::equal_before(all, cut, lds);
      int equal = equal0, taken = 0;
      all.each([&](int, const uint32_t(&key)[pkv::kBatch]) {
        bool in[pkv::kBatch];
        pkv::among_largest(key, cut, equal, in);
        for (int i = 0; i < pkv::kBatch; ++i) taken += __popcll(__ballot(in[i]));
      });
      lds.sums[pkv::this_wave()][2] = taken;
      __syncthreads();
      taken = pkv::before_wave(lds, 2).mine;
      equal = equal0;
      all.each([&](int r, const uint32_t(&key)[pkv::kBatch]) {
        bool in[pkv::kBatch];
        pkv::among_largest(key, cut, equal, in);
        for (int i = 0; i < pkv::kBatch; ++i) {
          const uint64_t some = __ballot(in[i]);
          const int at = taken + pkv::below_me(some);
          if (in[i] && (at < 0 || at >= k)) inside = false;
          if (in[i] && at >= 0 && at < k) got[at] = r + 64 * i;
          taken += __popcll(some);
        }
      });
    });
    if (!ended || !inside || got != want) {
      printf("order %d: %s\n", order, !ended ? "waves wait for one another" : !inside ? "more than k are taken" : "other keys are taken");
      return 1;
    }
  }
  return 0;
}
