// Host test of the causal work lists (no HIP): every tile's loop is covered once, partial slots are used once,
// the checks accept what the planner builds and report fields out of range, and cutting pays by the estimate.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <tuple>
#include <vector>

#include "../paper_2607_01701_amd/csrc/t2v_causal.h"

using namespace t2v;

static void require(bool ok, const char* what) {
  if (!ok) {
    std::printf("failed: %s\n", what);
    std::exit(1);
  }
}

int main() {
  std::mt19937 rng(7);
  auto draw = [&](int lo, int hi) { return lo + static_cast<int>(rng() % static_cast<unsigned>(hi - lo + 1)); };
  int changed = 0, lists = 0;
  for (int round = 0; round < 400; ++round) {
    const int nseq = draw(0, 6), group = draw(1, 7), kv = draw(1, 4);
    std::vector<int32_t> cq{0}, ck{0};
    for (int s = 0; s < nseq; ++s) {
      const int lk = draw(0, 3) == 0 ? draw(0, 3) : draw(0, 3000);
      cq.push_back(cq.back() + (draw(0, 1) ? lk : draw(0, 400)));
      ck.push_back(ck.back() + lk);
    }
    const CausalShape a{cq.data(), ck.data(), nseq, kv, group};
    for (CausalKernel kind : {kCausalFwd, kCausalDkdv, kCausalDq}) {
      const bool keys = kind == kCausalDkdv;
      const int block = keys ? 128 << draw(0, 1) : 32 << (draw(0, 1) ? draw(2, 3) : 0), stage = 32 << draw(0, 2);
      CausalCost cost{keys ? 2.0 : 0.03, keys ? 2.0 : 0.02, 4.0, 16, 16 * draw(1, 2), 1.0, 0.1, 1e-6, 64};
      double plain = 0.0, cut = 0.0;
      const int none = causal_chunk(kind, a, block, stage, cost, keys ? 1 : 64, 0, &plain);
      const int64_t most = draw(0, 1) ? 1 << 20 : draw(0, 40);
      const int chunk = causal_chunk(kind, a, block, stage, cost, keys ? 1 : 64, most, &cut);
      require(none == 0 && cut <= plain, "the cut is estimated to be faster, and none is made without slots");
      const int order = draw(0, 1);
      CausalList l = build_causal_list(kind, a, block, stage, order, chunk, 10.0, cost.workers);
      ++lists;
      require(l.slots <= most || l.slots == 0, "slots within the limit");
      std::map<std::tuple<int, int, int, int>, std::vector<std::pair<int, int>>> loops;
      std::set<int> slots;
      for (const CausalItem& it : l.items) {
        loops[{it.qrow0, it.krow0, it.head, it.tile0}].push_back({it.begin, it.end});
        if (it.slot >= 0) require(slots.insert(it.slot).second, "a slot is written once");
      }
      require(static_cast<int64_t>(slots.size()) == l.slots, "all slots are written");
      size_t want = 0;
      for (int s = 0; s < nseq; ++s) {
        const int lq = cq[s + 1] - cq[s], lk = ck[s + 1] - ck[s];
        const int rows = keys ? lk : lq * group;
        for (int h = 0; h < kv; ++h)
          for (int t = 0; t * block < rows; ++t) {
            ++want;
            // What the tile sees, by the definition.
            int len = 0;
            if (keys) {
              int first = lq;
              for (int i = 0; i < lq; ++i)
                if (t * block <= i + lk - lq) {
                  first = i;
                  break;
                }
              len = group * ((lq - first + stage - 1) / stage);
            } else {
              const int i = (std::min(rows, (t + 1) * block) - 1) / group;
              len = std::max(0, std::min(lk, i + 1 + lk - lq));
            }
            auto it = loops.find({cq[s], ck[s], h, t * block});
            require(it != loops.end(), "every tile has an item");
            std::sort(it->second.begin(), it->second.end());
            int at = 0;
            for (const auto& p : it->second) {
              require(p.first == at && (p.second > p.first || len == 0), "pieces follow each other");
              at = p.second;
            }
            require(at == len, "the loop covers what the tile sees");
          }
      }
      require(loops.size() == want, "no other tiles");
      const int n = static_cast<int>(l.items.size()), nr = static_cast<int>(l.reduce.size());
      require(check_causal_items(kind, l.items.data(), n, a, block, stage, l.slots, false).empty(), "a list passes");
      require(check_causal_items(kind, l.reduce.data(), nr, a, block, stage, l.slots, true).empty(), "a join list passes");
      for (int i = 0; i < std::min(n, 3); ++i)
        for (int f = 0; f < (l.items[i].slot < 0 ? 10 : 9); ++f) {  // only the join list's pieces are read
          std::vector<CausalItem> bad = l.items;
          int32_t* field = &bad[i].qrow0 + f;
          *field += f == 6 ? -(1 << 20) : 1 << 20;
          require(!check_causal_items(kind, bad.data(), n, a, block, stage, l.slots, false).empty(), "a field out of range is reported");
          ++changed;
        }
    }
  }
  std::printf("ok: %d lists, %d fields out of range reported\n", lists, changed);
  return 0;
}
