// Work lists of causal attention (t2v_causal.h): no HIP, compiled with g++ for CPU tests too.
#include "t2v_causal.h"

#include <algorithm>
#include <cmath>

#include "../../include/t2vattn.h"
#include "t2v_host.h"

namespace t2v {

namespace {

constexpr size_t kGroupedRounds = 8;  // of items, from which a die keeps groups together
constexpr double kAway = 0.05;        // of a die's share, for which an item leaves its group

// Tiles and the loop of tile t of one (sequence, key head).
struct Loops {
  CausalKernel kind;
  int32_t lq, lk;
  int group, block, stage;
  int tiles() const {
    const int64_t rows = kind == kCausalDkdv ? lk : static_cast<int64_t>(lq) * group;
    return static_cast<int>((rows + block - 1) / block);
  }
  int32_t length(int t) const {
    const int64_t r0 = static_cast<int64_t>(t) * block;
    if (kind == kCausalDkdv) return group * causal_stages(static_cast<int32_t>(r0), lq, lk, stage);
    const int64_t last = std::min<int64_t>(r0 + block, static_cast<int64_t>(lq) * group) - 1;
    return causal_keys(static_cast<int32_t>(last / group), lq, lk);
  }
};

Loops loops_of(CausalKernel kind, const CausalShape& a, int s, int block, int stage) {
  return {kind, a.cu_q[s + 1] - a.cu_q[s], a.cu_k[s + 1] - a.cu_k[s], a.group, block, stage};
}

// Equal pieces of a loop of n units cut at chunk: *count of *step units, the last shorter.
void pieces_of(CausalKernel kind, int n, int chunk, int* count, int* step) {
  *count = 1;
  *step = n;
  if (chunk <= 0 || n <= chunk) return;
  const int unit = kind == kCausalDkdv ? 1 : 64;
  const int most = (n + chunk - 1) / chunk;
  *step = ((n + most - 1) / most + unit - 1) / unit * unit;
  *count = (n + *step - 1) / *step;
}

}  // namespace

CausalList build_causal_list(CausalKernel kind, const CausalShape& a, int block, int stage, int order, int chunk,
                             double fixed, int workers) {
  CausalList out;
  // The items of one key head of a sequence, the same for each of its key heads but for head and slots.
  struct Sequence {
    size_t first;  // in `items`
    int n, slots;
    int64_t slot0;
    double longest, cost;
  };
  std::vector<CausalItem> items;
  std::vector<Sequence> seqs;
  size_t n = 0;
  for (int s = 0; s < a.nseq; ++s) {
    const Loops l = loops_of(kind, a, s, block, stage);
    const int tiles = l.tiles();
    if (tiles == 0) continue;
    Sequence q{items.size(), 0, 0, out.slots, 0.0, 0.0};
    for (int i = 0; i < tiles; ++i) {
      // Longest loop first: rows from the last tile, keys from the first.
      const int t = order == T2V_ORDER_NATURAL || kind == kCausalDkdv ? i : tiles - 1 - i;
      const int len = l.length(t);
      int count = 1, step = len;
      pieces_of(kind, len, chunk, &count, &step);
      CausalItem it{a.cu_q[s], l.lq, a.cu_k[s], l.lk, t * block, 0, 0, len, -1, count, 0, 0};
      for (int p = 0; p < count; ++p) {
        it.begin = p * step;
        it.end = std::min(len, (p + 1) * step);
        if (count > 1) it.slot = q.slots++;
        items.push_back(it);
        const double c = fixed + (it.end - it.begin);
        q.cost += c;
        q.longest = std::max(q.longest, c);
      }
    }
    q.n = static_cast<int>(items.size() - q.first);
    n += static_cast<size_t>(q.n) * a.kv_heads;
    out.slots += static_cast<int64_t>(q.slots) * a.kv_heads;
    seqs.push_back(q);
  }
  auto item_of = [&](const Sequence& q, int head, size_t i) {
    CausalItem it = items[q.first + i];
    it.head = head;
    if (it.slot >= 0) it.slot += static_cast<int32_t>(q.slot0 + static_cast<int64_t>(q.slots) * head);
    return it;
  };
  for (const Sequence& q : seqs)
    for (int h = 0; q.slots > 0 && h < a.kv_heads; ++h)
      for (int i = 0; i < q.n; i += items[q.first + i].pieces)
        if (items[q.first + i].pieces > 1) {
          CausalItem r = item_of(q, h, i);
          r.begin = r.end = 0;
          out.reduce.push_back(r);
        }
  out.items.reserve(n);
  if (order == T2V_ORDER_NATURAL) {
    for (const Sequence& q : seqs)
      for (int h = 0; h < a.kv_heads; ++h)
        for (int i = 0; i < q.n; ++i) out.items.push_back(item_of(q, h, i));
    return out;
  }
  // Workgroup b runs on die b % 8, whose L2 serves the keys or queries of a (sequence, key head) to all its tiles there.
  double total = 0.0;
  for (const Sequence& q : seqs) total += q.cost * a.kv_heads;
  const double share = total / kNumXcd * (1.0 + 1e-9);
  const size_t per_die = static_cast<size_t>(std::max(workers, 1) + kNumXcd - 1) / kNumXcd;
  struct Ref {
    int32_t length, seq, head, item;
  };
  std::vector<Ref> q[kNumXcd];
  double load[kNumXcd] = {};
  auto cost_of = [&](const CausalItem& it) { return fixed + (it.end - it.begin); };
  auto longer = [](const Ref& x, const Ref& y) { return x.length > y.length; };
  if (n < kGroupedRounds * kNumXcd * per_die) {
    // Few rounds: the longest first, and each die its share of long and short ones (a long one that starts in the last round
    // would outlast the others). Each item to the least loaded die, where one that has none of its group
    // counts as loaded by kAway of a share more. (9,999 tokens, 3 heads over 1, cut into 353 items: 109 us against 128
    // with whole groups on one die after the other; 20,280 tokens, 2 heads of 64, 476 items: 153 against 182.)
    std::vector<Ref> order;
    for (size_t s = 0; s < seqs.size(); ++s)
      for (int i = 0; i < seqs[s].n; ++i) {
        const CausalItem& it = items[seqs[s].first + i];
        order.push_back({it.end - it.begin, static_cast<int32_t>(s), 0, i});
      }
    std::stable_sort(order.begin(), order.end(), longer);
    std::vector<unsigned char> here(seqs.size() * a.kv_heads, 0);  // bit x: die x has items of the group
    for (Ref r : order) {
      const double c = cost_of(items[seqs[r.seq].first + r.item]);
      for (r.head = 0; r.head < a.kv_heads; ++r.head) {
        unsigned char& h = here[static_cast<size_t>(r.seq) * a.kv_heads + r.head];
        int best = 0;
        double least = HUGE_VAL;
        for (int x = 0; x < kNumXcd; ++x) {
          const double l = load[x] + (h >> x & 1 ? 0.0 : kAway * share);
          if (l < least) {
            least = l;
            best = x;
          }
        }
        h |= 1u << best;
        load[best] += c;
        q[best].push_back(r);
      }
    }
  } else {
    // Many rounds: a group goes to one die, longest tiles first; groups by their longest loop, each to the least loaded die,
    // and on to the next when that die has an even share of the cost. The shortest two rounds are kept for the end, and
    // the others stay with their group. (From eight rounds on the two orders differ by less than 1%, either way.)
    std::vector<int> by_length(seqs.size());
    for (size_t i = 0; i < seqs.size(); ++i) by_length[i] = static_cast<int>(i);
    std::stable_sort(by_length.begin(), by_length.end(), [&](int x, int y) { return seqs[x].longest > seqs[y].longest; });
    for (int s : by_length)
      for (int h = 0; h < a.kv_heads; ++h) {
        int x = static_cast<int>(std::min_element(load, load + kNumXcd) - load);
        for (int i = 0; i < seqs[s].n; ++i) {
          const CausalItem& it = items[seqs[s].first + i];
          const double c = cost_of(it);
          if (load[x] + 0.5 * c > share) x = static_cast<int>(std::min_element(load, load + kNumXcd) - load);
          q[x].push_back({it.end - it.begin, s, h, i});
          load[x] += c;
        }
      }
    std::vector<int32_t> lengths;
    for (auto& l : q) {
      if (l.size() < 2 * per_die) {
        std::stable_sort(l.begin(), l.end(), longer);
        continue;
      }
      lengths.clear();
      for (const Ref& r : l) lengths.push_back(r.length);
      std::nth_element(lengths.begin(), lengths.begin() + 2 * per_die - 1, lengths.end());
      const int32_t cut = lengths[2 * per_die - 1];
      const auto last = std::stable_partition(l.begin(), l.end(), [cut](const Ref& x) { return x.length > cut; });
      std::stable_sort(last, l.end(), longer);
    }
  }
  // One list: position b takes the next item of die b % 8, or, when that die has no more, the last
  // (shortest) item of the die with the most left, so that no position is empty.
  size_t next[kNumXcd] = {};
  for (size_t b = 0; b < n; ++b) {
    size_t x = b % kNumXcd;
    Ref r;
    if (next[x] < q[x].size()) {
      r = q[x][next[x]++];
    } else {
      for (size_t y = 0; y < kNumXcd; ++y)
        if (q[y].size() - next[y] > q[x].size() - next[x]) x = y;
      r = q[x].back();
      q[x].pop_back();
    }
    out.items.push_back(item_of(seqs[r.seq], r.head, r.item));
  }
  return out;
}

namespace {

// Time of the list cut at `chunk`. An item shares the GPU (its CU, or its power) with others for their mean length, and
// is faster after that. With a worker for every item: the longest's. Else the even share of all items, and, where they
// are of like length, what a part-empty last round costs (the longest go first; others fit together). And the join, which
// goes over a row's pieces in turn. Infinite when it would need more than max_slots slots. Of the cuts of ten lists
// measured at 10 cuts each, the least estimate was 1.4% slower than the best cut in the mean, 6.5% at most.
double causal_time(CausalKernel kind, const CausalShape& a, int block, int stage, const CausalCost& cost, int chunk,
                   int64_t max_slots, int64_t* items, double* longest) {
  double keys = 0.0, bytes = 0.0;  // loop lengths, and the pieces' results
  int64_t n = 0, slots = 0;
  int most = 0, deep = 1;
  for (int s = 0; s < a.nseq; ++s) {
    const Loops l = loops_of(kind, a, s, block, stage);
    const int tiles = l.tiles();
    const int64_t rows = kind == kCausalDkdv ? l.lk : static_cast<int64_t>(l.lq) * l.group;
    for (int t = 0; t < tiles; ++t) {
      int count = 1, step = 0;
      const int len = l.length(t);
      pieces_of(kind, len, chunk, &count, &step);
      keys += len;
      n += count;
      most = std::max(most, step);
      deep = std::max(deep, count);
      if (count > 1) {
        slots += count;
        bytes += static_cast<double>(count) * std::min<int64_t>(block, rows - static_cast<int64_t>(t) * block) * cost.slot_row;
      }
    }
  }
  n *= a.kv_heads;
  slots *= a.kv_heads;
  if (items != nullptr) *items = n;
  if (longest != nullptr) *longest = most;
  if (n == 0) return 0.0;
  if (slots > max_slots) return HUGE_VAL;
  // An item's speed follows from how many share its CU.
  const double per_cu = static_cast<double>(cost.workers) / cost.cus;
  const double beside = std::min(per_cu, std::ceil(static_cast<double>(n) / cost.cus));
  const double unit = beside < per_cu ? cost.alone + (cost.unit - cost.alone) * (beside - 1.0) / (per_cu - 1.0)
                                      : n <= cost.cus ? cost.alone + (cost.unit - cost.alone) * n / cost.cus : cost.unit;
  const double mean = keys * a.kv_heads / n, alike = std::max(0.0, 2.0 * mean - most);
  const double share = (unit * keys * a.kv_heads + cost.fixed * n) / cost.workers;
  const double one = cost.fixed + unit * mean + cost.alone * (most - mean);
  const double rounds = static_cast<double>(n) / cost.workers, idle = 0.3 + 0.7 * (std::ceil(rounds) - rounds);
  const double run = n <= cost.workers ? one : std::max(one, share + idle * (cost.fixed + 0.5 * (unit + cost.alone) * alike));
  return run + (slots > 0 ? cost.join + cost.piece * deep + cost.byte * bytes * a.kv_heads : 0.0);
}

}  // namespace

int causal_chunk(CausalKernel kind, const CausalShape& a, int block, int stage, const CausalCost& cost, int least,
                 int64_t max_slots, double* time) {
  int64_t items = 0;
  double longest = 0.0;
  double best = causal_time(kind, a, block, stage, cost, 0, max_slots, &items, &longest);
  int chunk = 0;
  // Many rounds of items none of which is long: nothing to gain.
  if (items < 8 * static_cast<int64_t>(cost.workers) || cost.fixed + cost.unit * longest > 0.25 * best) {
    for (int n : {2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64, 96, 128, 192, 256, 384, 512}) {
      const int cut = static_cast<int>((longest + n - 1) / n);
      if (cut < least) break;
      const double t = causal_time(kind, a, block, stage, cost, cut, max_slots, nullptr, nullptr);
      if (t < best) {
        best = t;
        chunk = cut;
      }
    }
  }
  if (time != nullptr) *time = best;
  return chunk;
}

std::string check_causal_items(CausalKernel kind, const CausalItem* items, int n, const CausalShape& a, int block,
                               int stage, int64_t max_slots, bool reduce) {
  for (int i = 0; i < n; ++i) {
    const CausalItem& it = items[i];
    auto bad = [&](const char* what) {
      return "item " + std::to_string(i) + " {qrow0 " + std::to_string(it.qrow0) + ", lq " + std::to_string(it.lq) +
             ", krow0 " + std::to_string(it.krow0) + ", lk " + std::to_string(it.lk) + ", tile0 " +
             std::to_string(it.tile0) + ", head " + std::to_string(it.head) + ", begin " + std::to_string(it.begin) +
             ", end " + std::to_string(it.end) + ", slot " + std::to_string(it.slot) + ", pieces " +
             std::to_string(it.pieces) + "}: " + what;
    };
    int s = 0;
    while (s < a.nseq && !(a.cu_q[s] == it.qrow0 && a.cu_q[s + 1] - a.cu_q[s] == it.lq && a.cu_k[s] == it.krow0 &&
                           a.cu_k[s + 1] - a.cu_k[s] == it.lk))
      ++s;
    if (s == a.nseq) return bad("its rows and keys are no sequence's");
    const Loops l = loops_of(kind, a, s, block, stage);
    if (it.tile0 < 0 || it.tile0 % block != 0 || it.tile0 / block >= l.tiles()) return bad("tile0 is outside");
    if (it.head < 0 || it.head >= a.kv_heads) return bad("head is out of range");
    if (reduce ? it.slot < 0 || it.pieces < 2 || it.slot + static_cast<int64_t>(it.pieces) > max_slots
               : it.slot < -1 || it.slot >= max_slots || (it.slot < 0) != (it.pieces == 1))
      return bad("partial slots are out of range");
    const int len = l.length(it.tile0 / block);
    if (!reduce && (it.begin < 0 || it.end < it.begin || it.end > len || (it.begin == it.end && len > 0)))
      return bad("the loop leaves the rows that the tile sees");
    if (!reduce && it.slot < 0 && (it.begin != 0 || it.end != len)) return bad("an uncut loop must be whole");
  }
  return std::string();
}

}  // namespace t2v
