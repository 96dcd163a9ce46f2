// Division of paged attention among workgroups (csrc/t2v_paged.h) on random batches: every key of every tile is taken by exactly one
// share, pieces fill their slots and no others, no piece is shorter than the rule allows.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <vector>

#include "../paper_2607_01701_amd/csrc/t2v_paged.h"

using namespace t2v;

static void fail(const char* what, int n) {
  std::printf("batch %d: %s\n", n, what);
  std::exit(1);
}

static void quotients() {
  std::mt19937_64 g(6);
  for (int i = 0; i < 2000000; ++i) {
    const int64_t b = 1 + static_cast<int64_t>(g() >> (12 + g() % 52)), q = g() % 60000;
    if (b > (int64_t(1) << 52) / (q + 1)) continue;
    for (int64_t a : {q * b, q * b + b - 1, q * b + static_cast<int64_t>(g() % b)})
      if (paged_ratio(a, b) != q) fail("a quotient", i);
  }
}

// Every workgroup has one place on one line; a line's shares cover it, and none is too short.
static void roles() {
  std::mt19937 g(7);
  for (int n = 0; n < 3000; ++n) {
    const int groups = n % 3 ? 8 * (1 + g() % 100) : 2 + g() % 40;
    const int64_t few = g() % 5 ? g() : 0, many = g() % 5 ? g() : 0;
    const int m = paged_many(groups, few, many, 0.5f + (g() % 8) * 0.25f);
    if (m < 0 || m > groups || (many && !m) || (few && m == groups) || (!many && m)) fail("roles", n);
    std::vector<std::vector<int>> seen[2];
    for (auto& x : seen) x.assign(8, std::vector<int>(groups, 0));
    for (int b = 0; b < groups; ++b) {
      const PagedRole r = paged_role(b, groups, m);
      const int dies = paged_by_die(groups) ? 8 : 1, each = (r.many ? m : groups - m) / dies;
      if (r.x < 0 || r.x >= dies || r.i < 0 || r.i >= each || seen[r.many][r.x][r.i]++) fail("a place of no or two workgroups", n);
      if (dies == 8 && r.x != b % 8) fail("a place on another die", n);
    }
    const int64_t total = (int64_t(1) << (g() % 52)) + g();
    const PagedRule rule = paged_rule(1, 32, 128, 128, 1, 1 + g() % 300, kPagedFew, 32);
    const int taken = m ? m : groups;
    const PagedShares s = paged_shares(rule, total, taken, groups);
    const int64_t count = int64_t(s.dies) * s.each, least = int64_t(rule.share) * 256;
    if (s.each < 1 || count > taken || s.length * count < total || s.length < least) fail("shares of a line", n);
    if (s.length > std::max(least, total / count + 256)) fail("a share's length", n);
    if (count < taken && s.length > least + total / count / rule.share) fail("workgroups without a share", n);
  }
}

// Offsets that decrease give many sequences the queries of one: the line's length stays within what is counted, or there is no work.
static void long_lines() {
  const PagedRule few = paged_rule(16, 32, 128, 128, 256, 128, kPagedFew, 32), many = paged_rule(16, 128, 64, 128, 256, 128, kPagedMany, 32);
  // Every second sequence has 1,024 tiles of a little more than 2^30 keys, 2^48 positions: 16 of them pass 2^52.
  for (const int nseq : {1, 2, 100, 1 << 12, 1 << 20}) {
    int64_t sum[2] = {0, 0};
    for (int s0 = 0; s0 < nseq; s0 += 64) {
      int64_t more[2] = {0, 0};
      for (int s = s0; s < std::min(nseq, s0 + 64); ++s) {
        const PagedSeq q = paged_seq(s % 2 ? 8192 : 0, s % 2 ? 0 : 8192, 1 << 30, 8192, 1 << 30);
        more[0] += paged_cost(few, paged_tiles(few, q));
        more[1] += paged_cost(many, paged_tiles(many, q));
      }
      for (int i = 0; i < 2; ++i) sum[i] = paged_add(sum[i], more[i]);
    }
    const int64_t total = paged_line(sum[1], sum[0]);
    const PagedShares shares = paged_shares(many, total, 512, 512);
    if (total < 0 || total > kPagedMost || (total == 0) != ((nseq + 1) / 2 >= 16) || 512 * shares.length < total) fail("a line's length", nseq);
    if (paged_line(sum[0], sum[1]) != 0) fail("work on an empty line", nseq);
  }
}

int main() {
  quotients();
  long_lines();
  roles();
  std::mt19937 g(5);
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(g); };
  int64_t cut = 0, empty = 0;
  for (int n = 0; n < 4000; ++n) {
    const int group = std::vector<int>{1, 2, 3, 4, 5, 7, 8, 16, 40}[pick(0, 8)];
    const bool few = pick(0, 1);
    const int unit = few ? 128 : 64, least = unit * pick(1, 3), share = unit * pick(1, 4);
    const int kv = pick(1, 4), nseq = pick(0, 9), shares = pick(1, 64), room = 5000;
    const PagedRule r = paged_rule(group, few ? 32 : 128, unit, least, pick(1, 600), share, few ? kPagedFew : kPagedMany, 32);
    std::vector<int> cu{0}, len;
    for (int s = 0; s < nseq; ++s) {
      const int longest = pick(0, 3) == 0 ? 6000 : 300;
      len.push_back(pick(-2, longest));
      cu.push_back(cu.back() + (pick(0, 3) == 0 ? pick(0, 300) : pick(0, 2)));
    }
    const int64_t tokens = std::max(0, cu.back() + pick(-1, 2));
    if (nseq && pick(0, 9) == 0) cu[pick(0, nseq)] = pick(-3, 900);  // offsets that decrease: nothing outside is touched
    struct Tile {
      std::vector<int> seen;
      int pieces = 0, wanted = -1, starter = -1, whole = 0;
    };
    std::map<std::vector<int>, Tile> tiles;
    int64_t per_head = 0;
    std::vector<int64_t> cost;
    for (int s = 0; s < nseq; ++s) {
      const PagedSeq q = paged_seq(cu[s], cu[s + 1], len[s], tokens, room);
      if (q.q0 < 0 || q.lq < 0 || q.q0 + q.lq > tokens || q.lk < 0 || q.lk > room) fail("rows outside", n);
      const PagedTiles t = paged_tiles(r, q);
      cost.push_back(paged_cost(r, t));
      per_head += cost.back();
      for (int h = 0; h < kv; ++h)
        for (int i = 0; i < t.tiles; ++i) {
          tiles[{h, s, i}].seen.assign(paged_keys(r, q, t, i), 0);
          if (paged_before(r, t, i + 1) <= paged_before(r, t, i)) fail("a tile without an interval", n);
        }
    }
    const int64_t total = per_head * kv;
    const PagedShares line = paged_shares(r, total, shares, shares);
    const int64_t length = line.length;
    if (line.dies * line.each * length < total) fail("shares too short", n);
    std::vector<char> slots(2 * shares, 0);
    for (int i = 0; i < line.dies * line.each; ++i) {
      int64_t from = i * length;
      const int64_t to = std::min(total, (i + 1) * length);
      int64_t at = 0;
      for (int s = 0; s < nseq; ++s)
        for (int h = 0; h < kv; ++h, at += cost[s]) {
          if (from >= to || from < at || from >= at + cost[s]) continue;
          const PagedSeq q = paged_seq(cu[s], cu[s + 1], len[s], tokens, room);
          const PagedTiles t = paged_tiles(r, q);
          for (int k = paged_tile_at(r, t, from - at); k < t.tiles && from < to; ++k) {
            const int64_t a = at + paged_before(r, t, k), b = at + paged_before(r, t, k + 1);
            if (from < a || from >= b) fail("a position outside its tile", n);
            PagedPiece p;
            if (paged_piece(r, q, t, k, a, from, std::min(to, b), length, i, &p)) {
              Tile& x = tiles[{h, s, k}];
              if (p.begin % r.unit || p.begin < 0 || p.end > p.n || (p.n && p.begin >= p.end)) fail("a piece's keys", n);
              if (p.end < p.n && p.end % r.unit) fail("a piece's end", n);
              for (int j = p.begin; j < p.end; ++j) ++x.seen[j];
              if (p.slot < 0) {
                ++x.whole;
                if (p.begin != 0 || p.end != p.n) fail("a part without a slot", n);
              } else {
                ++cut;
                if (p.end - p.begin < std::min(r.least, r.share)) fail("a short piece", n);
                if (p.slot < 0 || p.slot >= 2 * shares || slots[p.slot]++) fail("a slot twice", n);
                if (p.begin == 0) {
                  x.starter = i;
                  x.wanted = p.pieces;
                  if (p.slot != 2 * i + 1) fail("a first slot", n);
                } else if (x.starter < 0 || p.slot != 2 * (x.starter + x.pieces)) {
                  fail("slots out of order", n);
                }
                ++x.pieces;
              }
            }
            from = std::min(to, b);
          }
        }
      if (from < to) fail("a share's end", n);
    }
    for (auto& kv_ : tiles) {
      Tile& x = kv_.second;
      for (int c : x.seen)
        if (c != 1) fail("a key not taken once", n);
      if (x.seen.empty()) ++empty;
      if (x.whole + (x.pieces > 0) != 1) fail("a tile not done once", n);
      if (x.pieces && (x.pieces != x.wanted || x.pieces < 2)) fail("pieces miscounted", n);
    }
  }
  std::printf("ok: 4000 batches, %lld pieces, %lld tiles without keys\n", static_cast<long long>(cut), static_cast<long long>(empty));
  return 0;
}
