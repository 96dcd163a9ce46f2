// Work of attention over a paged cache, divided on the GPU: what host and device code share (no HIP needed).
//
// Offsets, lengths and page tables are in device memory, so that a captured call follows them as they grow. A launch has a fixed number
// of workgroups. Each works out the costs of all sequences by itself and takes an even share of their sum: an interval
// of one line on which every tile of packed rows (query, head of the group) of every key head has an interval,
// sequence by sequence, key head by key head. A position is 1 / 256 of a key. Sequence s has `rows` packed rows in tiles of `tile`; the
// interval of tile t is as long as a fixed part, the keys before the sequence's queries, and t + 1 tiles' queries, which is (but for
// rounding) its loop's length: an arithmetic series, so where a tile begins has a closed form. A boundary between two
// shares inside a tile cuts its loop at a multiple of `unit` keys, not nearer than `least` to either end; both shares work out the
// same cut. The pieces of a cut tile leave partial results, joined by a second kernel.
//
// Sequences with at most `few` packed rows (single tokens), whose loops wait for memory, and those with more, which keep the matrix cores busy,
// are two lines with tiles and costs of their own. The workgroups are dealt to them by their work, so that a CU has some of both.
//
// Nothing here divides 64-bit numbers, which would take the GPU longer than a short loop: a quotient is estimated in 32 bits and put right.
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#define T2V_HD __host__ __device__ __forceinline__
#else
#define T2V_HD inline
#endif

namespace t2v {

// The longest line. (Positions are exact in a double, and sums of 64 sequences' in 64 bits.) A call whose sequences can reach it is refused;
// where offsets decrease, they may all the same, as each has the queries that others have too: then no work is done.
constexpr int64_t kPagedMost = int64_t(1) << 52;
T2V_HD int64_t paged_add(int64_t sum, int64_t more) {
  const int64_t x = sum + more;
  return x > kPagedMost ? kPagedMost + 1 : x;
}
T2V_HD int64_t paged_line(int64_t sum, int64_t other) { return sum > kPagedMost || other > kPagedMost ? 0 : sum; }

// Which sequences a line takes: those with at most `few` rows, or those with more.
enum PagedClass { kPagedFew = 0, kPagedMany = 1 };

struct PagedRule {
  int group;   // query heads of a key head
  int tile;    // packed rows of a tile
  int span;    // a tile's queries, in positions, rounded up
  int unit;    // keys, a power of two from 16 on
  int least;   // keys of the shortest piece, a multiple of unit
  int fixed;   // a tile's cost besides its loop, in keys, at least 1
  int share;   // keys of the shortest share, at least unit
  int cls, few;
};
inline PagedRule paged_rule(int group, int tile, int unit, int least, int fixed, int share, int cls, int few) {
  return {group, tile, (tile * 256 + group - 1) / group, unit, least, fixed, share, cls, few};
}

// floor(a / b) of a >= 0 and b > 0, where it is below 2^16.
T2V_HD int paged_ratio(int64_t a, int64_t b) {
#if defined(__HIP_DEVICE_COMPILE__)
  int q = static_cast<int>(static_cast<float>(a) * __builtin_amdgcn_rcpf(static_cast<float>(b)));
#else
  int q = static_cast<int>(static_cast<float>(a) / static_cast<float>(b));
#endif
  while (q * b > a) --q;
  while ((q + 1) * b <= a) ++q;
  return q;
}

// A sequence as the kernels see it: rows of the packed queries and keys, whatever the device arrays hold.
struct PagedSeq {
  int64_t q0;
  int lq, lk;
  bool bad;  // longer than its row of the table: no key is read, and the results are NaN
};
T2V_HD PagedSeq paged_seq(int cu0, int cu1, int length, int64_t tokens, int room) {
  PagedSeq s;
  s.q0 = cu0 < 0 ? 0 : cu0 > tokens ? tokens : cu0;
  const int64_t q1 = cu1 < s.q0 ? s.q0 : cu1 > tokens ? tokens : cu1;
  s.lq = static_cast<int>(q1 - s.q0);
  s.bad = length > room;
  s.lk = length < 0 || s.bad ? 0 : length;
  return s;
}

struct PagedTiles {
  int rows, tiles;
  int64_t first;  // length of a tile's interval before its queries
  int64_t over;   // by how much the tiles' queries are more than the sequence's
};
// Tiles of a sequence on a line (none if it is on the other).
T2V_HD PagedTiles paged_tiles(const PagedRule& r, const PagedSeq& s) {
  PagedTiles t;
  t.rows = s.lq * r.group;
  const bool mine = (r.cls == kPagedFew) == (t.rows <= r.few);
  t.tiles = mine ? static_cast<int>(static_cast<unsigned>(t.rows + r.tile - 1) / static_cast<unsigned>(r.tile)) : 0;
  const int before = s.lk > s.lq ? s.lk - s.lq : 0;
  t.first = (static_cast<int64_t>(r.fixed) + before) * 256;
  t.over = static_cast<int64_t>(t.tiles) * r.span - static_cast<int64_t>(s.lq) * 256;
  return t;
}
// Length of the intervals of tiles 0 .. t - 1.
T2V_HD int64_t paged_before(const PagedRule& r, const PagedTiles& s, int t) {
  const int64_t full = t * s.first + (static_cast<int64_t>(t) * (t + 1) / 2) * r.span;
  return t < s.tiles ? full : full - s.over;
}
T2V_HD int64_t paged_cost(const PagedRule& r, const PagedTiles& s) { return s.tiles == 0 ? 0 : paged_before(r, s, s.tiles); }
// Tile that position u of the sequence's interval lies in.
T2V_HD int paged_tile_at(const PagedRule& r, const PagedTiles& s, int64_t u) {
  int lo = 0, hi = s.tiles - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (paged_before(r, s, mid) <= u)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}
// Keys that the tile's last row sees.
T2V_HD int paged_keys(const PagedRule& r, const PagedSeq& s, const PagedTiles& t, int tile) {
  const int64_t end = static_cast<int64_t>(tile + 1) * r.tile;
  const int last = static_cast<int>(end < t.rows ? end : t.rows) - 1;
  const int64_t n = static_cast<int64_t>(s.lk) - s.lq + static_cast<int>(static_cast<unsigned>(last) / static_cast<unsigned>(r.group)) + 1;
  return n < 0 ? 0 : n > s.lk ? s.lk : static_cast<int>(n);
}
// Key at which position x of a tile's interval of length cost cuts its loop over n keys.
T2V_HD int paged_cut(const PagedRule& r, int64_t x, int64_t cost, int n) {
  if (x >= cost) return n;
  const int64_t y = (x >> 8) - r.fixed;
  const int64_t k = y < 0 ? 0 : y & ~static_cast<int64_t>(r.unit - 1);
  return k < r.least ? 0 : k > n - r.least ? n : static_cast<int>(k);
}
// The first position that cuts at n.
T2V_HD int64_t paged_whole(const PagedRule& r, int64_t cost, int n) {
  int64_t k = n < r.least ? 0 : ((n - r.least) & ~(r.unit - 1)) + r.unit;
  if (k < r.least) k = r.least;
  const int64_t x = (k + r.fixed) * 256;
  return x < cost ? x : cost;
}

// How many of `groups` workgroups take the line of many rows, `weight` being the time of a position of few rows against one of many: as their
// share of the work, but each line that has any gets some. Dies (workgroup b runs on die b % 8) get as many each.
T2V_HD bool paged_by_die(int groups) { return groups % 8 == 0 && groups >= 16; }
T2V_HD int paged_many(int groups, int64_t few, int64_t many, float weight) {
  if (many == 0 || few == 0) return few == 0 && many != 0 ? groups : 0;
  const int each = paged_by_die(groups) ? 8 : 1, slots = groups / each;
  const float x = static_cast<float>(many), part = x / (x + weight * static_cast<float>(few));
  int n = static_cast<int>(part * slots + 0.5f);
  n = n < 1 ? 1 : n > slots - 1 ? slots - 1 : n;
  return n * each;
}
// Workgroup b's line and its place among those of its die (x) that take it, n_many of `groups` being the line of many rows': a die's first ones, which
// begin one to a CU, so that few CUs have two. (Dealt alternately, two of them met on a CU where their distance divided a die's CUs: 60
// tokens beside a chunk of 200, 40 heads over 8: 290 us against 229; the die's last ones: 249.)
struct PagedRole {
  bool many;
  int x, i;
};
T2V_HD PagedRole paged_role(int b, int groups, int n_many) {
  const bool dies = paged_by_die(groups);
  const int x = dies ? b % 8 : 0, i = dies ? b / 8 : b, m = dies ? n_many / 8 : n_many;
  return {i < m, x, i < m ? i : i - m};
}

// Shares of a line, `each` for each of the dies, one after the other; share i takes positions i * length .. (i + 1) * length - 1.
struct PagedShares {
  int dies, each;
  int64_t length;
};
// Even shares of `total` for the n workgroups of `groups` that take the line, a little more than even (total / n is off by less than 1), but none shorter
// than the rule's: where that leaves workgroups without one, every die has as many (a token over 2,000 keys, 24 heads over 8, in a
// table for 64,000: 14 us; on the first two dies 17).
T2V_HD PagedShares paged_shares(const PagedRule& r, int64_t total, int n, int groups) {
  PagedShares s;
  s.dies = paged_by_die(groups) ? 8 : 1;
  s.each = n / s.dies;
  const int64_t least = static_cast<int64_t>(r.share) * 256, keys = (total >> (s.dies == 8 ? 11 : 8)) + 1;  // keys: of a die
  if (keys < static_cast<int64_t>(s.each) * r.share) s.each = static_cast<int>((static_cast<unsigned>(keys) + r.share - 1) / static_cast<unsigned>(r.share));
  const int shares = s.dies * s.each;
#if defined(__HIP_DEVICE_COMPILE__)
  double inverse = __builtin_amdgcn_rcpf(static_cast<float>(shares));
#else
  double inverse = 1.0f / static_cast<float>(shares);
#endif
  inverse *= 2.0 - shares * inverse;  // 23 bits, 46, and what a double holds
  inverse *= 2.0 - shares * inverse;
  s.length = static_cast<int64_t>(static_cast<double>(total) * inverse) + 2;
  if (s.length < least) s.length = least;
  return s;
}

// A loop, or a piece of one: keys begin .. end - 1 of a tile of n keys. slot >= 0: a piece, whose partial results go there.
struct PagedPiece {
  int tile, begin, end, n;
  int slot;
  int pieces;  // of the tile, set where begin = 0
};
// What share `i` does of the tile whose interval begins at position `at` of the line, from position `from` on; false: nothing.
// The slots of a cut tile that share i begins are 2 i + 1, 2 (i + 1), 2 (i + 2), ..
T2V_HD bool paged_piece(const PagedRule& r, const PagedSeq& s, const PagedTiles& t, int tile, int64_t at, int64_t from, int64_t to,
                        int64_t length, int share, PagedPiece* p) {
  const int64_t cost = paged_before(r, t, tile + 1) - paged_before(r, t, tile);
  p->tile = tile;
  p->n = paged_keys(r, s, t, tile);
  p->begin = paged_cut(r, from - at, cost, p->n);
  p->end = paged_cut(r, to - at, cost, p->n);
  p->slot = -1;
  p->pieces = 1;
  if (p->n == 0) return from == at;
  if (p->begin >= p->end) return false;
  if (p->begin > 0) {
    p->slot = 2 * share;
  } else if (p->end < p->n) {
    p->slot = 2 * share + 1;
    p->pieces = paged_ratio(at + paged_whole(r, cost, p->n) - 1, length) - share + 1;
  }
  return true;
}

// Workgroups that join a cut tile of `tile` rows, in a call of `rows` packed rows in all sequences: several, unless no tile can have more rows than one holds.
// (What the call's sequences are is known on the GPU alone, and most of a cache's may have no queries: their number says nothing.)
inline int paged_join_blocks(int64_t rows, int few, int several) { return rows <= few ? 1 : several; }

}  // namespace t2v
