// Work of attention over a paged cache, divided on the GPU: what host and device code share (no HIP needed).
//
// Offsets, lengths and page tables are in device memory, so that a captured call follows them as they grow. A launch has a fixed number
// of workgroups. Each works out the costs of all sequences by itself and takes an even share of their sum: positions
// share * length .. on one line on which every tile of packed rows (query, head of the group) of every key head has an interval,
// key head by key head, sequence by sequence. Sequence s has `rows` packed rows in tiles of `tile`; the interval of tile t is as long as
// group * (fixed + keys before the sequence's queries) + its last row's number, which is its loop's length in keys and a fixed part, times the
// group: an arithmetic series, so where a tile begins has a closed form. A boundary between two shares inside a tile cuts its loop at a
// multiple of `unit` keys, not nearer than `least` to either end; both shares work out the same cut. The pieces of a cut
// tile leave partial results, joined by a second kernel.
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#define T2V_HD __host__ __device__ __forceinline__
#else
#define T2V_HD inline
#endif

namespace t2v {

// Which sequences a kernel takes: all, or those with at most / more than few rows.
enum PagedClass { kPagedAll = 0, kPagedFew = 1, kPagedMany = 2 };

struct PagedRule {
  int group;   // query heads of a key head
  int tile;    // packed rows of a tile
  int unit;    // keys, a multiple of 16
  int least;   // keys of the shortest piece, a multiple of unit
  int fixed;   // a tile's cost besides its loop, in keys
  int share;   // keys of the shortest share, at least unit
  int cls, few;
};

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
  int64_t first;  // cost of a tile before its rows: group * (fixed + keys before the queries)
};
// Tiles of a sequence for a kernel (none if another kernel takes it).
T2V_HD PagedTiles paged_tiles(const PagedRule& r, const PagedSeq& s) {
  PagedTiles t;
  t.rows = s.lq * r.group;
  const bool mine = r.cls == kPagedAll || (r.cls == kPagedFew) == (t.rows <= r.few);
  t.tiles = mine ? (t.rows + r.tile - 1) / r.tile : 0;
  const int before = s.lk > s.lq ? s.lk - s.lq : 0;
  t.first = static_cast<int64_t>(r.group) * (r.fixed + before);
  return t;
}
// Cost of tiles 0 .. t - 1.
T2V_HD int64_t paged_before(const PagedRule& r, const PagedTiles& s, int t) {
  const int64_t full = t * s.first + static_cast<int64_t>(r.tile) * t * (t + 1) / 2;
  return t < s.tiles ? full : full - (static_cast<int64_t>(t) * r.tile - s.rows);
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
  const int64_t n = static_cast<int64_t>(s.lk) - s.lq + last / r.group + 1;
  return n < 0 ? 0 : n > s.lk ? s.lk : static_cast<int>(n);
}
// Key at which position x of a tile's interval of length cost cuts its loop over n keys.
T2V_HD int paged_cut(const PagedRule& r, int64_t x, int64_t cost, int n) {
  if (x >= cost) return n;
  const int64_t y = x - static_cast<int64_t>(r.group) * r.fixed;
  const int64_t k = y < 0 ? 0 : y / (static_cast<int64_t>(r.group) * r.unit) * r.unit;
  return k < r.least ? 0 : k > n - r.least ? n : static_cast<int>(k);
}
// The first position that cuts at n.
T2V_HD int64_t paged_whole(const PagedRule& r, int64_t cost, int n) {
  int64_t m = n < r.least ? 0 : (n - r.least) / r.unit + 1;
  if (m * r.unit < r.least) m = r.least / r.unit;
  const int64_t x = static_cast<int64_t>(r.group) * (r.fixed + m * r.unit);
  return x < cost ? x : cost;
}

// Even shares of `total`: their length, so that share i takes positions i * length .. (i + 1) * length - 1.
T2V_HD int64_t paged_share(const PagedRule& r, int64_t total, int shares) {
  const int64_t even = (total + shares - 1) / shares, least = static_cast<int64_t>(r.group) * r.share;
  return even > least ? even : least;
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
    p->pieces = static_cast<int>((at + paged_whole(r, cost, p->n) + length - 1) / length) - share;
  }
  return true;
}

}  // namespace t2v
