// Host-side planning of causal attention with grouped heads (no HIP): work items, the cut of
// long loops into pieces, and the order in which items are handed to the GPU's dies.
//
// Sequence s has Lq queries and Lk keys; its query i sees keys 0 .. i + Lk - Lq (the last query
// sees every key). `group` query heads share one key head, so the queries of a key head form
// Lq * group packed rows, row r = query r / group, head r % group of the group: neighbouring rows
// see the same keys, one tile of rows serves all heads of a group, and a single token's
// heads fill a tile together.
#pragma once

#include <cstdint>
#include <string>
#include <vector>

namespace t2v {

// A tile of one (sequence, key head). Forward and dQ: `tile0` is a packed row and the loop runs
// over keys begin .. end - 1. dK/dV: `tile0` is a key and the loop runs over stages begin .. end - 1
// of `stage` queries each, causal_stages() of them for each head of the group, head by head.
// slot >= 0: the loop is one of `pieces` pieces, whose partial results go to that slot (an entry
// of a reduce list: slot is the first of `pieces` consecutive ones).
struct CausalItem {
  int32_t qrow0, lq;   // the sequence's queries in the packed tensors
  int32_t krow0, lk;   // its keys
  int32_t tile0, head; // first row or key of the tile; key head
  int32_t begin, end;
  int32_t slot, pieces;
  int32_t pad0, pad1;
};
static_assert(sizeof(CausalItem) == 48, "three 16-byte scalar loads");

enum CausalKernel { kCausalFwd = 4, kCausalDkdv = 5, kCausalDq = 6 };  // kinds of work list

// What one kind of work list is built for.
struct CausalShape {
  const int32_t* cu_q;
  const int32_t* cu_k;
  int nseq, kv_heads, group;
};

// First query that sees key `key` (not clamped to Lq).
inline int32_t causal_first_query(int32_t key, int32_t lq, int32_t lk) {
  const int32_t i = key - (lk - lq);
  return i > 0 ? i : 0;
}
// Keys that query i sees.
inline int32_t causal_keys(int32_t i, int32_t lq, int32_t lk) {
  const int64_t n = static_cast<int64_t>(i) + 1 + lk - lq;
  return n < 0 ? 0 : static_cast<int32_t>(n < lk ? n : lk);
}
// Stages of `stage` queries in one head's loop over the queries that see any key of the tile at `key`.
inline int32_t causal_stages(int32_t key, int32_t lq, int32_t lk, int stage) {
  const int32_t i = causal_first_query(key, lq, lk);
  return i >= lq ? 0 : (lq - i + stage - 1) / stage;
}

struct CausalList {
  std::vector<CausalItem> items, reduce;
  int64_t slots = 0;  // partial slots that the items write
};

// The work list of tiles of `block` packed rows (forward, dQ) or keys (dK/dV, whose loop is counted
// in stages of `stage` queries). chunk > 0 cuts loops longer than `chunk` keys or stages into equal
// pieces (multiples of 64 keys). order as in build_worklist. `fixed` is an item's cost besides its
// loop, in keys or stages; `workers` workgroups run at a time.
CausalList build_causal_list(CausalKernel kind, const CausalShape& a, int block, int stage, int order, int chunk,
                             double fixed, int workers);

// What running a work list costs, in microseconds: an item fixed + unit * loop length, with `workers`
// workgroups at a time, or alone instead of unit with a CU to itself; joining cut loops `join`, `piece` for each piece
// of the most cut tile, and byte * the bytes that the pieces write, slot_row of them for each row (or key).
struct CausalCost {
  double unit, alone, fixed;
  int cus, workers;
  double join, piece, byte;
  int64_t slot_row;
};

// Loop length at which to cut (0: nowhere) for the least estimated time, which is returned in *time. Pieces have at
// least `least` keys or stages; at most max_slots slots are used.
int causal_chunk(CausalKernel kind, const CausalShape& a, int block, int stage, const CausalCost& cost, int least,
                 int64_t max_slots, double* time);

// Checks items against the offsets that they were built from, as check_work_items does: an empty
// string, or what is wrong with the first bad one.
std::string check_causal_items(CausalKernel kind, const CausalItem* items, int n, const CausalShape& a, int block,
                               int stage, int64_t max_slots, bool reduce);

}  // namespace t2v
