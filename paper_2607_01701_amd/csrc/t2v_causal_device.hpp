// Device helpers shared by the causal attention kernels.
//
// A mask is one number per query: `lim`, the last key that it sees, relative to the first key of the
// step at hand (negative: none). Scores of masked pairs never reach a maximum, a sum or a
// product: P and dS are selected to zero. A masked row of V, K, dO or Q that holds an infinity or a NaN
// would still reach the sums (zero times it is NaN), so in masked steps such elements are taken out of
// the operands, and their products added index by index where the pair is visible.
#pragma once

#include "t2v_causal_kernels.h"
#include "t2v_kernel_common.hpp"

namespace t2v {
namespace kern {

// A packed row of a (sequence, key head): its query and its head's place in the group.
struct PackedRow {
  int query, head;
};
T2V_DEV PackedRow packed_row(int row, int group) {
  const int i = static_cast<int>(static_cast<unsigned>(row) / static_cast<unsigned>(group));
  return {i, row - i * group};
}

// This lane's row of a tile: where it is in [T, H, D] tensors, and the last key that it sees. A wave's lanes l and
// l + 32 hold the same row; rows behind the last have ok = false and repeat its query.
struct LaneRow {
  bool ok;
  int lim, head;
  int64_t token;
};
T2V_DEV LaneRow lane_row(const CausalItem& it, int group, int wave, int lane) {
  const int nrows = it.lq * group, row = it.tile0 + wave * 32 + (lane & 31);
  const PackedRow pr = packed_row(min(row, nrows - 1), group);
  return {row < nrows, pr.query + it.lk - it.lq, it.head * group + pr.head, static_cast<int64_t>(it.qrow0) + pr.query};
}

// What rounding to bf16 took from 8 values: hi + lo holds 16 bits of them.
T2V_DEV bf16x8 rest_bf16x8(const f32x16& x, int base, const bf16x8& hi) {
  bf16x8 r;
#pragma unroll
  for (int t = 0; t < 8; ++t) r[t] = static_cast<bf16>(x[base + t] - static_cast<float>(hi[t]));
  return r;
}

// The operand with only contraction index kk (0..15) kept: element t of a lane holds index
// 8 (t / 4) + 4 G + t % 4, as read_rows_opnd and the packed scores have it.
T2V_DEV bf16x8 only_index(const bf16x8& x, int kk, int G) {
  const int t = 4 * (kk >> 3) + (kk & 3);  // uniform, as kk is
  const unsigned half = G == ((kk >> 2) & 1) ? (t & 1 ? 0xFFFF0000u : 0xFFFFu) : 0u;
  u32x4 w = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] &= e == t >> 1 ? half : 0u;
  return __builtin_bit_cast(bf16x8, w);
}

// acc[db] += the products of p with the infinities and NaN of the rows operand, over the 32 contraction
// indices of a step, one at a time; sees(kk, r): whether this lane's result r takes index kk. read(half, db)
// gives the operand of indices half .. half + 15 again.
template <int DB, typename Read, typename Sees>
T2V_DEV void add_nonfinite(f32x16 (&acc)[DB], const bf16x8 (&p)[2], int G, Read&& read, Sees&& sees) {
#pragma unroll 1
  for (int kk = 0; kk < 32; ++kk) {
    u32x4 w = __builtin_bit_cast(u32x4, p[0]);
    const u32x4 w1 = __builtin_bit_cast(u32x4, p[1]);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = kk < 16 ? w[e] : w1[e];
    const bf16x8 pk = only_index(__builtin_bit_cast(bf16x8, w), kk & 15, G);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      fence();  // one product at a time: the sums leave few registers
      const bf16x8 x = only_index(split_finite<false>(read(kk & 16, db)), kk & 15, G);
      const f32x16 t = mfma(x, pk, zero16());
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[db][r] += sees(kk, r) ? t[r] : 0.0f;
    }
  }
}

}  // namespace kern
}  // namespace t2v
