// The 32-query step of the dK/dV kernels whose four waves own 64 keys each (head_dim 128): one
// hand-scheduled stream of MFMAs, LDS reads and arithmetic (see t2v_bwd_dkdv_wide.hip), for bidirectional
// and for causal attention.
#pragma once

#include "t2v_kernel_common.hpp"

namespace t2v {
namespace kern {
namespace wide {

constexpr int kWideKeys = 256;  // keys per workgroup
constexpr int kBM = 32;         // queries per LDS stage and per step

constexpr int D = 128;          // head dim
constexpr int KK = D / 16;      // k-steps of the head-dim contraction
constexpr int DB = D / 32;      // 32-wide head-dim blocks
constexpr int kStages = 5;      // LDS stages
constexpr int kAhead = 4;       // operands read ahead of their MFMA
constexpr int kWideThreads = 256;
constexpr int kOps = 2 * (kBM * D / 512) / 4 + 1;  // DMA instructions per wave and stage
// Arithmetic per slot of a step: one P element from slot kPFirst on (when S of block 0 is
// ready), then two dS elements.
constexpr int kPRate = 1, kPFirst = KK + 1;
constexpr int kSRate = 2, kSFirst = kPFirst + 32 / kPRate;

constexpr int clamp32(int x) { return x < 0 ? 0 : x > 32 ? 32 : x; }

// Copy of 64 consecutive floats into LDS, one per lane: lane i takes row i0 + i, clamped to
// L - 1 (i0 < L).
T2V_DEV void rows_dma(float* lds, const float* g, int i0, int L, int lane) {
  const uint32_t r = static_cast<uint32_t>(min(lane, L - 1 - i0));
  const uint32_t dst = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
#if T2V_CHECKED
  if (!check_row(i0 + static_cast<int>(r), L)) {  // copy the segment's first row instead
    dma_lds4_s(g, 0u, dst);
    return;
  }
#endif
  dma_lds4_s(g + i0, r * 4, dst);
}

// LDS addresses of one step's operands: this lane's base in the Q and dO tiles (16-byte and
// transposing reads), in the next stage's Q tile, and in this wave's K rows.
struct StepAddr {
  uint32_t q, g, qr0, qr1, gr0, gr1, qnext, k;
  const float *lse2, *ndelta;
};

// One 32-query step. Slots: S of key block 0 (KK MFMAs), S of block 1 (KK), dP of both (2 KK),
// dV of both (4 DB), dK of both (4 DB); 64 MFMAs at D = 128. Block 0's scores come first so that
// its softmax runs under block 1's; P of a 16-query half is due at its dV products, dS at its dK
// products. `sync` sits between dP and dV: it waits for the next stage, whose first operands
// the dK slots read, and frees the previous stage's buffer for a new copy.
// aq holds this step's Q operands on entry and the next one's on return; kb likewise the first K
// operands. MASK kRagged: only the first nvalid queries count. kCausal: of those, query n sees keys
// 0 .. first + n of the wave; where `odd` (the step's Q or dO holds an infinity or a NaN) such elements are taken
// out of the products dS^T Q and P^T dO: zero times them would reach keys that their query does not see. (A
// query with such a Q or dO has a dS of its own that is none or NaN, which keeps dK right; dV is the caller's to
// mend.) TRANSPOSED: the sums have lane = key in place of lane = column.
enum Mask { kFull, kRagged, kCausal };
template <Mask MASK, bool TRANSPOSED, typename Sync>
T2V_DEV void dkdv_wide_step(const StepAddr& a, int nvalid, int first, bool odd, float c, bf16x8 (&aq)[KK],
                            bf16x8 (&kb)[kAhead],
                            const bf16x8 (&vop)[2][KK], f32x16 (&dka)[2][DB], f32x16 (&dva)[2][DB], int lane,
                            Sync&& sync) {
  constexpr int AH = kAhead;
  const int G = lane >> 5;
  f32x16 s[2], dp[2], nd;
  s[0] = zero16();
  s[1] = zero16();
  f32x4 lv[4];
  bf16x8 ag[KK], pb[2][2], sb[2][2], bg[2][DB], bq[2][DB];
  auto read_k = [&](int i) { kb[i % AH] = read_opnd<D>(a.k, (i / KK) * 32, i % KK); };
  // Register r's query is 8 (r / 4) + r % 4 + 4 G; it sees the lane's key of block b if that number is at least
  // `from` + 32 b and below `from` + `span`, less 4 G: one unsigned comparison.
  const int from = (lane & 31) - first - 4 * G;
  const unsigned span[2] = {static_cast<unsigned>(max(nvalid - 4 * G - from, 0)),
                            static_cast<unsigned>(max(nvalid - 4 * G - from - 32, 0))};
  auto sees = [&](int b, int r) {
    return static_cast<unsigned>((r >> 2) * 8 + (r & 3) - 32 * b - from) < span[b];
  };
  // Arithmetic unit u of 32: element u % 8 of 16-query half u / 16 of key block (u / 8) % 2, i.e.
  // in the order in which the dV (dK) products need the halves; the eighth converts the half.
  auto p_unit = [&](int u) {
    const int b = (u >> 3) & 1, h = u >> 4, r = 8 * h + (u & 7);
    float p = __builtin_amdgcn_exp2f(fmaf(s[b][r], c, -lv[r >> 2][r & 3]));
    if constexpr (MASK != kFull) {
      const int qi = (r >> 2) * 8 + G * 4 + (r & 3);
      if constexpr (MASK == kRagged)
        p = qi < nvalid ? p : 0.0f;
      else
        p = sees(b, r) ? p : 0.0f;
    }
    pin(p);
    s[b][r] = p;
    if ((u & 7) == 7) {
      pb[b][h] = to_bf16x8(s[b], 8 * h);
      pin(pb[b][h]);
    }
  };
  auto s_unit = [&](int u) {
    const int b = (u >> 3) & 1, h = u >> 4, r = 8 * h + (u & 7);
    float x = s[b][r] * dp[b][r];
    if constexpr (MASK == kCausal) {  // zero whatever dP is where the pair is masked
      x = sees(b, r) ? x : 0.0f;
    }
    pin(x);
    dp[b][r] = x;
    if ((u & 7) == 7) {
      sb[b][h] = to_bf16x8(dp[b], 8 * h);
      pin(sb[b][h]);
    }
  };
  auto arithmetic = [&](int slot) {
#pragma unroll
    for (int u = clamp32((slot - kPFirst) * kPRate); u < clamp32((slot + 1 - kPFirst) * kPRate); ++u)
      p_unit(u);
#pragma unroll
    for (int u = clamp32((slot - kSFirst) * kSRate); u < clamp32((slot + 1 - kSFirst) * kSRate); ++u)
      s_unit(u);
  };
  fence();
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {  // S of block 0; the row statistics arrive
    s[0] = mfma(aq[kk], kb[kk % AH], s[0]);
    fence();
    read_k(kk + AH);
    const f32x4 x = *reinterpret_cast<const f32x4*>((kk < 4 ? a.lse2 : a.ndelta) + (kk & 3) * 8 + G * 4);
    if (kk < 4) {
      lv[kk & 3] = x;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) nd[(kk & 3) * 4 + e] = x[e];
    }
    fence();
  }
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {  // S of block 1
    s[1] = mfma(aq[kk], kb[(KK + kk) % AH], s[1]);
    fence();
    if (kk + KK + AH < 2 * KK) read_k(kk + KK + AH);
    if (kk >= KK - AH) ag[kk - (KK - AH)] = read_opnd<D>(a.g, 0, kk - (KK - AH));
    arithmetic(KK + kk);
    fence();
  }
#pragma unroll
  for (int i = 0; i < 2 * KK; ++i) {  // dP - Delta of both blocks (the accumulators start at -Delta)
    const int kk = i >> 1, b = i & 1;
    dp[b] = mfma(ag[kk], vop[b][kk], kk == 0 ? nd : dp[b]);
    fence();
    if (b == 0) {
      if (kk + AH < KK) ag[kk + AH] = read_opnd<D>(a.g, 0, kk + AH);
      if (kk >= KK - DB) bg[0][kk - (KK - DB)] = read_rows_opnd<D>(a.gr0, a.gr1, 0, kk - (KK - DB));
    }
    arithmetic(2 * KK + i);
    fence();
  }
  sync();
  fence();
#pragma unroll
  for (int i = 0; i < 4 * DB; ++i) {  // dV += P^T dO
    const int h = i / (2 * DB), b = (i / DB) & 1, db = i % DB;
    if constexpr (MASK == kCausal) {
      if (i % (2 * DB) == 0 && odd) {
#pragma unroll
        for (int n = 0; n < DB; ++n) bg[h][n] = split_finite<true>(bg[h][n]);
      }
      fence();
    }
    if constexpr (TRANSPOSED)
      mfma_acc(dva[b][db], bg[h][db], pb[b][h]);
    else
      mfma_acc(dva[b][db], pb[b][h], bg[h][db]);
    fence();
    if (i < DB) bg[1][i] = read_rows_opnd<D>(a.gr0, a.gr1, 16, i);
    if (i >= 2 * DB && i < 3 * DB) bq[0][i - 2 * DB] = read_rows_opnd<D>(a.qr0, a.qr1, 0, i - 2 * DB);
    arithmetic(4 * KK + i);
    fence();
  }
#pragma unroll
  for (int i = 0; i < 4 * DB; ++i) {  // dK += dS^T Q; the next step's first operands arrive
    const int h = i / (2 * DB), b = (i / DB) & 1, db = i % DB;
    if constexpr (MASK == kCausal) {
      if (i % (2 * DB) == 0 && odd) {
#pragma unroll
        for (int n = 0; n < DB; ++n) bq[h][n] = split_finite<true>(bq[h][n]);
      }
      fence();
    }
    if constexpr (TRANSPOSED)
      mfma_acc(dka[b][db], bq[h][db], sb[b][h]);
    else
      mfma_acc(dka[b][db], sb[b][h], bq[h][db]);
    fence();
    if (i < DB) bq[1][i] = read_rows_opnd<D>(a.qr0, a.qr1, 16, i);
    if (i >= 4 * DB - KK) aq[i - (4 * DB - KK)] = read_opnd<D>(a.qnext, 0, i - (4 * DB - KK));
    if (i >= 4 * DB - AH) read_k(i - (4 * DB - AH));
    arithmetic(4 * KK + 4 * DB + i);
    fence();
  }
}

}  // namespace wide
}  // namespace kern
}  // namespace t2v
