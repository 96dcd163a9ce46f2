// dK/dV kernel of causal attention for long query loops at head_dim 128: a workgroup of four waves owns 256
// keys, 64 per wave, and takes 32-query steps (t2v_dkdv_wide_step.hpp) over the queries that see any of
// them, for all heads of the group, whose sums stay in accumulator registers (lane = key). First come the masked
// steps of all heads: those at the start of a head's queries that do not see the whole tile (eight at most: in
// each, some wave has pairs to mask, and the others would wait for it), and a last, partial one. Then the plain
// steps of all heads. Two loops in a row, because the sums fill the accumulator registers: where code
// paths over them met again, the compiler would have to copy them.
//
// Bound by the matrix cores and power: busy 65% of the cycles with 2.8 vector instructions for each matrix instruction (16 clips
// of 1,280 to 20,280 tokens, 12 heads: 7.56 to 7.9 ms, 1,225 to 1,280 TFLOP/s). What the masked steps waste counts where
// loops are short: 8 x 4,096 tokens, 24 heads over 8: 1.41 to 1.45 ms, 1,140 to 1,170.
#include "t2v_causal_device.hpp"
#include "t2v_dkdv_wide_step.hpp"

namespace t2v {

using namespace kern;
using namespace kern::wide;

namespace {

__global__ __launch_bounds__(kWideThreads, 1) void causal_dkdv_wide_kernel(
    const bf16* __restrict__ q, const bf16* __restrict__ k, const bf16* __restrict__ v, int64_t qs, int64_t ks,
    int64_t vs, const bf16* __restrict__ dout, const float* __restrict__ lse2, const float* __restrict__ ndelta,
    const CausalItem* __restrict__ items, int H, int Hk, int g, int64_t T, float c, float scale, bf16* __restrict__ dk,
    bf16* __restrict__ dv, float* __restrict__ partial, unsigned long long* __restrict__ trace) {
  constexpr int NS = kStages, BM = kBM;
  constexpr uint32_t kTile = BM * D * 2;  // bytes of one stage of Q or dO
  __shared__ __attribute__((aligned(1024))) bf16 sK[kWideKeys * D];
  __shared__ __attribute__((aligned(1024))) bf16 sQ[NS][BM * D];
  __shared__ __attribute__((aligned(1024))) bf16 sG[NS][BM * D];  // dO
  __shared__ __attribute__((aligned(16))) float sL[NS][64];       // lse * log2(e); BM of each 64 are used
  __shared__ __attribute__((aligned(16))) float sD[NS][64];       // -Delta

  const unsigned long long trace_t0 = trace != nullptr ? trace_clock() : 0ull;
  const CausalItem it = items[blockIdx.x];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int key_wave0 = it.tile0 + wave * 64;
  const int off = it.lk - it.lq;  // query i sees keys up to i + off
  const int i_first = max(it.tile0 - off, 0);  // first query that sees the tile
  const int64_t rs = static_cast<int64_t>(H) * D;
  const bf16* const q0 = q + it.qrow0 * qs + static_cast<int64_t>(it.head) * g * D;
  const bf16* const g0 = dout + it.qrow0 * rs + static_cast<int64_t>(it.head) * g * D;

  f32x16 dka[2][DB], dva[2][DB];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      dka[b][db] = zero16();
      dva[b][db] = zero16();
    }
  bool odd = false;  // some masked step's Q or dO held an infinity or a NaN
  const int ntiles = it.end - it.begin;
  if (ntiles > 0) {
    const int per_head = (it.lq - i_first + BM - 1) / BM;  // steps of one head
    // Two waves copy lse2, two -Delta (the same rows twice, so every wave issues kOps copies a stage).
    const float* const vec0 = (wave < 2 ? lse2 : ndelta) + static_cast<int64_t>(it.head) * g * T + it.qrow0;
    const TileDma<D, BM, kWideThreads> qdma(tid, qs), gdma(tid, rs);
    // Of each head, steps 0 .. np - 1 do not see the whole tile; nm steps are masked, step j of them being step j of
    // the head, or its last; nf steps, from np on, are plain.
    const int np = min((max(min(it.tile0 + kWideKeys, it.lk) - 1 - off - i_first, 0) + BM - 1) / BM, per_head);
    const int nm = np + (per_head > np && (it.lq - i_first) % BM != 0), nf = per_head - nm;
    struct At {  // step j of its kind of head `head`
      int head, j, n;
    };
    auto place = [&](int t) {
      const bool masked = t < g * nm;
      const int u = masked ? t : t - g * nm, n = max(masked ? nm : nf, 1);
      return At{u / n, u % n, masked ? nm : nf};
    };
    auto first_query = [&](const At& x, bool masked) {
      return i_first + BM * (masked ? (x.j < np ? x.j : per_head - 1) : np + x.j);
    };
    int ti = it.begin, slot_in = 0;  // of the next stage to copy
    At in = place(ti);
    auto stage = [&] {
      const int i0 = first_query(in, ti < g * nm);
      qdma.copy(sQ[slot_in], q0 + in.head * D, qs, i0, it.lq);
      gdma.copy(sG[slot_in], g0 + in.head * D, rs, i0, it.lq);
      rows_dma(wave < 2 ? sL[slot_in] : sD[slot_in], vec0 + in.head * T, i0, it.lq, lane);
      slot_in = slot_in + 1 == NS ? 0 : slot_in + 1;
      ++ti;
      if (++in.j == in.n) {
        in.j = 0;
        if (ti == g * nm)
          in = At{0, 0, nf};
        else
          ++in.head;
      }
    };
    stage();
    const TileDma<D, kWideKeys, kWideThreads> kd(tid, ks);
    kd.copy(sK, k + it.krow0 * ks + static_cast<int64_t>(it.head) * D, ks, it.tile0, it.lk);
    bf16x8 vop[2][KK];  // V of this wave's 64 keys, as B operands
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int kj = key_wave0 + b * 32 + (lane & 31);
      const bool ok = kj < it.lk;
      const bf16* vp = v + (static_cast<int64_t>(it.krow0) + kj) * vs + static_cast<int64_t>(it.head) * D + (lane >> 5) * 8;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) vop[b][kk] = load8(vp + kk * 16, ok);
    }
    // Stage 0, the K tile and the operand loads complete here.
    wait_vmcnt0();
#pragma unroll
    for (int t = 1; t < NS - 1; ++t)
      if (t < ntiles) stage();
    __syncthreads();

    const uint32_t oo = opnd_lane_off<D>(lane);
    const uint32_t ro0 = rows_lane_off<D>(lane, 0), ro1 = rows_lane_off<D>(lane, 1);
    const uint32_t kbase = lds_addr(sK) + oo + wave * 64 * 2 * D;
    const uint32_t lq = lds_addr(sQ), lg = lds_addr(sG);
    auto address = [&](int b, int nb) {
      const uint32_t tq = lq + b * kTile, tg = lg + b * kTile;
      return StepAddr{tq + oo, tg + oo, tq + ro0, tq + ro1, tg + ro0, tg + ro1, lq + nb * kTile + oo, kbase, sL[b], sD[b]};
    };
    bf16x8 aq[KK], kb[kAhead];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) aq[kk] = read_opnd<D>(lq + oo, 0, kk);
#pragma unroll
    for (int kk = 0; kk < kAhead; ++kk) kb[kk] = read_opnd<D>(kbase, 0, kk);
    int tt = 0, b = 0;
    // In the middle of step tt: stage tt + 1 has arrived (those issued after it may be in flight), and every wave
    // is past step tt - 1, whose buffer takes stage tt + NS - 1.
    auto arrive = [&] {
      const int after = min(NS - 3, ntiles - 2 - tt);
      if (after >= 2)
        wait_vmcnt<2 * kOps>();
      else if (after == 1)
        wait_vmcnt<kOps>();
      else
        wait_vmcnt0();
    };
    static_assert(NS == 5, "arrive counts two stages in flight");
    auto publish = [] {  // a barrier without the waits that __syncthreads adds for reads in flight
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    const int masked_end = min(g * nm, it.end) - it.begin;
    At at = place(it.begin);
    for (; tt < masked_end; ++tt) {
      const int i0 = first_query(at, true), nb = b + 1 == NS ? 0 : b + 1;
      // An infinity or a NaN in a row of Q leaves none of its scores' sum finite, one in a row of dO no Delta. (A scale
      // of 0 hides it from the scores.)
      const float stat = sL[b][lane & 31] - sD[b][lane & 31];
      const bool odd_step = scale == 0.0f || __any(!(fabsf(stat) < kInf));
      odd |= odd_step;
      dkdv_wide_step<kCausal, true>(address(b, nb), it.lq - i0, i0 + off - key_wave0, odd_step, c, aq, kb, vop, dka, dva,
                                    lane, [&] {
                                      arrive();
                                      publish();
                                      if (tt + NS - 1 < ntiles) stage();
                                    });
      b = nb;
      if (++at.j == nm) {
        at.j = 0;
        ++at.head;
      }
    }
#if !T2V_CHECKED
    // Plain steps whose copy exists: plain stages are whole tiles, so a copy has no branches; the next head's
    // queries follow after a jump.
    {
      const int64_t head_jump = (D - static_cast<int64_t>(nf - 1) * BM * qs) * 2, step = BM * qs * 2;
      const int64_t ghead_jump = (D - static_cast<int64_t>(nf - 1) * BM * rs) * 2, gstep = BM * rs * 2;
      const int64_t lhead_jump = T - static_cast<int64_t>(nf - 1) * BM;
      const int i0 = first_query(in, false);
      const char* qn = reinterpret_cast<const char*>(q0 + in.head * D + i0 * qs);
      const char* gn = reinterpret_cast<const char*>(g0 + in.head * D + i0 * rs);
      const float* vn = vec0 + in.head * T + i0;
      const uint32_t lv = wave < 2 ? lds_addr(sL) : lds_addr(sD), voff = static_cast<uint32_t>(min(lane, BM - 1)) * 4;
      constexpr int kRowsPerCopy = 2048 / D;  // rows that the four waves copy with one instruction each
      const int64_t qj = kRowsPerCopy * qs * 2, gj = kRowsPerCopy * rs * 2;
      for (; tt < ntiles - (NS - 1); ++tt) {
        const int nb = b + 1 == NS ? 0 : b + 1;
        const uint32_t free_slot = b == 0 ? NS - 1 : b - 1;  // the buffer of step tt - 1
        dkdv_wide_step<kFull, true>(address(b, nb), BM, 0, false, c, aq, kb, vop, dka, dva, lane, [&] {
          wait_vmcnt<(NS - 3) * kOps>();
          publish();
          const uint32_t to_q = lq + free_slot * kTile + wave * 1024, to_g = lg + free_slot * kTile + wave * 1024;
#pragma unroll
          for (int j = 0; j < BM / kRowsPerCopy; ++j) dma_lds16_s(qn + j * qj, qdma.off0, to_q + j * 4096);
#pragma unroll
          for (int j = 0; j < BM / kRowsPerCopy; ++j) dma_lds16_s(gn + j * gj, gdma.off0, to_g + j * 4096);
          dma_lds4_s(vn, voff, lv + free_slot * 256);
          const bool last = ++in.j == nf;
          in.j = last ? 0 : in.j;
          qn += last ? head_jump : step;
          gn += last ? ghead_jump : gstep;
          vn += last ? lhead_jump : BM;
        });
        b = nb;
      }
    }
#endif
    for (; tt < ntiles; ++tt) {  // the last steps (in checked builds, all plain ones)
      const int nb = b + 1 == NS ? 0 : b + 1;
      dkdv_wide_step<kFull, true>(address(b, nb), BM, 0, false, c, aq, kb, vop, dka, dva, lane, [&] {
        arrive();
        publish();
#if T2V_CHECKED
        if (tt + NS - 1 < ntiles) stage();
#endif
      });
      b = nb;
    }
  }

  // Sums: lane = key, register r = column 8 (r / 4) + 4 G + r % 4 of each 32.
  acc_settle();
  const int el = lane_again(), eG = el >> 5;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const f32x16(&acc)[2][DB] = which == 0 ? dka : dva;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int kr = wave * 64 + b * 32 + (el & 31);  // key of the tile
      const int key = it.tile0 + kr;
      const bool ok = key < it.lk;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        f32x16 x;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = acc_read(acc[b][db][r]);
        if (which == 1 && odd) {
          // The infinities and NaN of dO that the masked steps (those of the tile's first queries, and a partial
          // last one) left out, for the keys that see their query.
          const int plain = i_first + (max(min(it.tile0 + kWideKeys, it.lk) - 1 - off - i_first, 0) + BM - 1) / BM * BM;
          const int tail = it.lq - (it.lq - i_first) % BM;
#pragma unroll 1
          for (int i = i_first; i < it.lq; i = i + 1 == plain ? max(i + 1, tail) : i + 1)
#pragma unroll 1
            for (int h = 0; h < g; ++h) {
              const bf16* row = g0 + i * rs + h * D + db * 32 + 4 * eG;
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const float y = static_cast<float>(row[8 * (r >> 2) + (r & 3)]);
                if (key <= i + off && !(fabsf(y) < kInf)) x[r] += y;
              }
            }
        }
        if (it.slot >= 0) {
          float* p = partial + static_cast<int64_t>(it.slot) * (2 * kWideKeys * D) + which * kWideKeys * D + kr * D + db * 32;
          if (ok) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<f32x4*>(p + i * 8 + eG * 4) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
          }
        } else {
          const int64_t at = ((static_cast<int64_t>(it.krow0) + key) * Hk + it.head) * D + db * 32;
          store_rows((which == 0 ? dk : dv) + at, x, which == 0 ? scale : 1.0f, eG, ok);
        }
      }
    }
  }
  if (trace != nullptr) trace_end(trace, trace_t0, 2, blockIdx.x, wave == 0 && el == 0);
}

}  // namespace

int causal_dkdv_wide_keys() { return kWideKeys; }
int causal_dkdv_wide_stage() { return kBM; }

hipError_t launch_causal_dkdv_wide(const CausalArgs& a, const CausalItem* items, int n, hipStream_t s) {
  if (a.head_dim != D) return hipErrorInvalidValue;
  hipLaunchKernelGGL(causal_dkdv_wide_kernel, dim3(n), dim3(kWideThreads), 0, s, static_cast<const bf16*>(a.q),
                     static_cast<const bf16*>(a.k), static_cast<const bf16*>(a.v), a.q_stride, a.k_stride, a.v_stride,
                     static_cast<const bf16*>(a.dout), a.delta + a.tq * a.heads, a.delta, items, a.heads, a.kv_heads,
                     a.heads / a.kv_heads, a.tq, a.scale * kLog2e, a.scale, static_cast<bf16*>(a.dk),
                     static_cast<bf16*>(a.dv), a.partial, a.trace);
  return hipGetLastError();
}

#if T2V_CHECKED
hipError_t causal_dkdv_wide_check_take(unsigned int* rec, unsigned int canary) {
  return kern::check_take_here(rec, canary);
}
#endif
}  // namespace t2v
