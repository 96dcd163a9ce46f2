// Backward dK/dV kernel for long query loops: a workgroup of four waves owns 256 keys of one
// (clip, head), 64 per wave, and loops over the clip's queries in 32-query steps.
//
// What bounds it: the matrix cores, through power. The 32-keys-per-wave kernel
// (t2v_bwd_dkdv.hip) spends 56 LDS reads on 32 MFMAs and leaves the softmax arithmetic of its
// only wave per SIMD exposed (MFMAs busy 55% of cycles). Here every Q and dO operand feeds two
// key blocks, so at D = 128 a step of 64 MFMAs takes 72 LDS reads (1.1 per MFMA instead of
// 1.75) and half the LDS copies per MFMA, and the step is one hand-scheduled stream in which the
// softmax arithmetic runs under the MFMAs (64% busy, at a clock that the card lowers from 1.96
// to 1.82 GHz as it reaches its power limit). Measured on the heterogeneous mix (24 x 128):
// 34.9 -> 30.6 ms, 1,110 -> 1,267 TFLOP/s; results are bitwise those of the other kernel.
//
// Registers (D = 128): the dK and dV sums of 64 keys fill all 256 AGPRs; V operands take 64
// VGPRs; K operands, which would take 64 more, are read from an LDS tile instead (16 reads of
// the 72). LDS: 64 KB of K and five 16 KB stages of Q and dO. head_dim 64 keeps the other kernel:
// there a step's arithmetic is as long as its MFMAs, and two waves per SIMD, which can issue
// both at once, do better than one (1,131 against 1,085 TFLOP/s at 16,384 tokens).
#include "t2v_dkdv_wide_step.hpp"

namespace t2v {

using namespace kern;
using namespace kern::wide;

namespace {

__global__ __launch_bounds__(kWideThreads, 1) void attn_bwd_dkdv_wide_kernel(
    const bf16* __restrict__ q, const bf16* __restrict__ k, const bf16* __restrict__ v,
    const bf16* __restrict__ dout, const float* __restrict__ lse2, const float* __restrict__ ndelta,
    const Item* __restrict__ items, int H, int64_t T, float c, float scale, bf16* __restrict__ dk,
    bf16* __restrict__ dv, unsigned long long* __restrict__ trace) {
  constexpr int NS = kStages, BM = kBM;
  constexpr uint32_t kTile = BM * D * 2;  // bytes of one stage of Q or dO
  __shared__ __attribute__((aligned(1024))) bf16 sK[kWideKeys * D];
  __shared__ __attribute__((aligned(1024))) bf16 sQ[NS][BM * D];
  __shared__ __attribute__((aligned(1024))) bf16 sG[NS][BM * D];  // dO
  // Row statistics of a stage; each copy fills 64 floats, of which the first BM are used.
  __shared__ __attribute__((aligned(16))) float sL[NS][64];  // lse * log2(e)
  __shared__ __attribute__((aligned(16))) float sD[NS][64];  // -Delta

  const unsigned long long trace_t0 = trace != nullptr ? trace_clock() : 0ull;
  const Item it = items[blockIdx.x];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int Lk = it.len;   // keys of the sequence (this tile's rows)
  const int L = it.llen;   // queries of the sequence (the loop)
  const int64_t rs = static_cast<int64_t>(H) * D;
  const int64_t base = static_cast<int64_t>(it.row0) * rs + static_cast<int64_t>(it.head) * D;
  const int64_t qbase = static_cast<int64_t>(it.lrow0) * rs + static_cast<int64_t>(it.head) * D;
  const int64_t lbase = static_cast<int64_t>(it.head) * T + it.lrow0;
  const bf16* qh = q + qbase;
  const bf16* gh = dout + qbase;
  // Two waves copy lse2, two -Delta (the same rows twice, so every wave issues kOps copies a stage).
  const float* vec_src = (wave < 2 ? lse2 : ndelta) + lbase;
  const int key_wave0 = it.tile0 + wave * 64;

  const TileDma<D, BM, kWideThreads> dma(tid, rs);
  auto stage = [&](int t) {
    const int b = t % NS, i0 = t * BM;
    dma.copy(sQ[b], qh, rs, i0, L);
    dma.copy(sG[b], gh, rs, i0, L);
    rows_dma(wave < 2 ? sL[b] : sD[b], vec_src, i0, L, lane);
  };
  const int ntiles = (L + BM - 1) / BM;
  stage(0);
  const TileDma<D, kWideKeys, kWideThreads> kd(tid, rs);
  kd.copy(sK, k + base, rs, it.tile0, Lk);
  // V of this wave's 64 keys, as B operands (lane = key, elements along head dim).
  bf16x8 vop[2][KK];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int kj = key_wave0 + b * 32 + (lane & 31);
    const bool ok = kj < Lk;
    const int64_t off = base + kj * rs + (lane >> 5) * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) vop[b][kk] = load8(v + off + kk * 16, ok);
  }
  f32x16 dka[2][DB], dva[2][DB];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      dka[b][db] = zero16();
      dva[b][db] = zero16();
    }
  // Stage 0, the K tile and the operand loads complete here (see t2v_bwd_dkdv.hip).
  wait_vmcnt0();
#pragma unroll
  for (int t = 1; t < NS - 1; ++t)
    if (t < ntiles) stage(t);
  __syncthreads();

  const uint32_t oo = opnd_lane_off<D>(lane);
  const uint32_t ro0 = rows_lane_off<D>(lane, 0), ro1 = rows_lane_off<D>(lane, 1);
  const uint32_t kbase = lds_addr(sK) + oo + wave * 64 * 2 * D;
  const uint32_t lq = lds_addr(sQ), lg = lds_addr(sG);
  auto address = [&](int b, int nb) {
    const uint32_t tq = lq + b * kTile, tg = lg + b * kTile;
    return StepAddr{tq + oo, tg + oo, tq + ro0, tq + ro1, tg + ro0, tg + ro1, lq + nb * kTile + oo, kbase, sL[b], sD[b]};
  };
  auto publish = [] {  // a barrier without the waits that __syncthreads adds for reads in flight
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  bf16x8 aq[KK], kb[kAhead];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) aq[kk] = read_opnd<D>(lq + oo, 0, kk);
#pragma unroll
  for (int kk = 0; kk < kAhead; ++kk) kb[kk] = read_opnd<D>(kbase, 0, kk);
  int tt = 0, b = 0;
#if !T2V_CHECKED
  // Steps whose copy (stage tt + NS - 1) is a full tile: no branches inside a step. After the
  // wait, stages tt + 2 .. tt + NS - 2 may still be in flight.
  const char* qn = reinterpret_cast<const char*>(qh + static_cast<int64_t>(NS - 1) * BM * rs);
  const char* gn = reinterpret_cast<const char*>(gh + static_cast<int64_t>(NS - 1) * BM * rs);
  const uint32_t lv = wave < 2 ? lds_addr(sL) : lds_addr(sD);
  constexpr int kRowsPerCopy = 2048 / D;  // rows the four waves copy with one instruction each
  const int64_t jstep = static_cast<int64_t>(kRowsPerCopy) * rs * 2;
  for (const int nsteady = L / BM - (NS - 1); tt < nsteady; ++tt) {
    const int nb = b + 1 == NS ? 0 : b + 1;
    const uint32_t free_slot = b == 0 ? NS - 1 : b - 1;  // the buffer of step tt - 1
    dkdv_wide_step<kFull, false>(address(b, nb), BM, 0, false, c, aq, kb, vop, dka, dva, lane, [&] {
      wait_vmcnt<(NS - 3) * kOps>();
      publish();
      const uint32_t dq_ = lq + free_slot * kTile + wave * 1024, dg_ = lg + free_slot * kTile + wave * 1024;
#pragma unroll
      for (int j = 0; j < BM / kRowsPerCopy; ++j) dma_lds16_s(qn + j * jstep, dma.off0, dq_ + j * 4096);
#pragma unroll
      for (int j = 0; j < BM / kRowsPerCopy; ++j) dma_lds16_s(gn + j * jstep, dma.off0, dg_ + j * 4096);
      const int i0 = (tt + NS - 1) * BM;
      dma_lds4_s(vec_src + i0, static_cast<uint32_t>(min(lane, L - 1 - i0)) * 4, lv + free_slot * 256);
      qn += static_cast<int64_t>(BM) * rs * 2;
      gn += static_cast<int64_t>(BM) * rs * 2;
    });
    b = nb;
  }
#endif
  for (; tt < ntiles; ++tt) {  // the last steps (in checked builds, all): general copies and masks
    const int nb = b + 1 == NS ? 0 : b + 1;
    dkdv_wide_step<kRagged, false>(address(b, nb), L - tt * BM, 0, false, c, aq, kb, vop, dka, dva, lane, [&] {
      wait_vmcnt0();
      publish();
      if (tt + NS - 1 < ntiles) stage(tt + NS - 1);
    });
    b = nb;
  }

  // Accumulators: lane = head-dim column db*32 + l32, register r = key 8 (r/4) + 4 G + r % 4. They
  // leave through this wave's own 16 KB of the K tile, written column by column ([head dim][key],
  // four keys a lane) and read back transposed, so a lane stores 16 bytes of one key row: 32
  // stores a wave in place of 256 two-byte ones.
  acc_settle();
  const int el = lane_again();
  const int eg = el >> 5, ej = el & 15, gr = el >> 4;
  bf16* tile = sK + wave * 64 * D;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const f32x16(&acc)[2][DB] = which == 0 ? dka : dva;
    const float m = which == 0 ? scale : 1.0f;
#pragma unroll
    for (int b2 = 0; b2 < 2; ++b2)
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          bf16x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = static_cast<bf16>(acc_read(acc[b2][db][4 * i + e]) * m);
          *reinterpret_cast<bf16x4*>(tile + swz_off<64>(db * 32 + (el & 31), b2 * 32 + 8 * i + 4 * eg)) = w;
        }
    bf16* const g = (which == 0 ? dk : dv) + base;
#pragma unroll
    for (int k16 = 0; k16 < 4; ++k16) {
      const int kj = key_wave0 + 16 * k16 + ej;
#pragma unroll
      for (int d32 = 0; d32 < DB; ++d32) {
        const int d0 = 32 * d32 + 8 * gr, r = d0 + (ej >> 2), col = 16 * k16 + 4 * (ej & 3);
        const bf16x4 lo = lds_read_tr4(tile + swz_off<64>(r, col));
        const bf16x4 hi = lds_read_tr4(tile + swz_off<64>(r + 4, col));
        bf16x8 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = lo[e];
          w[4 + e] = hi[e];
        }
        if (kj < Lk) *reinterpret_cast<bf16x8*>(g + kj * rs + d0) = w;
      }
    }
  }
  if (trace != nullptr) trace_end(trace, trace_t0, 2, blockIdx.x, wave == 0 && el == 0);
}

}  // namespace

int dkdv_wide_rows() { return kWideKeys; }

hipError_t launch_bwd_dkdv_wide(const AttnArgs& a, const Item* items, int n_items, hipStream_t stream) {
  if (a.head_dim != D) return hipErrorInvalidValue;
  const float c = a.scale * kLog2e;
  const float* lse2 = a.delta + a.total_tokens * a.heads;
  const dim3 grid(n_items), block(kWideThreads);
  hipLaunchKernelGGL(attn_bwd_dkdv_wide_kernel, grid, block, 0, stream, static_cast<const bf16*>(a.q),
                     static_cast<const bf16*>(a.k), static_cast<const bf16*>(a.v), static_cast<const bf16*>(a.dout),
                     lse2, a.delta, items, a.heads, a.total_tokens, c, a.scale, static_cast<bf16*>(a.dk),
                     static_cast<bf16*>(a.dv), a.trace);
  return hipGetLastError();
}
#if T2V_CHECKED
hipError_t dkdv_wide_check_take(unsigned int* rec, unsigned int canary) { return kern::check_take_here(rec, canary); }
#endif
}  // namespace t2v
