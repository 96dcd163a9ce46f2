// dK/dV kernel of causal attention with grouped heads: a workgroup owns 32 keys per wave of one
// (sequence, key head) and loops over the queries that see any of them, head by head of the group, so
// that the group's sum stays in registers (128 keys and 64-query stages at head_dim 128, 256
// and 128 at 64). The loop starts at the first query that sees the tile; a wave skips 32-query steps
// that see none of its keys and masks those that see some. A cut loop leaves fp32 sums in its slot, which the
// join adds in piece order.
//
// What bounds it. At 64, power and the waits between stages: an item takes 2.85 us for a stage alone on its CU and 4.1 with
// all CUs at work; matrix cores busy 50%, LDS 62% of the cycles (seven sequences of 77 to 6,001 tokens, 30 heads over 10:
// 497 us, 920 TFLOP/s; long ones 1,000 to 1,100. 64 keys a wave, as in t2v_causal_dkdv_wide.hip, took 540). At 128 it serves short loops, where its 128-key tiles fill the GPU (4 x 640 tokens,
// 24 heads over 8: 58 us against 65 of t2v_causal_dkdv_wide.hip's 256 keys); long ones are the other's (16 clips of 1,280 to
// 20,280 tokens, 12 heads: 9.4 against 7.9 ms).
#include "t2v_causal_device.hpp"

namespace t2v {

using namespace kern;

namespace {

constexpr int kStages = 4;  // LDS stages: up to 3 tiles of Q / dO in flight during one tile's work
template <int D>
constexpr int threads() { return D == 64 ? 512 : 256; }
template <int D>
constexpr int stage_queries() { return D == 64 ? 128 : 64; }
template <int D>
constexpr int tile_keys() { return threads<D>() / 64 * 32; }

// Lane i copies row i0 + off + i of g, at most L - 1, to lds[i]; i0 < L.
T2V_DEV void rows_dma(float* lds, const float* g, int i0, int off, int L, int lane) {
  const uint32_t r = static_cast<uint32_t>(min(off + lane, L - 1 - i0));
  const uint32_t to = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
#if T2V_CHECKED
  if (!check_row(i0 + static_cast<int>(r), L)) {
    dma_lds4_s(g, 0u, to);
    return;
  }
#endif
  dma_lds4_s(g + i0, r * 4, to);
}

// One 32-query step for this wave's 32 keys. MASK: key m (0..31 of the wave) is seen by query n of the step when
// m <= first + n and n < nq.
template <int D, bool MASK>
T2V_DEV void dkdv_step(uint32_t qbase, uint32_t gbase, uint32_t qr0, uint32_t qr1, uint32_t gr0, uint32_t gr1,
                       const float* sL2, const float* sDl, int q0, int first, int nq, float c,
                       const bf16x8 (&kop)[D / 16], const bf16x8 (&vop)[D / 16], f32x16 (&dka)[D / 32],
                       f32x16 (&dva)[D / 32], int lane) {
  __builtin_amdgcn_iglp_opt(0);
  constexpr int KK = D / 16;
  constexpr int DB = D / 32;
  const int G = lane >> 5;
  // S and dP - Delta (32 queries x 32 keys): lane = key, register r = query 8 (r / 4) + 4 G + r % 4. dP's
  // sums start at -Delta (stored negated).
  f32x16 s = zero16(), dp;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(sDl + q0 + i * 8 + G * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) dp[i * 4 + e] = x[e];
  }
  bf16x8 aq[KK], ag[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) aq[kk] = read_opnd<D>(qbase, q0, kk);
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) ag[kk] = read_opnd<D>(gbase, q0, kk);
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) s = mfma(aq[kk], kop[kk], s);
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) dp = mfma(ag[kk], vop[kk], dp);
  f32x4 lv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) lv[i] = *reinterpret_cast<const f32x4*>(sL2 + q0 + i * 8 + G * 4);
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const float p = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lv[r >> 2][r & 3]));
    const int n = (r >> 2) * 8 + G * 4 + (r & 3);
    const bool sees = !MASK || ((lane & 31) <= first + n && n < nq);
    s[r] = sees ? p : 0.0f;
    dp[r] = sees ? p * dp[r] : 0.0f;
  }
  // P and dS in bf16 for their products, the sums in 32 bits; in masked steps with the rest, as in the forward kernel.
  bf16x8 pb[2] = {to_bf16x8(s, 0), to_bf16x8(s, 8)};
  bf16x8 sb[2] = {to_bf16x8(dp, 0), to_bf16x8(dp, 8)};
  if constexpr (MASK) {  // the operands of the sums only now: read ahead, they and the tests below would spill
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      pin(pb[hf]);
      pin(sb[hf]);
    }
    fence();
  }
  // dV^T += dO^T P, then dK^T += Q^T dS: the dS arithmetic finishes under the first.
  bf16x8 bg[2][DB], bq[2][DB];
  auto read_g = [&](int half, int db) { return read_rows_opnd<D>(gr0, gr1, q0 + half, db); };
  auto read_q = [&](int half, int db) { return read_rows_opnd<D>(qr0, qr1, q0 + half, db); };
  auto sees = [&](int n, int) { return (lane & 31) <= first + n && n < nq; };
#pragma unroll
  for (int hf = 0; hf < 2; ++hf)
#pragma unroll
    for (int db = 0; db < DB; ++db) bg[hf][db] = read_g(hf * 16, db);
  const bool odd_g = MASK && (take_nonfinite(bg[0]) | take_nonfinite(bg[1]));
#pragma unroll
  for (int hf = 0; hf < 2; ++hf)
#pragma unroll
    for (int db = 0; db < DB; ++db) dva[db] = mfma(bg[hf][db], pb[hf], dva[db]);
  if constexpr (MASK) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const bf16x8 rest = rest_bf16x8(s, 8 * hf, pb[hf]);
#pragma unroll
      for (int db = 0; db < DB; ++db) dva[db] = mfma(bg[hf][db], rest, dva[db]);
    }
    fence();
  }
#pragma unroll
  for (int hf = 0; hf < 2; ++hf)
#pragma unroll
    for (int db = 0; db < DB; ++db) bq[hf][db] = read_q(hf * 16, db);
  const bool odd_q = MASK && (take_nonfinite(bq[0]) | take_nonfinite(bq[1]));
#pragma unroll
  for (int hf = 0; hf < 2; ++hf)
#pragma unroll
    for (int db = 0; db < DB; ++db) dka[db] = mfma(bq[hf][db], sb[hf], dka[db]);
  if constexpr (MASK) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const bf16x8 rest = rest_bf16x8(dp, 8 * hf, sb[hf]);
#pragma unroll
      for (int db = 0; db < DB; ++db) dka[db] = mfma(bq[hf][db], rest, dka[db]);
    }
    if (odd_g) add_nonfinite(dva, pb, G, read_g, sees);
    if (odd_q) add_nonfinite(dka, sb, G, read_q, sees);
  }
}

template <int D>
__global__ __launch_bounds__(threads<D>(), 1) void causal_dkdv_kernel(
    const bf16* __restrict__ q, const bf16* __restrict__ k, const bf16* __restrict__ v, int64_t qs, int64_t ks,
    int64_t vs, const bf16* __restrict__ dout, const float* __restrict__ lse2, const float* __restrict__ ndelta,
    const CausalItem* __restrict__ items, int H, int Hk, int g, int64_t T, float c, float scale, bf16* __restrict__ dk,
    bf16* __restrict__ dv, float* __restrict__ partial, unsigned long long* __restrict__ trace) {
  constexpr int KK = D / 16;
  constexpr int DB = D / 32;
  constexpr int BM = stage_queries<D>();
  constexpr int NS = kStages;
  constexpr int NW = threads<D>() / 64;
  // DMA instructions per wave and stage: the Q and dO tiles, plus one 32-float piece of
  // lse * log2(e) or -Delta.
  constexpr int kOps = 2 * (BM * D / 512) / NW + 1;
  static_assert(2 * BM == 32 * NW, "each wave stages one 32-float piece of lse2 / -Delta");
  __shared__ __attribute__((aligned(1024))) bf16 sQ[NS][BM * D];
  __shared__ __attribute__((aligned(1024))) bf16 sG[NS][BM * D];  // dO
  __shared__ __attribute__((aligned(16))) float sL[NS][BM];       // lse * log2(e)
  __shared__ __attribute__((aligned(16))) float sD[NS][BM];       // -Delta
  const unsigned long long trace_t0 = trace != nullptr ? trace_clock() : 0ull;
  const CausalItem it = items[blockIdx.x];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = lane >> 5;
  const int l32 = lane & 31;
  const int key_wave0 = it.tile0 + wave * 32;
  const bool wave_active = key_wave0 < it.lk;
  const int off = it.lk - it.lq;  // query i sees keys up to i + off

  f32x16 dka[DB], dva[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    dka[db] = zero16();
    dva[db] = zero16();
  }
  const int ntiles = it.end - it.begin;
  if (ntiles > 0) {
    const int i_first = max(it.tile0 - off, 0);         // first query that sees the tile
    const int per_head = (it.lq - i_first + BM - 1) / BM;  // stages of one head
    const int64_t rs = static_cast<int64_t>(H) * D;
    const bf16* q0 = q + it.qrow0 * qs + static_cast<int64_t>(it.head) * g * D;
    const bf16* g0 = dout + it.qrow0 * rs + static_cast<int64_t>(it.head) * g * D;
    const float* vec0 = (wave < NW / 2 ? lse2 : ndelta) + static_cast<int64_t>(it.head) * g * T + it.qrow0;
    const int vec_off = (wave % (NW / 2)) * 32;
    // Every wave issues exactly kOps DMA instructions per stage, so counted waits work.
    const TileDma<D, BM, threads<D>()> qdma(tid, qs), gdma(tid, rs);
    int shead = it.begin / per_head, si = it.begin - shead * per_head;  // of the next stage to copy
    int slot_in = 0;
    auto stage = [&]() {
      const int i0 = i_first + si * BM;
      qdma.copy(sQ[slot_in], q0 + shead * D, qs, i0, it.lq);
      gdma.copy(sG[slot_in], g0 + shead * D, rs, i0, it.lq);
      float* dst = (wave < NW / 2 ? sL[slot_in] : sD[slot_in]) + vec_off;
      if (lane < 32) rows_dma(dst, vec0 + shead * T, i0, vec_off, it.lq, lane);
      slot_in = (slot_in + 1) % NS;
      if (++si == per_head) {
        si = 0;
        ++shead;
      }
    };
    // Before reading stage t + 1: wait for it, leaving the stages issued after it in flight.
    auto wait_next = [&](int t) {
      const int after = min(NS - 2, ntiles - 2 - t);
      if (after >= 2)
        wait_vmcnt<2 * kOps>();
      else if (after == 1)
        wait_vmcnt<kOps>();
      else
        wait_vmcnt0();
    };
    static_assert(NS == 4, "wait_next counts two stages in flight");

    int ci = si;  // stage of its head that is worked on
    stage();
    bf16x8 kop[KK], vop[KK];  // this wave's 32 keys as B operands
    {
      const int kj = key_wave0 + l32;
      const bool ok = kj < it.lk;
      const bf16* kp = k + (static_cast<int64_t>(it.krow0) + kj) * ks + static_cast<int64_t>(it.head) * D;
      const bf16* vp = v + (static_cast<int64_t>(it.krow0) + kj) * vs + static_cast<int64_t>(it.head) * D;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        kop[kk] = load8(kp + kk * 16 + G * 8, ok);
        vop[kk] = load8(vp + kk * 16 + G * 8, ok);
      }
    }
    wait_vmcnt0();
#pragma unroll
    for (int t = 1; t < NS - 1; ++t)
      if (t < ntiles) stage();
    __syncthreads();

    const uint32_t oo = opnd_lane_off<D>(lane);
    const uint32_t ro0 = rows_lane_off<D>(lane, 0), ro1 = rows_lane_off<D>(lane, 1);
    // Stages f0 .. f1 - 1 of a head are seen whole: every query is there and sees all keys of the wave. The
    // others (a head's first ones and its last) take the masked steps; every wave passes ntiles barriers.
    const int f0 = (max(key_wave0 + 31 - off - i_first, 0) + BM - 1) / BM;
    const int f1 = wave_active ? (it.lq - i_first) / BM : 0;
    int tt = 0;
    while (tt < ntiles) {
      for (; tt < ntiles && (ci < f0 || ci >= f1); ++tt) {
        const int b = tt % NS, i0 = i_first + ci * BM;
        if (tt + NS - 1 < ntiles) stage();
        if (wave_active) {
          const uint32_t tq = lds_addr(sQ[b]), tg = lds_addr(sG[b]);
          const int first = i0 + off - key_wave0;  // the wave's last key that query i0 sees
#pragma unroll 1
          for (int n = 0; n < BM && i0 + n < it.lq; n += 32)
            if (D == 64 && first + n >= 31 && i0 + n + 32 <= it.lq)
              dkdv_step<D, false>(tq + oo, tg + oo, tq + ro0, tq + ro1, tg + ro0, tg + ro1, sL[b], sD[b], n, 0, 0, c, kop,
                                  vop, dka, dva, lane);
            else if (first + n + 31 >= 0)
              dkdv_step<D, true>(tq + oo, tg + oo, tq + ro0, tq + ro1, tg + ro0, tg + ro1, sL[b], sD[b], n, first + n,
                                 it.lq - i0 - n, c, kop, vop, dka, dva, lane);
        }
        if (++ci == per_head) ci = 0;
        wait_next(tt);
        __syncthreads();
      }
      for (; tt < ntiles && ci >= f0 && ci < f1; ++tt) {
        const int b = tt % NS;
        if (tt + NS - 1 < ntiles) stage();
        const uint32_t tq = lds_addr(sQ[b]), tg = lds_addr(sG[b]);
#pragma unroll
        for (int n = 0; n < BM; n += 32)
          dkdv_step<D, false>(tq + oo, tg + oo, tq + ro0, tq + ro1, tg + ro0, tg + ro1, sL[b], sD[b], n, 0, 0, c, kop,
                              vop, dka, dva, lane);
        if (++ci == per_head) ci = 0;
        wait_next(tt);
        __syncthreads();
      }
    }
  }

  if (wave_active) {
    // Sums: lane = key, register r = column 8 (r / 4) + 4 G + r % 4 of each 32.
    const int kr = wave * 32 + l32;  // key of the tile
    const bool ok = it.tile0 + kr < it.lk;
    if (it.slot >= 0) {
      float* pk = partial + static_cast<int64_t>(it.slot) * (2 * tile_keys<D>() * D) + kr * D;
      float* pv = pk + tile_keys<D>() * D;
      if (ok) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            f32x4 x, y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[e] = dka[db][i * 4 + e];
              y[e] = dva[db][i * 4 + e];
            }
            *reinterpret_cast<f32x4*>(pk + db * 32 + i * 8 + G * 4) = x;
            *reinterpret_cast<f32x4*>(pv + db * 32 + i * 8 + G * 4) = y;
          }
      }
    } else {
      const int64_t at = ((static_cast<int64_t>(it.krow0) + it.tile0 + kr) * Hk + it.head) * D;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        store_rows(dk + at + db * 32, dka[db], scale, G, ok);
        store_rows(dv + at + db * 32, dva[db], 1.0f, G, ok);
      }
    }
  }
  if (trace != nullptr) trace_end(trace, trace_t0, 2, blockIdx.x);
}

// Adds the pieces of the cut tiles (of `keys` keys) in order. A workgroup takes 32 keys; a thread four columns. Bound by the
// pieces' bytes (95 MB in 18 us).
template <int D>
__global__ __launch_bounds__(kThreads) void causal_dkdv_join_kernel(const float* __restrict__ partial,
                                                                     const CausalItem* __restrict__ tiles, int keys,
                                                                     int Hk, float scale, bf16* __restrict__ dk,
                                                                     bf16* __restrict__ dv) {
  constexpr int C4 = D / 4;
  const int parts = keys / 32;
  const CausalItem it = tiles[blockIdx.x / parts];
  const int k0 = (blockIdx.x % parts) * 32;
  const int nkeys = min(32, it.lk - it.tile0 - k0);
  const int64_t rs = static_cast<int64_t>(Hk) * D, slot = 2 * keys * D;
  for (int e = threadIdx.x; e < 2 * 32 * C4; e += kThreads) {
    const int which = e / (32 * C4), r = e / C4 % 32, c4 = e % C4;  // which: 0 dK, 1 dV
    if (r >= nkeys) continue;
    const float* p = partial + it.slot * slot + which * keys * D + (k0 + r) * D + c4 * 4;
    f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int i = 0; i < it.pieces; ++i) a += *reinterpret_cast<const f32x4*>(p + i * slot);
    const float m = which == 0 ? scale : 1.0f;
    bf16x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = static_cast<bf16>(a[i] * m);
    const int64_t kj = static_cast<int64_t>(it.krow0) + it.tile0 + k0 + r;
    *reinterpret_cast<bf16x4*>((which == 0 ? dk : dv) + kj * rs + static_cast<int64_t>(it.head) * D + c4 * 4) = w;
  }
}

template <int D>
void launch_as(const CausalArgs& a, const CausalItem* items, int n, hipStream_t s) {
  hipLaunchKernelGGL((causal_dkdv_kernel<D>), dim3(n), dim3(threads<D>()), 0, s, static_cast<const bf16*>(a.q),
                     static_cast<const bf16*>(a.k), static_cast<const bf16*>(a.v), a.q_stride, a.k_stride, a.v_stride,
                     static_cast<const bf16*>(a.dout), a.delta + a.tq * a.heads, a.delta, items, a.heads, a.kv_heads,
                     a.heads / a.kv_heads, a.tq, a.scale * kLog2e, a.scale, static_cast<bf16*>(a.dk),
                     static_cast<bf16*>(a.dv), a.partial, a.trace);
}

}  // namespace

int causal_dkdv_keys(int head_dim, bool wide) {
  return head_dim == 64 ? tile_keys<64>() : wide ? causal_dkdv_wide_keys() : tile_keys<128>();
}
int causal_dkdv_stage(int head_dim, int keys) {
  if (head_dim == 64) return stage_queries<64>();
  return keys == causal_dkdv_wide_keys() ? causal_dkdv_wide_stage() : stage_queries<128>();
}
int64_t causal_dkdv_slot_bytes(int keys, int head_dim) { return 8LL * keys * head_dim; }

hipError_t launch_causal_dkdv(const CausalArgs& a, int keys, const CausalItem* items, int n, hipStream_t s) {
  if (a.head_dim == 128 && keys == causal_dkdv_wide_keys()) return launch_causal_dkdv_wide(a, items, n, s);
  a.head_dim == 128 ? launch_as<128>(a, items, n, s) : launch_as<64>(a, items, n, s);
  return hipGetLastError();
}

hipError_t launch_causal_dkdv_join(const CausalArgs& a, int keys, const CausalItem* tiles, int n, hipStream_t s) {
  const dim3 grid(n * (keys / 32));
  auto *dk = static_cast<bf16*>(a.dk), *dv = static_cast<bf16*>(a.dv);
  if (a.head_dim == 128)
    hipLaunchKernelGGL((causal_dkdv_join_kernel<128>), grid, dim3(kThreads), 0, s, a.partial, tiles, keys, a.kv_heads,
                       a.scale, dk, dv);
  else
    hipLaunchKernelGGL((causal_dkdv_join_kernel<64>), grid, dim3(kThreads), 0, s, a.partial, tiles, keys, a.kv_heads,
                       a.scale, dk, dv);
  return hipGetLastError();
}

#if T2V_CHECKED
hipError_t causal_dkdv_check_take(unsigned int* rec, unsigned int canary) { return kern::check_take_here(rec, canary); }
#endif
}  // namespace t2v
