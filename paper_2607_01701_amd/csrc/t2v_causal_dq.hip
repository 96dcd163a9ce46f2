// dQ kernel of causal attention with grouped heads: a workgroup owns a tile of packed rows and loops
// over the keys that its last row sees, as the forward kernel does; P comes from the stored lse. Before its loop it works out
// Delta of its rows, of which it holds dO, for itself and for the dK/dV kernel, which runs after it (a kernel of its own for that
// read dO again and took 2% of a training step). A cut
// loop leaves fp32 sums in its slot, which the join adds in piece order.
//
// Three products a pair against the forward's two, and no maximum: matrix cores and power bound it at both head dims, busy 70%
// of the cycles at 128 (16 clips of 1,280 to 20,280 tokens, 12 heads: 5.68 to 6.1 ms, 1,195 to 1,280 TFLOP/s) and 65% at 64
// (seven sequences of 77 to 6,001 tokens, 30 heads over 10: 318 us, 1,080). Wide tiles (256 rows) read each staged key for
// twice the rows (5.86 against 6.06 ms); narrow ones end sooner where a CU has one or two (4 x 640 tokens, 24 heads
// over 8: 31 against 35 us).
#include "t2v_causal_device.hpp"

namespace t2v {

using namespace kern;

namespace {

constexpr int kBN = 64;  // keys per LDS stage
constexpr int kThreadsWide = 512, kThreadsNarrow = 256;

// dP's sums start at -Delta where 16 registers for it leave as many waves (at head_dim 64 three a SIMD: 328 -> 318 us for
// seven sequences of 77 to 6,001 tokens and 30 heads); at 128 it is added after.
template <int D>
constexpr bool kDeltaFirst = D == 64;

// One 32-key step. MASK: this lane's row sees keys 0 .. lim of the step.
template <int D, bool MASK>
T2V_DEV void dq_step(uint32_t kbase, uint32_t vbase, uint32_t kr0, uint32_t kr1, int kb, int lim, float c,
                     const bf16x8 (&qop)[D / 16], const bf16x8 (&gop)[D / 16], float nl2, float ndl,
                     f32x16 (&dqa)[D / 32], int lane) {
  __builtin_amdgcn_iglp_opt(0);
  constexpr int KK = D / 16;
  constexpr int DB = D / 32;
  const int G = lane >> 5;
  // S^T and dP^T (32 keys x 32 rows): lane = row, register r = key 8 (r / 4) + 4 G + r % 4.
  f32x16 s = zero16(), dp = zero16();
  if constexpr (kDeltaFirst<D>) {
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] = ndl;
  }
  {
    bf16x8 ka[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) ka[kk] = read_opnd<D>(kbase, kb, kk);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) s = mfma(ka[kk], qop[kk], s);
  }
  {
    bf16x8 va[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) va[kk] = read_opnd<D>(vbase, kb, kk);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) dp = mfma(va[kk], gop[kk], dp);
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const float ds = __builtin_amdgcn_exp2f(fmaf(s[r], c, nl2)) * (kDeltaFirst<D> ? dp[r] : dp[r] + ndl);
    s[r] = MASK && (r >> 2) * 8 + G * 4 + (r & 3) > lim ? 0.0f : ds;
  }
  // dS in bf16 for its product, the sums in 32 bits; in masked steps with the rest, as P in the forward kernel.
  bf16x8 sb[2] = {to_bf16x8(s, 0), to_bf16x8(s, 8)};
  bf16x8 rest[2];
  if constexpr (MASK) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      rest[hf] = rest_bf16x8(s, 8 * hf, sb[hf]);
      pin(sb[hf]);
      pin(rest[hf]);
    }
    fence();  // the K operands only now: read ahead, they and the test below would spill
  }
  bf16x8 kt[2][DB];
#pragma unroll
  for (int hf = 0; hf < 2; ++hf)
#pragma unroll
    for (int db = 0; db < DB; ++db) kt[hf][db] = read_rows_opnd<D>(kr0, kr1, kb + hf * 16, db);
  const bool odd = MASK && (take_nonfinite(kt[0]) | take_nonfinite(kt[1]));
#pragma unroll
  for (int hf = 0; hf < 2; ++hf)
#pragma unroll
    for (int db = 0; db < DB; ++db) dqa[db] = mfma(kt[hf][db], sb[hf], dqa[db]);
  if constexpr (MASK) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int db = 0; db < DB; ++db) dqa[db] = mfma(kt[hf][db], rest[hf], dqa[db]);
    if (odd)
      add_nonfinite(dqa, sb, G, [&](int half, int db) { return read_rows_opnd<D>(kr0, kr1, kb + half, db); },
                          [&](int kk, int) { return kk <= lim; });
  }
}

template <int D, int NT>
__global__ __launch_bounds__(NT, 512 / NT) void causal_dq_kernel(
    const bf16* __restrict__ q, const bf16* __restrict__ k, const bf16* __restrict__ v, int64_t qs, int64_t ks,
    int64_t vs, const bf16* __restrict__ out, const bf16* __restrict__ dout, const float* __restrict__ lse,
    const CausalItem* __restrict__ items, int H, int g, int64_t T, float c, float scale, bf16* __restrict__ dq,
    float* __restrict__ delta, float* __restrict__ partial, unsigned long long* __restrict__ trace) {
  constexpr int KK = D / 16;
  constexpr int DB = D / 32;
  constexpr int R = NT / 2;
  __shared__ __attribute__((aligned(1024))) bf16 sK[2][kBN * D];
  __shared__ __attribute__((aligned(1024))) bf16 sV[2][kBN * D];
  const unsigned long long trace_t0 = trace != nullptr ? trace_clock() : 0ull;
  const CausalItem it = items[blockIdx.x];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = lane >> 5;
  const bool wave_active = it.tile0 + wave * 32 < it.lq * g;
  const LaneRow me = lane_row(it, g, wave, lane);
  const int lim_lo = __builtin_amdgcn_readlane(me.lim, 0), lim_hi = __builtin_amdgcn_readlane(me.lim, 31);

  f32x16 dqa[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dqa[db] = zero16();

  const int ntiles = (it.end - it.begin + kBN - 1) / kBN;
  const bf16* kh = k + it.krow0 * ks + static_cast<int64_t>(it.head) * D;
  const bf16* vh = v + it.krow0 * vs + static_cast<int64_t>(it.head) * D;
  const TileDma<D, kBN, NT> kdma(tid, ks), vdma(tid, vs);
  if (ntiles > 0) {
    kdma.copy(sK[0], kh, ks, it.begin, it.lk);
    vdma.copy(sV[0], vh, vs, it.begin, it.lk);
  }
  // This lane's half of its row of dO (a B operand of every step) and of out, and Delta from them, which goes to the dK/dV
  // kernel with lse * log2(e) (from the first piece of a cut loop).
  bf16x8 gop[KK];
  float nl2, ndl;
  {
    const int64_t row = (me.token * H + me.head) * D, at = static_cast<int64_t>(me.head) * T + me.token;
    bf16x8 oop[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) gop[kk] = load8(dout + row + kk * 16 + G * 8, me.ok);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) oop[kk] = load8(out + row + kk * 16 + G * 8, me.ok);
    nl2 = me.ok ? -kLog2e * lse[at] : 0.0f;
    float d = 0.0f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) d = fmaf(static_cast<float>(oop[kk][e]), static_cast<float>(gop[kk][e]), d);
    ndl = -half_sum(d);
    if (it.begin == 0 && me.ok && G == 0) {
      delta[at] = ndl;
      delta[static_cast<int64_t>(H) * T + at] = -nl2;
    }
  }
  if (ntiles > 0) {
    bf16x8 qop[KK];
    const bf16* qp = q + me.token * qs + static_cast<int64_t>(me.head) * D;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qop[kk] = load8(qp + kk * 16 + G * 8, me.ok);
    const uint32_t oo = opnd_lane_off<D>(lane);
    const uint32_t ro0 = rows_lane_off<D>(lane, 0), ro1 = rows_lane_off<D>(lane, 1);
    wait_vmcnt0();
    __syncthreads();
    auto prefetch = [&](int tt) {
      if (tt + 1 < ntiles) {
        kdma.copy(sK[(tt & 1) ^ 1], kh, ks, it.begin + (tt + 1) * kBN, it.lk);
        vdma.copy(sV[(tt & 1) ^ 1], vh, vs, it.begin + (tt + 1) * kBN, it.lk);
      }
    };
    // Stages that all rows of this wave see whole, then the others: every wave passes ntiles barriers.
    const int nfull = wave_active ? min(max(lim_lo + 1 - it.begin, 0) / kBN, ntiles) : 0;
    int tt = 0;
    for (; tt < nfull; ++tt) {
      const int b = tt & 1;
      prefetch(tt);
      const uint32_t tk = lds_addr(sK[b]);
      const uint32_t kb0 = tk + oo, vb0 = lds_addr(sV[b]) + oo, k0 = tk + ro0, k1 = tk + ro1;
#pragma unroll
      for (int kb = 0; kb < kBN; kb += 32)
        dq_step<D, false>(kb0, vb0, k0, k1, kb, 0, c, qop, gop, nl2, ndl, dqa, lane);
      wait_vmcnt0();
      __syncthreads();
    }
    // Worked out again, rather than kept in registers through the first loop.
    const int mlane = lane_again(), mlim = lane_row(it, g, wave, mlane).lim;
    for (; tt < ntiles; ++tt) {
      const int b = tt & 1;
      const int key0 = it.begin + tt * kBN;
      prefetch(tt);
      if (wave_active) {
        const uint32_t tk = lds_addr(sK[b]);
        const uint32_t kb0 = tk + oo, vb0 = lds_addr(sV[b]) + oo, k0 = tk + ro0, k1 = tk + ro1;
#pragma unroll 1
        for (int kb = 0; kb < kBN && key0 + kb <= lim_hi; kb += 32)
          dq_step<D, true>(kb0, vb0, k0, k1, kb, mlim - key0 - kb, c, qop, gop, nl2, ndl, dqa, mlane);
      }
      wait_vmcnt0();
      __syncthreads();
    }
  }

  if (wave_active) {
    // Worked out again, rather than kept in registers through the loop.
    const int lane = lane_again(), G = lane >> 5, l32 = lane & 31;
    const LaneRow me = lane_row(it, g, wave, lane);
    if (it.slot >= 0) {
      float* p = partial + (static_cast<int64_t>(it.slot) * R + wave * 32 + l32) * D;
      if (me.ok) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            f32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = dqa[db][i * 4 + e];
            *reinterpret_cast<f32x4*>(p + db * 32 + i * 8 + G * 4) = w;
          }
      }
    } else {
      bf16* p = dq + (me.token * H + me.head) * D;
#pragma unroll
      for (int db = 0; db < DB; ++db) store_rows(p + db * 32, dqa[db], scale, G, me.ok);
    }
  }
  if (trace != nullptr) trace_end(trace, trace_t0, 3, blockIdx.x);
}

// Adds the pieces of the cut tiles in order. D / 8 lanes hold a row, eight columns each.
template <int D>
__global__ __launch_bounds__(kThreads) void causal_dq_join_kernel(const float* __restrict__ partial,
                                                                   const CausalItem* __restrict__ tiles, int R, int H,
                                                                   int g, float scale, bf16* __restrict__ dq) {
  constexpr int LPR = D / 8, RPB = kThreads / LPR;
  const int blocks = R / RPB;
  const CausalItem it = tiles[blockIdx.x / blocks];
  const int r = (blockIdx.x % blocks) * RPB + threadIdx.x / LPR;
  const int col = threadIdx.x % LPR * 8;
  const int row = it.tile0 + r;
  if (row >= it.lq * g) return;
  const PackedRow pr = packed_row(row, g);
  const int64_t slot = static_cast<int64_t>(R) * D;
  const float* p = partial + it.slot * slot + r * D + col;
  f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f}, b = a;
#pragma unroll 4
  for (int i = 0; i < it.pieces; ++i) {
    a += *reinterpret_cast<const f32x4*>(p + i * slot);
    b += *reinterpret_cast<const f32x4*>(p + i * slot + 4);
  }
  bf16x8 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    w[e] = static_cast<bf16>(a[e] * scale);
    w[4 + e] = static_cast<bf16>(b[e] * scale);
  }
  const int64_t token = static_cast<int64_t>(it.qrow0) + pr.query;
  *reinterpret_cast<bf16x8*>(dq + (token * H + it.head * g + pr.head) * D + col) = w;
}

template <int D, int NT>
void launch_as(const CausalArgs& a, const CausalItem* items, int n, hipStream_t s) {
  hipLaunchKernelGGL((causal_dq_kernel<D, NT>), dim3(n), dim3(NT), 0, s, static_cast<const bf16*>(a.q),
                     static_cast<const bf16*>(a.k), static_cast<const bf16*>(a.v), a.q_stride, a.k_stride, a.v_stride,
                     static_cast<const bf16*>(a.out), static_cast<const bf16*>(a.dout), a.lse, items, a.heads,
                     a.heads / a.kv_heads, a.tq, a.scale * kLog2e, a.scale, static_cast<bf16*>(a.dq), a.delta, a.partial,
                     a.trace);
}

}  // namespace

int causal_dq_rows(bool narrow) { return (narrow ? kThreadsNarrow : kThreadsWide) / 2; }
int64_t causal_dq_slot_bytes(int rows, int head_dim) { return static_cast<int64_t>(rows) * head_dim * 4; }

hipError_t launch_causal_dq(const CausalArgs& a, int rows, const CausalItem* items, int n, hipStream_t s) {
  const bool narrow = rows == causal_dq_rows(true);
  if (a.head_dim == 128)
    narrow ? launch_as<128, kThreadsNarrow>(a, items, n, s) : launch_as<128, kThreadsWide>(a, items, n, s);
  else
    narrow ? launch_as<64, kThreadsNarrow>(a, items, n, s) : launch_as<64, kThreadsWide>(a, items, n, s);
  return hipGetLastError();
}

hipError_t launch_causal_dq_join(const CausalArgs& a, int rows, const CausalItem* tiles, int n, hipStream_t s) {
  const int per = rows / (kThreads / (a.head_dim / 8));
  auto* p = static_cast<bf16*>(a.dq);
  const int g = a.heads / a.kv_heads;
  if (a.head_dim == 128)
    hipLaunchKernelGGL((causal_dq_join_kernel<128>), dim3(n * per), dim3(kThreads), 0, s, a.partial, tiles, rows,
                       a.heads, g, a.scale, p);
  else
    hipLaunchKernelGGL((causal_dq_join_kernel<64>), dim3(n * per), dim3(kThreads), 0, s, a.partial, tiles, rows,
                       a.heads, g, a.scale, p);
  return hipGetLastError();
}

#if T2V_CHECKED
hipError_t causal_dq_check_take(unsigned int* rec, unsigned int canary) { return kern::check_take_here(rec, canary); }
#endif
}  // namespace t2v
