// Forward kernel of causal attention with grouped heads.
//
// A workgroup owns a tile of packed rows (query, head of the group) of one (sequence, key head):
// 8 waves and 256 rows, or 4 waves and 128; a wave owns 32 rows, one per lane pair. It loops over the
// keys that the tile's last row sees, staged through LDS 64 at a time and shared by all heads
// of the group. Scores are computed transposed (S^T = K Q^T), the softmax runs online over 32-key
// steps with a lazily moved reference maximum (it moves when a step exceeds it by 2^kTau). A wave skips
// steps that none of its rows sees, and masks the others from the first 64-key stage on that one of its rows does not see
// whole: three at most (with one head to a group), the first of which all rows may see. A cut loop leaves the unnormalised sums, the reference and the sum of each row in its
// slot; the join weighs and adds the pieces in order.
//
// What bounds it. At head_dim 128 the matrix cores and the card's power: they are busy 60 to 63% of the cycles, at 1,120 to
// 1,160 TFLOP/s of visible pairs (16 clips of 1,280 to 20,280 tokens, 12 heads: 4.28 to 4.33 ms; 20,280 tokens, 24
// heads over 8: 2.17 to 2.20 ms). 256 rows read a staged key eight times from LDS and once from memory; two waves a SIMD run one's
// softmax under the other's products. At 64 the vector instructions: 10.7 for each matrix instruction (5.3 at
// 128), 875 TFLOP/s (seven sequences of 77 to 6,001 tokens, 30 heads over 10: 262 us); three workgroups of 128
// rows a CU do better there than one of 256 (288 us).
// Steps that mask something run by themselves after the plain ones: code paths over the sums that meet again in one loop
// made the compiler spill.
#include "t2v_causal_device.hpp"

namespace t2v {

using namespace kern;

namespace {

constexpr int kBN = 64;  // keys per LDS stage
constexpr int kThreadsWide = 512, kThreadsNarrow = 256;

T2V_DEV float sum16(const f32x16& x) {
  float a[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = x[i] + x[i + 8];
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] += a[i + 4];
  return (a[0] + a[2]) + (a[1] + a[3]);
}

T2V_DEV float max16(const f32x16& x) {
  float a[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = max_nan(x[i], x[i + 8]);
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = max_nan(a[i], a[i + 4]);
  return max_nan(max_nan(a[0], a[2]), max_nan(a[1], a[3]));
}

// Which of the waves on a SIMD goes first: at head_dim 128 the one whose scores wait for the softmax, which the other's
// products then run beside (2 to 4% faster than without: 20,280 tokens, 24 heads over 8, 2,259 -> 2,209 us; 8 x 4,096 839 ->
// 813); at 64, where the vector unit is the scarcer one, the wave with products ready (0.5 to 1%; the other way 2% slower).
template <int D>
constexpr bool kSoftmaxFirst = D == 128;

// One 32-key step. MASK: this lane's row sees keys 0 .. lim of the step. c > 0.
template <int D, bool MASK>
T2V_DEV void fwd_step(uint32_t kbase, uint32_t vbase0, uint32_t vbase1, int kb, int lim, float c,
                      const bf16x8 (&qop)[D / 16], f32x16 (&o)[D / 32], float& m_run, float& l_run, int lane) {
  __builtin_amdgcn_iglp_opt(0);
  constexpr int KK = D / 16;
  constexpr int DB = D / 32;
  const int G = lane >> 5;
  // S^T (32 keys x 32 rows): lane = row, register r = key 8 (r / 4) + 4 G + r % 4.
  bf16x8 ka[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) ka[kk] = read_opnd<D>(kbase, kb, kk);
  f32x16 s = zero16();
  if constexpr (!kSoftmaxFirst<D>) __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) s = mfma(ka[kk], qop[kk], s);
  if constexpr (!kSoftmaxFirst<D>) __builtin_amdgcn_s_setprio(0);
  bf16x8 va[2][DB];
#pragma unroll
  for (int hf = 0; hf < 2; ++hf)
#pragma unroll
    for (int db = 0; db < DB; ++db) va[hf][db] = read_rows_opnd<D>(vbase0, vbase1, kb + hf * 16, db);
  if constexpr (kSoftmaxFirst<D>) __builtin_amdgcn_s_setprio(1);
  if constexpr (MASK) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = (r >> 2) * 8 + G * 4 + (r & 3) <= lim ? s[r] : -kInf;
  }
  const float mblk = half_max(max16(s)) * c;  // largest scaled score of this step
  if (__builtin_expect(__any(mblk > m_run + kTau), 0)) {
    // Each row by itself, so that no row's rounding depends on its neighbours in the tile.
    const float mn = mblk > m_run + kTau ? mblk : m_run;
    // A row that has seen no key (or only scores of -inf) keeps a reference of -inf: its sums are zero.
    const float alpha = __builtin_amdgcn_exp2f(m_run - (mn == -kInf ? 0.0f : mn));
    l_run *= alpha;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float x = o[db][r] * alpha;
        pin(x);  // in its place: a new tuple would be copied back in every stage (head_dim 64: 31 moves beside 166 others)
        o[db][r] = x;
      }
    m_run = mn;
  }
  const float nm = m_run == -kInf ? 0.0f : -m_run;
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, nm));  // a masked score gives 0
  l_run += sum16(s);
  // P in bf16 for its product; the row sum above took it in 32 bits. In masked steps, which hold all keys of a sequence's
  // first rows, the rest is multiplied too: those rows' few large weights make up half of a gradient's norm,
  // and the steps are few (errors against 64 bits at 256 tokens, of their norm: out 2.3e-3 -> 1.9e-3).
  const bf16x8 pb[2] = {to_bf16x8(s, 0), to_bf16x8(s, 8)};
  __builtin_amdgcn_s_setprio(kSoftmaxFirst<D> ? 0 : 1);
  const bool odd = MASK && (take_nonfinite(va[0]) | take_nonfinite(va[1]));
#pragma unroll
  for (int hf = 0; hf < 2; ++hf)
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = mfma(va[hf][db], pb[hf], o[db]);
  if constexpr (!kSoftmaxFirst<D>) __builtin_amdgcn_s_setprio(0);
  if constexpr (MASK) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const bf16x8 rest = rest_bf16x8(s, 8 * hf, pb[hf]);
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] = mfma(va[hf][db], rest, o[db]);
    }
    if (odd)
      add_nonfinite(o, pb, G, [&](int half, int db) { return read_rows_opnd<D>(vbase0, vbase1, kb + half, db); },
                          [&](int kk, int) { return kk <= lim; });
  }
}

template <int D, int NT>
__global__ __launch_bounds__(NT, 512 / NT) void causal_fwd_kernel(
    const bf16* __restrict__ q, const bf16* __restrict__ k, const bf16* __restrict__ v, int64_t qs, int64_t ks,
    int64_t vs, const CausalItem* __restrict__ items, int H, int g, int64_t T, float c, unsigned qkeep, unsigned qflip,
    bf16* __restrict__ out, float* __restrict__ lse, float* __restrict__ partial,
    unsigned long long* __restrict__ trace) {
  constexpr int KK = D / 16;
  constexpr int DB = D / 32;
  constexpr int R = NT / 2;  // rows of the tile
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
  const int lim = me.lim, lim_lo = __builtin_amdgcn_readlane(lim, 0), lim_hi = __builtin_amdgcn_readlane(lim, 31);

  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = zero16();
  float m_run = -kInf, l_run = 0.0f;

  const int ntiles = (it.end - it.begin + kBN - 1) / kBN;
  if (ntiles > 0) {
    const bf16* kh = k + it.krow0 * ks + static_cast<int64_t>(it.head) * D;
    const bf16* vh = v + it.krow0 * vs + static_cast<int64_t>(it.head) * D;
    const TileDma<D, kBN, NT> kdma(tid, ks), vdma(tid, vs);
    kdma.copy(sK[0], kh, ks, it.begin, it.lk);
    vdma.copy(sV[0], vh, vs, it.begin, it.lk);
    // A negative scale turns the sign of Q (so that the largest scaled score is that of the largest
    // product), a scale of 0 clears it.
    bf16x8 qop[KK];
    const bf16* qp = q + me.token * qs + static_cast<int64_t>(me.head) * D;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      u32x4 w = load_raw16(qp + kk * 16 + G * 8, me.ok);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (w[e] & qkeep) ^ qflip;
      qop[kk] = __builtin_bit_cast(bf16x8, w);
    }
    const uint32_t ko = opnd_lane_off<D>(lane);
    const uint32_t vo0 = rows_lane_off<D>(lane, 0), vo1 = rows_lane_off<D>(lane, 1);
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
      const uint32_t kbase = lds_addr(sK[b]) + ko;
      const uint32_t vb0 = lds_addr(sV[b]) + vo0, vb1 = lds_addr(sV[b]) + vo1;
#pragma unroll
      for (int kb = 0; kb < kBN; kb += 32)
        fwd_step<D, false>(kbase, vb0, vb1, kb, 0, c, qop, o, m_run, l_run, lane);
      wait_vmcnt0();
      __syncthreads();
    }
    for (; tt < ntiles; ++tt) {
      const int b = tt & 1;
      const int key0 = it.begin + tt * kBN;
      prefetch(tt);
      if (wave_active) {
        const uint32_t kbase = lds_addr(sK[b]) + ko;
        const uint32_t vb0 = lds_addr(sV[b]) + vo0, vb1 = lds_addr(sV[b]) + vo1;
#pragma unroll 1
        for (int kb = 0; kb < kBN && key0 + kb <= lim_hi; kb += 32)
          fwd_step<D, true>(kbase, vb0, vb1, kb, lim - key0 - kb, c, qop, o, m_run, l_run, lane);
      }
      wait_vmcnt0();
      __syncthreads();
    }
  }

  if (wave_active) {
    // Worked out again, rather than kept in registers through the loop.
    const int lane = lane_again(), G = lane >> 5, l32 = lane & 31;
    const LaneRow me = lane_row(it, g, wave, lane);
    const float lt = half_sum(l_run);
    if (it.slot >= 0) {  // one piece: unnormalised sums, reference and sum of each row
      float* po = partial + static_cast<int64_t>(it.slot) * (R * (D + 2));
      float* pm = po + R * D;
      const int r = wave * 32 + l32;
      if (me.ok) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            f32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = o[db][i * 4 + e];
            *reinterpret_cast<f32x4*>(po + r * D + db * 32 + i * 8 + G * 4) = w;
          }
        if (G == 0) {
          pm[2 * r] = m_run;
          pm[2 * r + 1] = lt;
        }
      }
    } else {
      // A row that sees no key has no softmax: its output is 0 and its lse -inf.
      const float inv = me.lim < 0 ? 0.0f : 1.0f / lt;
      bf16* op = out + (me.token * H + me.head) * D;
#pragma unroll
      for (int db = 0; db < DB; ++db) store_rows(op + db * 32, o[db], inv, G, me.ok);
      if (me.ok && G == 0)
        lse[static_cast<int64_t>(me.head) * T + me.token] = (m_run + __builtin_amdgcn_logf(lt)) * kLn2;
    }
  }
  if (trace != nullptr) trace_end(trace, trace_t0, 0, blockIdx.x);
}

// ------------------------------------------------------------------ few rows: single tokens
//
// A (sequence, key head) with at most 32 packed rows: a workgroup's four waves hold the same rows and take
// every fourth 32-key step, each through LDS buffers of its own (the copy of the next step in flight), so
// nothing but its own copies holds a wave up; the waves' sums meet in LDS at the end. The keys and values, read
// once, bound it: one workgroup a CU (two at head_dim 64) has 64 KB in flight. 32 tokens over 0.81 GB of them (40 heads over
// 8): 154 us, 5.3 TB/s, 161 with the join; 128-row tiles take 174. One token over 1,280 keys (30 heads of 64 over
// 10): 11.5 us with the join against 12.1.
constexpr int kFewRows = 32;

// Copy of 32 rows of a (sequence, key head) by one wave into a swizzled tile; rows behind the last repeat it.
// Instruction j covers RPI rows; its swizzle differs from instruction 0's by a constant.
template <int D>
struct WaveDma {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, NJ = 32 / RPI;
  int r0;
  uint32_t chunk0;
  T2V_DEV explicit WaveDma(int lane) : r0(lane / CPR), chunk0(static_cast<uint32_t>((lane % CPR) ^ swz<D>(lane / CPR))) {}
  T2V_DEV void copy(uint32_t lds, const bf16* g, int64_t rs, int row0, int L) const {
    const bf16* base = g + row0 * rs;
    const int last = L - 1 - row0;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int r = min(r0 + RPI * j, last);
      const uint32_t col = (chunk0 ^ static_cast<uint32_t>(swz<D>(RPI * j))) * 16;
#if T2V_CHECKED
      if (!check_row(row0 + r, L)) {
        dma_lds16_s(g, col, lds + j * 1024);
        continue;
      }
#endif
      dma_lds16_s(base, static_cast<uint32_t>(r) * static_cast<uint32_t>(rs * 2) + col, lds + j * 1024);
    }
  }
};

template <int D>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void causal_fwd_few_kernel(
    const bf16* __restrict__ q, const bf16* __restrict__ k, const bf16* __restrict__ v, int64_t qs, int64_t ks,
    int64_t vs, const CausalItem* __restrict__ items, int H, int g, int64_t T, float c, unsigned qkeep, unsigned qflip,
    bf16* __restrict__ out, float* __restrict__ lse, float* __restrict__ partial,
    unsigned long long* __restrict__ trace) {
  constexpr int KK = D / 16, DB = D / 32, R = kFewRows;
  constexpr int kTile = 32 * D;                       // elements of a step's K or V
  constexpr int kOps = 2 * WaveDma<D>::NJ;            // copies of a step
  __shared__ __attribute__((aligned(1024))) bf16 sKV[4][2][2][kTile];  // [wave][buffer][K, V]
  __shared__ float sM[4][R], sL[4][R];
  const unsigned long long trace_t0 = trace != nullptr ? trace_clock() : 0ull;
  const CausalItem it = items[blockIdx.x];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = lane >> 5;
  const LaneRow me = lane_row(it, g, 0, lane);
  const int lim_lo = __builtin_amdgcn_readlane(me.lim, 0);

  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = zero16();
  float m_run = -kInf, l_run = 0.0f;

  const int nsteps = (it.end - it.begin + 31) / 32;
  if (wave < nsteps) {
    const bf16* kh = k + it.krow0 * ks + static_cast<int64_t>(it.head) * D;
    const bf16* vh = v + it.krow0 * vs + static_cast<int64_t>(it.head) * D;
    const WaveDma<D> dma(lane);
    const uint32_t buf = lds_addr(sKV[wave]);
    auto fetch = [&](int n, uint32_t b) {
      dma.copy(buf + b * (4 * kTile), kh, ks, it.begin + n * 32, it.lk);
      dma.copy(buf + b * (4 * kTile) + 2 * kTile, vh, vs, it.begin + n * 32, it.lk);
    };
    fetch(wave, 0);
    bf16x8 qop[KK];
    const bf16* qp = q + me.token * qs + static_cast<int64_t>(me.head) * D;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      u32x4 w = load_raw16(qp + kk * 16 + G * 8, me.ok);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (w[e] & qkeep) ^ qflip;
      qop[kk] = __builtin_bit_cast(bf16x8, w);
      pin(qop[kk]);  // the loads end here, not between counted copies
    }
    const uint32_t ko = opnd_lane_off<D>(lane);
    const uint32_t vo0 = rows_lane_off<D>(lane, 0), vo1 = rows_lane_off<D>(lane, 1);
    uint32_t b = 0;
    for (int n = wave; n < nsteps; n += 4, b ^= 1) {
      // This wave's reads of the buffer that is filled next have returned: their results are used.
      if (n + 4 < nsteps) {
        fetch(n + 4, b ^ 1);
        wait_vmcnt<kOps>();
      } else {
        wait_vmcnt0();
      }
      asm volatile("" ::: "memory");
      const uint32_t tile = buf + b * (4 * kTile);
      const uint32_t vb = tile + 2 * kTile;
      const int key0 = it.begin + n * 32;
      if (key0 + 31 <= lim_lo)
        fwd_step<D, false>(tile + ko, vb + vo0, vb + vo1, 0, 0, c, qop, o, m_run, l_run, lane);
      else
        fwd_step<D, true>(tile + ko, vb + vo0, vb + vo1, 0, me.lim - key0, c, qop, o, m_run, l_run, lane);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // before the next copy over what this step read
    }
  }

  // The waves' sums, unnormalised and each with its own reference, in fp32: wave w's in its buffers.
  const float lt = half_sum(l_run);
  float* mine = reinterpret_cast<float*>(sKV[wave]);
  const int l32 = lane & 31;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = o[db][i * 4 + e];
      *reinterpret_cast<f32x4*>(mine + l32 * D + db * 32 + i * 8 + G * 4) = w;
    }
  if (G == 0) {
    sM[wave][l32] = m_run;
    sL[wave][l32] = lt;
  }
  __syncthreads();
  // A thread takes D / 8 columns of one row.
  constexpr int C = D / 8;
  const int r = tid >> 3, col = (tid & 7) * C;
  const LaneRow row = lane_row(it, g, 0, r);
  if (row.ok) {
    float m = sM[0][r];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = max_nan(m, sM[w][r]);
    const float ref = m == -kInf ? 0.0f : m;
    float l = 0.0f, x[C];
#pragma unroll
    for (int e = 0; e < C; ++e) x[e] = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a = __builtin_amdgcn_exp2f(sM[w][r] - ref);
      l = fmaf(a, sL[w][r], l);
      const float* src = reinterpret_cast<const float*>(sKV[w]) + r * D + col;
#pragma unroll
      for (int e = 0; e < C; ++e) x[e] = fmaf(a, src[e], x[e]);
    }
    if (it.slot >= 0) {
      float* po = partial + static_cast<int64_t>(it.slot) * (R * (D + 2));
#pragma unroll
      for (int e = 0; e < C; e += 4) *reinterpret_cast<f32x4*>(po + r * D + col + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
      if (col == 0) {
        po[R * D + 2 * r] = m;
        po[R * D + 2 * r + 1] = l;
      }
    } else {
      const float inv = row.lim < 0 ? 0.0f : 1.0f / l;
      bf16* op = out + (row.token * H + row.head) * D + col;
#pragma unroll
      for (int e = 0; e < C; e += 8) {
        bf16x8 w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = static_cast<bf16>(x[e + i] * inv);
        *reinterpret_cast<bf16x8*>(op + e) = w;
      }
      if (col == 0) lse[static_cast<int64_t>(row.head) * T + row.token] = (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
  }
  if (trace != nullptr) trace_end(trace, trace_t0, 0, blockIdx.x);
}

// Joins the pieces of the cut tiles: with the largest reference m of a row, out = sum_p 2^(m_p - m) O_p / l,
// l = sum_p 2^(m_p - m) l_p, in piece order. D / 8 lanes hold a row, eight columns each; they read the
// references and sums of D / 8 pieces at once, and the sums of several pieces are in flight together. Bound by the pieces'
// bytes: 26 MB in 6.4 us.
template <int D>
__global__ __launch_bounds__(kThreads) void causal_fwd_join_kernel(const float* __restrict__ partial,
                                                                    const CausalItem* __restrict__ tiles, int R, int H,
                                                                    int g, int64_t T, bf16* __restrict__ out,
                                                                    float* __restrict__ lse) {
  constexpr int LPR = D / 8, RPB = kThreads / LPR;
  const int blocks = R / RPB;
  const CausalItem it = tiles[blockIdx.x / blocks];
  const int r = (blockIdx.x % blocks) * RPB + threadIdx.x / LPR;  // row of the tile
  const int sub = threadIdx.x % LPR, col = sub * 8;
  const int row = it.tile0 + r;
  if (row >= it.lq * g) return;  // all lanes of a row alike
  const PackedRow pr = packed_row(row, g);
  const int64_t slot = static_cast<int64_t>(R) * (D + 2);
  const float* po = partial + it.slot * slot;
  const float* pm = po + R * D + 2 * r;
  po += r * D + col;
  float m = -kInf;
  for (int p = sub; p < it.pieces; p += LPR) m = max_nan(m, pm[p * slot]);
#pragma unroll
  for (int off = LPR / 2; off > 0; off >>= 1) m = max_nan(m, __shfl_xor(m, off, LPR));
  const float ref = m == -kInf ? 0.0f : m;
  float l = 0.0f;
  f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f}, b = a;
  for (int p0 = 0; p0 < it.pieces; p0 += LPR) {
    const int mine = p0 + sub;
    const bool has = mine < it.pieces;
    const float w_mine = has ? __builtin_amdgcn_exp2f(pm[mine * slot] - ref) : 0.0f;
    const float l_mine = has ? pm[mine * slot + 1] : 0.0f;
    const int n = min(LPR, it.pieces - p0);
    const float* x = po + p0 * slot;
#pragma unroll 4
    for (int p = 0; p < n; ++p) {
      const float w = __shfl(w_mine, p, LPR);
      l = fmaf(w, __shfl(l_mine, p, LPR), l);
      const f32x4 u = *reinterpret_cast<const f32x4*>(x + p * slot);
      const f32x4 v = *reinterpret_cast<const f32x4*>(x + p * slot + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[e] = fmaf(w, u[e], a[e]);
        b[e] = fmaf(w, v[e], b[e]);
      }
    }
  }
  const float inv = pr.query + it.lk - it.lq < 0 ? 0.0f : 1.0f / l;
  const int64_t token = static_cast<int64_t>(it.qrow0) + pr.query;
  const int head = it.head * g + pr.head;
  bf16x8 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    w[e] = static_cast<bf16>(a[e] * inv);
    w[4 + e] = static_cast<bf16>(b[e] * inv);
  }
  *reinterpret_cast<bf16x8*>(out + (token * H + head) * D + col) = w;
  if (col == 0) lse[static_cast<int64_t>(head) * T + token] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int D, int NT>  // NT 0: the kernel of few rows
void launch_as(const CausalArgs& a, const CausalItem* items, int n, hipStream_t s) {
  const float c = a.scale == 0.0f ? 1.0f : fabsf(a.scale) * kLog2e;
  const unsigned keep = a.scale == 0.0f ? 0u : ~0u, flip = a.scale < 0.0f ? 0x80008000u : 0u;
  auto launch = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, dim3(n), dim3(threads), 0, s, static_cast<const bf16*>(a.q), static_cast<const bf16*>(a.k),
                       static_cast<const bf16*>(a.v), a.q_stride, a.k_stride, a.v_stride, items, a.heads,
                       a.heads / a.kv_heads, a.tq, c, keep, flip, static_cast<bf16*>(a.out), a.lse, a.partial, a.trace);
  };
  if constexpr (NT == 0)
    launch(causal_fwd_few_kernel<D>, 256);
  else
    launch(causal_fwd_kernel<D, NT>, NT);
}

}  // namespace

int causal_fwd_rows(bool narrow) { return (narrow ? kThreadsNarrow : kThreadsWide) / 2; }
int causal_fwd_few_rows() { return kFewRows; }
int64_t causal_fwd_slot_bytes(int rows, int head_dim) { return static_cast<int64_t>(rows) * (head_dim + 2) * 4; }

hipError_t launch_causal_fwd(const CausalArgs& a, int rows, const CausalItem* items, int n, hipStream_t s) {
  const bool narrow = rows == causal_fwd_rows(true), d128 = a.head_dim == 128;
  if (rows == kFewRows)
    d128 ? launch_as<128, 0>(a, items, n, s) : launch_as<64, 0>(a, items, n, s);
  else if (d128)
    narrow ? launch_as<128, kThreadsNarrow>(a, items, n, s) : launch_as<128, kThreadsWide>(a, items, n, s);
  else
    narrow ? launch_as<64, kThreadsNarrow>(a, items, n, s) : launch_as<64, kThreadsWide>(a, items, n, s);
  return hipGetLastError();
}

hipError_t launch_causal_fwd_join(const CausalArgs& a, int rows, const CausalItem* tiles, int n, hipStream_t s) {
  const int per = rows / (kThreads / (a.head_dim / 8));
  auto* o = static_cast<bf16*>(a.out);
  const int g = a.heads / a.kv_heads;
  if (a.head_dim == 128)
    hipLaunchKernelGGL((causal_fwd_join_kernel<128>), dim3(n * per), dim3(kThreads), 0, s, a.partial, tiles, rows,
                       a.heads, g, a.tq, o, a.lse);
  else
    hipLaunchKernelGGL((causal_fwd_join_kernel<64>), dim3(n * per), dim3(kThreads), 0, s, a.partial, tiles, rows,
                       a.heads, g, a.tq, o, a.lse);
  return hipGetLastError();
}

#if T2V_CHECKED
hipError_t causal_fwd_check_take(unsigned int* rec, unsigned int canary) { return kern::check_take_here(rec, canary); }
#endif
}  // namespace t2v
