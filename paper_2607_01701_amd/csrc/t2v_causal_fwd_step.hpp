// One 32-key step of the causal forward kernels, over keys and values in swizzled LDS tiles: scores of a wave's 32 packed rows, the online
// softmax with a lazily moved reference, and the product with the values.
#pragma once

#include "t2v_causal_device.hpp"

namespace t2v {
namespace kern {

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

struct Nothing {
  T2V_DEV void operator()() const {}
};

// One 32-key step. MASK: this lane's row sees keys 0 .. lim of the step. REST: what rounding P to bf16 for its product takes is multiplied too. c > 0.
// read(): called when all of the tiles' reads have been issued.
template <int D, bool MASK, bool REST = MASK, typename Read = Nothing>
T2V_DEV void fwd_step(uint32_t kbase, uint32_t vbase0, uint32_t vbase1, int kb, int lim, float c,
                      const bf16x8 (&qop)[D / 16], f32x16 (&o)[D / 32], float& m_run, float& l_run, int lane,
                      Read&& read = Read()) {
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
  read();
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
  // and the steps are few (errors against 64 bits at 256 tokens, of their norm: out 2.3e-3 -> 1.9e-3). So it is for single tokens over pages, whose
  // kernel waits for memory (32 tokens over 31 to 20,280 keys: 140 us without it, 141 with it). Where the matrix cores are busy, half as many
  // products again and the vector work beside them would take 232 us for 140 (three chunks over pages): there it is left out.
  const bf16x8 pb[2] = {to_bf16x8(s, 0), to_bf16x8(s, 8)};
  __builtin_amdgcn_s_setprio(kSoftmaxFirst<D> ? 0 : 1);
  const bool odd = MASK && (take_nonfinite(va[0]) | take_nonfinite(va[1]));
#pragma unroll
  for (int hf = 0; hf < 2; ++hf)
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = mfma(va[hf][db], pb[hf], o[db]);
  if constexpr (!kSoftmaxFirst<D>) __builtin_amdgcn_s_setprio(0);
  if constexpr (REST) {
    if constexpr (!MASK) {  // infinities count with P, whose sign they keep, and not with the rest, which may be 0 or negative
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) take_nonfinite(va[hf]);
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const bf16x8 rest = rest_bf16x8(s, 8 * hf, pb[hf]);
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] = mfma(va[hf][db], rest, o[db]);
    }
  }
  if constexpr (MASK) {
    if (odd)
      add_nonfinite(o, pb, G, [&](int half, int db) { return read_rows_opnd<D>(vbase0, vbase1, kb + half, db); },
                          [&](int kk, int) { return kk <= lim; });
  }
}

}  // namespace kern
}  // namespace t2v
