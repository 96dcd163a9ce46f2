// Norms of the heads of q and k with the rotary turn after them: y = R(p f) (w x r), r = 1 / sqrt(mean x^2 + eps), over a
// head's D elements; and the backward pass, with dn = R^T dy and x^ = x r: dx = r (w dn - x^ mean(w dn x^)), dw = sum dn x^.
//
// A row (token, head) is held by L = D / 16 lanes, 16 elements each in two 16-byte vectors that hold both elements of
// eight pairs, so that the turn stays within a lane and the norm's sums take log2 L steps between neighbouring lanes; the lanes of a row read
// two runs of consecutive bytes. Pairs (j, j + n) with n no multiple of 8 have no such vectors: there a row goes through LDS in 32 bits
// (VIA_LDS). Sines and cosines are worked out once a token and shared by its heads through LDS, after the first loads.
//
// Bound by memory, each element being read and written once (backward: two read, one written): 116,904 tokens of 24 + 24 heads of 128
// forward 476 us, 6.0 TB/s (in a training step, behind a backward pass, 489), backward 819 us, 5.3 TB/s; 20,280 tokens of 24 + 8 heads 57 us, 5.8 TB/s; through LDS (14,750 tokens of 30 + 10
// heads of 64, 36 dimensions turned) 37 and 50 us. Forward, many short workgroups with one row a lane in flight are fastest: with two rows
// 514 us of the 492 that it takes without the marks of set_once, with 2 tokens a workgroup in place of 1 525, with 8 555. Backward, 512
// workgroups, which leave few sums for the weights, lose nothing (512 to 32,768 of them with tokens of their own: 846 to 870 us), and marks gain
// nothing (860 to 889).
#include <algorithm>
#include <cmath>
#include <string>
#include <vector>

#include "../../include/t2vattn.h"
#include "t2v_device.hpp"
#include "t2v_host.h"
#include "t2v_paged_host.h"
#include "t2v_rotary.hpp"

namespace t2v {
namespace {

constexpr int kThreads = 256;
constexpr int kElems = 16;        // of a lane
constexpr int kRows = 1;          // in flight per lane, forward
constexpr int kLeastRows128 = 48; // of a workgroup at head_dim 128, four times as many at 64
constexpr int kRowsBack = 2;      // backward
constexpr int kMaxAngles = 2048;  // of a workgroup's tokens (16 KB of LDS)
constexpr int kMaxBackBlocks = 512;
constexpr int kChunkBack = 8;     // tokens

struct NormArgs {
  const bf16* in[2];    // q, k
  const bf16* grad[2];  // backward: the gradients of the outputs
  bf16* out[2];
  int64_t stride[2], grad_stride[2];  // elements between tokens; outputs are contiguous
  int heads[2];
  const void* weight[2];
  void* dweight[2];
  int weights_f32;
  int norm;
  float eps;
  const int32_t* positions;  // [axes, tokens]
  int64_t tokens;
  int pairs;
  float mscale;
  float* partial;  // backward: [blocks, 2, D]
  int read_once, write_once;  // forward: inputs and outputs that the caches need not keep
  RotaryAngles angles;
};

typedef __attribute__((address_space(1))) bf16 gbf16;
typedef __attribute__((address_space(1))) u32x4 gu32x4;
T2V_DEV bf16x8 load_vec(const gbf16* p) { return __builtin_bit_cast(bf16x8, *(const gu32x4*)(p)); }
T2V_DEV void store_vec(gbf16* p, const bf16x8& x) { *(gu32x4*)(p) = __builtin_bit_cast(u32x4, x); }

// A lane's two vectors; once: bytes that the caches need not keep. (The empty assembly keeps the compiler from making one access, without
// the mark, of the two.)
T2V_DEV void load_row(bf16x8& x, bf16x8& y, const gbf16* p, const gbf16* q, int once) {
  if (once) {
    asm volatile("");
    x = __builtin_bit_cast(bf16x8, __builtin_nontemporal_load((const gu32x4*)(p)));
    y = __builtin_bit_cast(bf16x8, __builtin_nontemporal_load((const gu32x4*)(q)));
    asm volatile("");
  } else {
    x = load_vec(p);
    y = load_vec(q);
  }
}
T2V_DEV void store_row(gbf16* p, gbf16* q, const bf16x8& x, const bf16x8& y, int once) {
  if (once) {
    asm volatile("");
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), (gu32x4*)(p));
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, y), (gu32x4*)(q));
    asm volatile("");
  } else {
    store_vec(p, x);
    store_vec(q, y);
  }
}

// Sum over the L neighbouring lanes of a row, in every one of them.
template <int L>
T2V_DEV float row_sum(float x) {
  auto add = [&](auto ctrl) {
    const int o = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true);
    x += __builtin_bit_cast(float, o);
  };
  add(std::integral_constant<int, 0xB1>{});  // lane ^ 1
  add(std::integral_constant<int, 0x4E>{});  // lane ^ 2
  if constexpr (L == 8) add(std::integral_constant<int, 0x141>{});  // the other four of eight
  return x;
}

// 1 / sqrt(mean x^2 + eps) of a row, f its elements' factor: 1, or, where the mean leaves the range in which 32 bits hold the squares of all that count, a power of
// two by which u is multiplied first (a head of 2^70, or of 2^-80 with eps 0), and the reciprocal root is of the multiplied row.
template <int D>
T2V_DEV float row_root(float (&u)[kElems], float eps, float& f) {
  constexpr int L = D / kElems;
  auto mean = [&](float add) {
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < kElems; ++e) s = fmaf(u[e], u[e], s);
    return row_sum<L>(s) * (1.0f / D) + add;
  };
  float m = mean(eps);
  f = 1.0f;
  if (__builtin_expect(!(m >= 0x1p-90f && m <= 0x1p120f), 0)) {  // alike in a row's lanes
    f = m < 1.0f ? 0x1p80f : 0x1p-70f;
#pragma unroll
    for (int e = 0; e < kElems; ++e) u[e] *= f;
    m = mean(eps * f * f);
  }
  return rsqrtf(m);
}

// Places of a lane's two vectors within a row, and what of them turns.
template <int D, bool INTERLEAVED, bool VIA_LDS>
struct RowLane {
  static constexpr int L = D / kElems;
  int v0, v1;
  // Pair e of the eight that the lane turns. (Those of dimensions that are copied are no pair's; their numbers are not below `pairs`.)
  T2V_DEV static int pair(int sub, int e) { return INTERLEAVED ? 4 * sub + (e < 4 ? e : D / 4 + e - 4) : 8 * sub + e; }
  T2V_DEV RowLane(int sub, int pairs) {
    if constexpr (VIA_LDS || INTERLEAVED) {
      v0 = 8 * sub;
      v1 = D / 2 + 8 * sub;
    } else {  // pairs is a multiple of 8: lanes hold pairs 8 sub .. 8 sub + 7, or share what follows the turned dimensions
      v0 = 8 * sub < pairs ? 8 * sub : 8 * sub + pairs;
      v1 = v0 + (8 * sub < pairs ? pairs : D / 2 - pairs);
    }
  }
};

T2V_DEV void lds_step() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Turns a row in place: u holds this lane's 16 elements (of v0, then v1), row[p] cosine and sine of pair p.
// buf: D floats of this row's own in LDS (VIA_LDS).
template <int D, bool INTERLEAVED, bool VIA_LDS>
T2V_DEV void turn_row(float (&u)[kElems], const float2* row, int pairs, int sub, const RowLane<D, INTERLEAVED, VIA_LDS>& at,
                      float* buf) {
  float a[8], b[8];
  if constexpr (VIA_LDS) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      buf[at.v0 + e] = u[e];
      buf[at.v1 + e] = u[8 + e];
    }
    lds_step();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int p = 8 * sub + e;
      a[e] = buf[p < pairs ? p : 2 * p];
      b[e] = buf[p < pairs ? p + pairs : 2 * p + 1];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      a[e] = INTERLEAVED ? u[2 * e] : u[e];
      b[e] = INTERLEAVED ? u[2 * e + 1] : u[8 + e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int p = at.pair(sub, e);
    const float2 k = row[p];
    const bool turned = p < pairs;  // chosen, not multiplied by 1 and 0: the others may hold an infinity
    const float c = fmaf(a[e], k.x, -(b[e] * k.y)), d = fmaf(a[e], k.y, b[e] * k.x);
    a[e] = turned ? c : a[e];
    b[e] = turned ? d : b[e];
  }
  if constexpr (VIA_LDS) {
    lds_step();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int p = 8 * sub + e;
      buf[p < pairs ? p : 2 * p] = a[e];
      buf[p < pairs ? p + pairs : 2 * p + 1] = b[e];
    }
    lds_step();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[e] = buf[at.v0 + e];
      u[8 + e] = buf[at.v1 + e];
    }
    lds_step();
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[INTERLEAVED ? 2 * e : e] = a[e];
      u[INTERLEAVED ? 2 * e + 1 : 8 + e] = b[e];
    }
  }
}

T2V_DEV void unpack(float (&u)[kElems], const bf16x8& x, const bf16x8& y) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    u[e] = static_cast<float>(x[e]);
    u[8 + e] = static_cast<float>(y[e]);
  }
}
T2V_DEV bf16x8 packed(const float (&u)[kElems], int first) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = static_cast<bf16>(u[first + e]);
  return r;
}

// Weights of q and k (ones where there are none) to LDS, in 32 bits.
template <int D>
T2V_DEV void load_weights(float (&wt)[2][D], const NormArgs& a) {
  for (int e = threadIdx.x; e < 2 * D; e += kThreads) {
    const int which = e / D, d = e % D;
    const void* w = which ? a.weight[1] : a.weight[0];
    wt[which][d] = w == nullptr ? 1.0f
                   : a.weights_f32 ? static_cast<const float*>(w)[d]
                                   : static_cast<float>(static_cast<const bf16*>(w)[d]);
  }
}

// Cosines and sines (times mscale; sign -1: of the turn back) of tokens t0 .. t0 + nt - 1.
template <int D>
T2V_DEV void load_angles(float2* cs, const NormArgs& a, int64_t t0, int nt, float sign) {
  for (int e = threadIdx.x; e < nt * a.pairs; e += kThreads) {
    const int t = e / a.pairs, j = e - t * a.pairs;
    const float2 k = angle_of(a.angles, j, a.positions[a.angles.axis[j] * a.tokens + t0 + t]);
    cs[t * (D / 2) + j] = make_float2(k.x * a.mscale, sign * k.y * a.mscale);
  }
}

// Where a group of lanes is: head h (q's, then k's) of the workgroup's token t; it moves by as many rows as there are groups.
struct RowPlace {
  int t, h;
};

template <int D, bool INTERLEAVED, bool VIA_LDS>
__global__ __launch_bounds__(kThreads) void norm_rotary_kernel(const NormArgs a, int tokens_per_block) {
  using Lane = RowLane<D, INTERLEAVED, VIA_LDS>;
  constexpr int L = Lane::L, NG = kThreads / L;
  __shared__ __attribute__((aligned(16))) float2 cs[kMaxAngles];
  __shared__ __attribute__((aligned(16))) float wt[2][D];
  __shared__ float ex[VIA_LDS ? NG * (D + 4) : 1];
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * tokens_per_block;
  const int nt = static_cast<int>(min(static_cast<int64_t>(tokens_per_block), a.tokens - t0));
  const int hq = a.heads[0], heads = hq + a.heads[1], total = nt * heads;
  const int sub = threadIdx.x % L, group = threadIdx.x / L;
  const Lane at(sub, a.pairs);
  float* buf = ex + (VIA_LDS ? group * (D + 4) : 0);
  const int st = NG / heads, sh = NG % heads;
  auto advance = [&](RowPlace& x) {
    x.h += sh;
    const int c = x.h >= heads;
    x.h -= c ? heads : 0;
    x.t += st + c;
  };
  // A row's tensor is picked from scalar registers: a choice between two arguments would become a load from the
  // argument block at an address of the lane's.
  const gbf16 *q = (const gbf16*)(a.in[0]), *k = (const gbf16*)(a.in[1]);
  gbf16 *qo = (gbf16*)(a.out[0]), *ko = (gbf16*)(a.out[1]);
  int64_t qs = a.stride[0], ks = a.stride[1];
  asm volatile("" : "+s"(q), "+s"(k), "+s"(qo), "+s"(ko), "+s"(qs), "+s"(ks));
  auto source = [&](const RowPlace& x) {
    const bool second = x.h >= hq;
    return (second ? k : q) + (t0 + x.t) * (second ? ks : qs) + static_cast<int64_t>(x.h - (second ? hq : 0)) * D;
  };
  auto target = [&](const RowPlace& x) {
    const bool second = x.h >= hq;
    return (second ? ko : qo) + ((t0 + x.t) * (second ? heads - hq : hq) + (x.h - (second ? hq : 0))) * D;
  };
  RowPlace w{group / heads, group % heads};
  bf16x8 x[kRows], y[kRows];
  auto load = [&](RowPlace p, int r0) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (r0 + i * NG < total) {
        const gbf16* s = source(p);
        load_row(x[i], y[i], s + at.v0, s + at.v1, a.read_once);
      }
      advance(p);
    }
  };
  load(w, group);
  load_weights<D>(wt, a);
  load_angles<D>(cs, a, t0, nt, 1.0f);
  __syncthreads();
  for (int r0 = group; r0 < total; r0 += kRows * NG) {
    if (r0 != group) load(w, r0);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (r0 + i * NG < total) {
        float u[kElems];
        unpack(u, x[i], y[i]);
        if (a.norm) {
          float f;
          const float r = row_root<D>(u, a.eps, f);
          const float* wr = wt[w.h >= hq];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            u[e] = u[e] * r * wr[at.v0 + e];
            u[8 + e] = u[8 + e] * r * wr[at.v1 + e];
          }
        }
        if (a.pairs > 0) turn_row(u, cs + w.t * (D / 2), a.pairs, sub, at, buf);
        gbf16* o = target(w);
        store_row(o + at.v0, o + at.v1, packed(u, 0), packed(u, 8), a.write_once);
      }
      advance(w);
    }
  }
}

// A workgroup takes `chunk` tokens at a time (their angles are in its table), every gridDim-th such chunk, q's heads and then k's, and
// leaves its sums for the weights in partial[block].
template <int D, bool INTERLEAVED, bool VIA_LDS>
__global__ __launch_bounds__(kThreads) void norm_rotary_bwd_kernel(const NormArgs a, int chunk) {
  using Lane = RowLane<D, INTERLEAVED, VIA_LDS>;
  constexpr int L = Lane::L, NG = kThreads / L;
  __shared__ __attribute__((aligned(16))) float2 cs[kMaxAngles];
  __shared__ __attribute__((aligned(16))) float wt[2][D];
  __shared__ float ex[VIA_LDS ? NG * (D + 4) : 1];
  const int sub = threadIdx.x % L, group = threadIdx.x / L;
  const Lane at(sub, a.pairs);
  float* buf = ex + (VIA_LDS ? group * (D + 4) : 0);
  load_weights<D>(wt, a);
  float dw[2][kElems];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < kElems; ++e) dw[i][e] = 0.0f;
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * chunk; t0 < a.tokens; t0 += static_cast<int64_t>(gridDim.x) * chunk) {
    const int nt = static_cast<int>(min(static_cast<int64_t>(chunk), a.tokens - t0));
    __syncthreads();
    load_angles<D>(cs, a, t0, nt, -1.0f);
    __syncthreads();
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const int heads = a.heads[which], total = nt * heads;
      if (heads == 0) continue;
      const gbf16 *in = (const gbf16*)(a.in[which]), *grad = (const gbf16*)(a.grad[which]);
      gbf16* out = (gbf16*)(a.out[which]);
      const int64_t xs = a.stride[which], gs = a.grad_stride[which];
      const int st = NG / heads, sh = NG % heads;
      auto advance = [&](RowPlace& x) {
        x.h += sh;
        const int c = x.h >= heads;
        x.h -= c ? heads : 0;
        x.t += st + c;
      };
      RowPlace w{group / heads, group % heads};
      for (int r0 = group; r0 < total; r0 += kRowsBack * NG) {
        bf16x8 x[kRowsBack][2], g[kRowsBack][2];
        RowPlace p = w;
#pragma unroll
        for (int i = 0; i < kRowsBack; ++i) {
          if (r0 + i * NG < total) {
            const gbf16* s = in + (t0 + p.t) * xs + p.h * D;
            const gbf16* d = grad + (t0 + p.t) * gs + p.h * D;
            x[i][0] = load_vec(s + at.v0);
            x[i][1] = load_vec(s + at.v1);
            g[i][0] = load_vec(d + at.v0);
            g[i][1] = load_vec(d + at.v1);
          }
          advance(p);
        }
#pragma unroll
        for (int i = 0; i < kRowsBack; ++i) {
          if (r0 + i * NG < total) {
            float u[kElems], v[kElems];
            unpack(u, x[i][0], x[i][1]);
            unpack(v, g[i][0], g[i][1]);
            if (a.pairs > 0) turn_row(v, cs + w.t * (D / 2), a.pairs, sub, at, buf);
            float f;
            const float r = row_root<D>(u, a.eps, f);
            float c = 0.0f;
#pragma unroll
            for (int e = 0; e < kElems; ++e) {
              u[e] *= r;
              dw[which][e] = fmaf(v[e], u[e], dw[which][e]);
              v[e] *= wt[which][(e < 8 ? at.v0 : at.v1 - 8) + e];
              c = fmaf(v[e], u[e], c);
            }
            c = row_sum<L>(c) * (1.0f / D);
#pragma unroll
            for (int e = 0; e < kElems; ++e) v[e] = r * fmaf(-u[e], c, v[e]) * f;
            gbf16* o = out + ((t0 + w.t) * heads + w.h) * D;
            store_vec(o + at.v0, packed(v, 0));
            store_vec(o + at.v1, packed(v, 8));
          }
          advance(w);
        }
      }
    }
  }
  if (a.partial == nullptr) return;
  // The groups' sums, in their order.
  float* sums = reinterpret_cast<float*>(cs);  // [NG][D]
  static_assert(sizeof(cs) >= NG * D * sizeof(float), "the groups' sums fit the angles' place");
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kElems; ++e) sums[group * D + (e < 8 ? at.v0 : at.v1 - 8) + e] = dw[which][e];
    __syncthreads();
    if (threadIdx.x < D) {
      float s = 0.0f;
      for (int g = 0; g < NG; ++g) s += sums[g * D + threadIdx.x];
      a.partial[(static_cast<int64_t>(blockIdx.x) * 2 + which) * D + threadIdx.x] = s;
    }
  }
}

// dw of one dimension: the workgroups' sums, every 256th by a thread and then the threads' in order.
template <int D>
__global__ __launch_bounds__(kThreads) void norm_weights_kernel(const float* partial, int blocks, int weights_f32, void* dq,
                                                                void* dk) {
  __shared__ float sums[kThreads];
  const int which = blockIdx.x / D, d = blockIdx.x % D;
  float s = 0.0f;
  for (int b = threadIdx.x; b < blocks; b += kThreads) s += partial[(static_cast<int64_t>(b) * 2 + which) * D + d];
  sums[threadIdx.x] = s;
  for (int n = kThreads / 2; n > 0; n /= 2) {
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < n) sums[threadIdx.x] += sums[threadIdx.x + n];
  }
  if (threadIdx.x != 0) return;
  void* o = which ? dk : dq;
  if (o == nullptr) return;
  if (weights_f32)
    static_cast<float*>(o)[d] = sums[0];
  else
    static_cast<bf16*>(o)[d] = static_cast<bf16>(sums[0]);
}

// ------------------------------------------------------------------ storing in pages

struct AppendArgs {
  NormArgs n;  // q and k (its out[1] is not used)
  const bf16* v;
  int64_t v_stride;
  bf16 *k_pages, *v_pages;
  int64_t k_page, k_token, k_head, v_page, v_token, v_head;  // strides in elements
  const int32_t *cu, *lengths, *table;
  int64_t table_stride;
  int nseq, pages, shift, room;
};

constexpr int kMaxTokens = 2 * kMaxAngles / 64;  // of a workgroup

// Page and row of token i, {-1, 0} if it has none, {-2, 0} behind the last sequence.
T2V_DEV int2 place_of(const AppendArgs& a, int64_t i) {
  int lo = 0, hi = a.nseq;  // the last s with cu[s] <= i
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.cu[mid] <= i)
      lo = mid;
    else
      hi = mid - 1;
  }
  if (lo == a.nseq || a.cu[lo] > i) return make_int2(-2, 0);
  const int64_t key = a.lengths[lo] - (a.cu[lo + 1] - i);
  if (key < 0 || key >= a.room || a.lengths[lo] > a.room) return make_int2(-1, 0);
  const int page = a.table[lo * a.table_stride + (key >> a.shift)];
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.pages)) return make_int2(-1, 0);
  return make_int2(page, static_cast<int>(key) & ((1 << a.shift) - 1));
}

// c ? b : a, chosen as a value: a choice of three variables would become a choice of their addresses, and these stay in memory.
template <typename T>
T2V_DEV T pick(T a, T b, bool c) {
  T x = c ? b : a;
  asm("" : "+v"(x));
  return x;
}

// As norm_rotary_kernel, with a token's heads of v after those of q and k.
template <int D, bool INTERLEAVED, bool VIA_LDS>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(const AppendArgs p, int tokens_per_block) {
  const NormArgs& a = p.n;
  using Lane = RowLane<D, INTERLEAVED, VIA_LDS>;
  constexpr int L = Lane::L, NG = kThreads / L;
  __shared__ __attribute__((aligned(16))) float2 cs[kMaxAngles];
  __shared__ __attribute__((aligned(16))) float wt[2][D];
  __shared__ int2 place[kMaxTokens];
  __shared__ float ex[VIA_LDS ? NG * (D + 4) : 1];
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * tokens_per_block;
  const int nt = static_cast<int>(min(static_cast<int64_t>(tokens_per_block), a.tokens - t0));
  const int hq = a.heads[0], hk = a.heads[1], heads = hq + 2 * hk, total = nt * heads;
  const int sub = threadIdx.x % L, group = threadIdx.x / L;
  const Lane at(sub, a.pairs);
  float* buf = ex + (VIA_LDS ? group * (D + 4) : 0);
  const int st = NG / heads, sh = NG % heads;
  auto advance = [&](RowPlace& x) {
    x.h += sh;
    const int c = x.h >= heads;
    x.h -= c ? heads : 0;
    x.t += st + c;
  };
  const gbf16 *q = (const gbf16*)(a.in[0]), *k = (const gbf16*)(a.in[1]), *v = (const gbf16*)(p.v);
  int64_t qs = a.stride[0], ks = a.stride[1], vs = p.v_stride;
  gbf16 *qo = (gbf16*)(a.out[0]), *ko = (gbf16*)(p.k_pages), *vo = (gbf16*)(p.v_pages);
  int64_t kp = p.k_page, kt = p.k_token, kh = p.k_head, vp = p.v_page, vt = p.v_token, vh = p.v_head;
  // Picked from scalar registers, as above.
  asm volatile("" : "+s"(q), "+s"(k), "+s"(v), "+s"(qs), "+s"(ks), "+s"(vs), "+s"(qo), "+s"(ko), "+s"(vo));
  asm volatile("" : "+s"(kp), "+s"(kt), "+s"(kh), "+s"(vp), "+s"(vt), "+s"(vh));
  auto source = [&](const RowPlace& x) {
    const bool not_q = x.h >= hq, is_v = x.h >= hq + hk;
    return pick(pick(q, k, not_q), v, is_v) + (t0 + x.t) * pick(pick(qs, ks, not_q), vs, is_v) +
           static_cast<int64_t>(x.h - (is_v ? hq + hk : not_q ? hq : 0)) * D;
  };
  RowPlace w{group / heads, group % heads};
  bf16x8 x[kRows], y[kRows];
  auto load = [&](RowPlace r, int r0) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (r0 + i * NG < total) {
        const gbf16* s = source(r);
        load_row(x[i], y[i], s + at.v0, s + at.v1, a.read_once);
      }
      advance(r);
    }
  };
  load(w, group);
  if (static_cast<int>(threadIdx.x) < nt) place[threadIdx.x] = place_of(p, t0 + threadIdx.x);
  load_weights<D>(wt, a);
  load_angles<D>(cs, a, t0, nt, 1.0f);
  __syncthreads();
  const bool plain = !a.norm && a.pairs == 0;
  for (int r0 = group; r0 < total; r0 += kRows * NG) {
    if (r0 != group) load(w, r0);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const bool not_q = w.h >= hq, is_v = w.h >= hq + hk;
      int2 to = make_int2(-2, 0);
      if (r0 + i * NG < total) to = place[w.t];
      if (to.x >= (not_q ? 0 : -1)) {
        bf16x8 z0 = x[i], z1 = y[i];
        if (!is_v && !plain) {
          float u[kElems];
          unpack(u, z0, z1);
          if (a.norm) {
            float f;
            const float r = row_root<D>(u, a.eps, f);
            const float* wr = wt[not_q];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              u[e] = u[e] * r * wr[at.v0 + e];
              u[8 + e] = u[8 + e] * r * wr[at.v1 + e];
            }
          }
          if (a.pairs > 0) turn_row(u, cs + w.t * (D / 2), a.pairs, sub, at, buf);
          z0 = packed(u, 0);
          z1 = packed(u, 8);
        }
        gbf16* o = qo + ((t0 + w.t) * hq + w.h) * D;
        if (not_q)
          o = pick(ko, vo, is_v) + to.x * pick(kp, vp, is_v) + to.y * pick(kt, vt, is_v) + (w.h - (is_v ? hq + hk : hq)) * pick(kh, vh, is_v);
        store_row(o + at.v0, o + at.v1, z0, z1, a.write_once);
      }
      advance(w);
    }
  }
}

// ------------------------------------------------------------------------ host

int bad(const std::string& what) { return set_error(T2V_ERR_INVALID_ARG, what); }

bool via_lds(const NormArgs& a, bool interleaved) { return !interleaved && a.pairs % 8 != 0; }

// f with the kernel's template arguments.
template <typename F>
void with_form(const NormArgs& a, int head_dim, bool interleaved, F&& f) {
  const bool lds = via_lds(a, interleaved);
  auto pick = [&](auto d) {
    if (interleaved)
      f(d, std::true_type{}, std::false_type{});
    else if (lds)
      f(d, std::false_type{}, std::true_type{});
    else
      f(d, std::false_type{}, std::false_type{});
  };
  head_dim == 128 ? pick(std::integral_constant<int, 128>{}) : pick(std::integral_constant<int, 64>{});
}

// Checks what t2v_turn says and fills a's part of it; *read gets the ranges that a kernel reads, *axes the positions' rows.
int check_turn(const t2v_turn* t, int head_dim, int heads, int kv_heads, NormArgs* a, bool* interleaved, int* axes,
               std::vector<Range>* read) {
  if (t == nullptr) return bad("turn is NULL");
  if (t->n_sections != 0) {
    int64_t pairs = 0;
    if (int st = check_rotary(t->freqs, t->sections, t->n_sections, t->layout, t->mscale, head_dim, &pairs)) return st;
    a->pairs = static_cast<int>(pairs);
    a->mscale = t->mscale;
    fill_angles(&a->angles, t->freqs, t->sections, t->n_sections);
  }
  *axes = t->n_sections;
  *interleaved = t->n_sections != 0 && t->layout == T2V_ROTARY_INTERLEAVED;
  if (std::isnan(t->eps) || std::isinf(t->eps)) return bad("eps must be finite");
  a->norm = t->eps >= 0.0f;
  a->eps = t->eps;
  a->weights_f32 = t->weights_f32 != 0;
  const struct {
    const void* w;
    int heads;
    const char* name;
  } weights[2] = {{t->q_weight, heads, "q_weight"}, {t->k_weight, kv_heads, "k_weight"}};
  for (int i = 0; i < 2; ++i) {
    if (weights[i].w == nullptr || weights[i].heads == 0) continue;
    if (!a->norm) return bad(std::string(weights[i].name) + " is given without a norm (eps < 0)");
    a->weight[i] = weights[i].w;
    read->push_back({weights[i].w, head_dim * (t->weights_f32 ? 4 : 2), weights[i].name});
  }
  return T2V_OK;
}

int check_heads(int64_t tokens, int heads, int kv_heads, int head_dim) {
  if (head_dim != 64 && head_dim != 128)
    return set_error(T2V_ERR_UNSUPPORTED, "head_dim must be 64 or 128, got " + std::to_string(head_dim));
  if (tokens < 0 || tokens > INT32_MAX) return bad("tokens must be in 0 .. 2^31 - 1");
  if (heads < 0 || kv_heads < 0 || heads + static_cast<int64_t>(kv_heads) < 1)
    return bad("heads and kv_heads must be >= 0, and one of them >= 1");
  if ((heads + static_cast<int64_t>(kv_heads)) * head_dim > (int64_t(1) << 22)) return bad("heads * head_dim is too large");
  return T2V_OK;
}

int check_stride(int64_t stride, int heads, int head_dim, const char* name) {
  if (heads == 0 || (stride >= static_cast<int64_t>(heads) * head_dim && stride % 8 == 0 && stride <= (int64_t(1) << 22)))
    return T2V_OK;
  return bad(std::string(name) + " must be a multiple of 8 between heads * head_dim and 2^22, got " + std::to_string(stride));
}

int64_t rows_bytes(int64_t tokens, int64_t stride, int heads, int head_dim) {
  return 2 * ((tokens - 1) * stride + static_cast<int64_t>(heads) * head_dim);
}

// The positions (4-byte aligned) against the outputs; the other pointers by validate_pointers.
int check_pointers(const NormArgs& a, int axes, const std::vector<Range>& in, const std::vector<Range>& out) {
  if (int st = validate_pointers(in, out)) return st;
  if (axes == 0) return T2V_OK;
  if (a.positions == nullptr) return bad("positions is NULL");
  if (reinterpret_cast<uintptr_t>(a.positions) % 4 != 0) return bad("positions is not 4-byte aligned");
  for (const Range& r : out) {
    const auto p0 = reinterpret_cast<uintptr_t>(a.positions), o0 = reinterpret_cast<uintptr_t>(r.ptr);
    if (p0 < o0 + r.bytes && o0 < p0 + 4 * a.tokens * axes) return bad(std::string(r.name) + " overlaps input positions");
  }
  return T2V_OK;
}

// Tokens of a workgroup: the fewest with kLeast rows of which a quarter at most is missing in the last round of the groups of lanes, as long as
// there are two workgroups a CU, and no more than the table of angles holds.
int tokens_per_block(int64_t tokens, int heads, int head_dim) {
  const int groups = kThreads * kElems / head_dim, least = kLeastRows128 * 128 * 128 / (head_dim * head_dim);
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(tokens / 512, 2 * kMaxAngles / head_dim));
  for (int per = 1; per < most; ++per) {
    const int rows = per * heads, rounds = (rows + groups - 1) / groups * groups;
    if (rows >= least && 4 * rows >= 3 * rounds) return per;
  }
  return static_cast<int>(most);
}

// What the caches need not keep, by the bytes that a call writes (it reads as many) against the 256 MB that lie before the memory. Where both fit:
// nothing (14,750 tokens, 75 MB: 36 us, 38 to 39 with either hint on reads). Where only the outputs fit: the inputs, so that the outputs wait there for the
// attention (20,280 tokens, 24 + 8 heads, 166 MB: 57 us against 64; stored in pages, 210 MB: 77 against 90; with the outputs marked too
// 84, or 81 for 90 where no call writes the memory of another). Else both
// (116,904 tokens, 1.4 GB: 476 us against 492).
void set_once(NormArgs* a, int64_t out_bytes) {
  constexpr int64_t kCache = 256 << 20;
  a->read_once = 2 * out_bytes > kCache;
  a->write_once = out_bytes > kCache;
}

int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? T2V_OK : set_error(T2V_ERR_HIP, std::string(what) + " launch: " + hipGetErrorString(e));
}

int norm_rotary_impl(const void* q, const void* k, int64_t q_stride, int64_t k_stride, int64_t tokens, int heads, int kv_heads,
                     int head_dim, const t2v_turn* turn, void* q_out, void* k_out, void* stream) {
  if (int st = check_heads(tokens, heads, kv_heads, head_dim)) return st;
  NormArgs a{};
  bool interleaved = false;
  int axes = 0;
  std::vector<Range> in, out;
  if (int st = check_turn(turn, head_dim, heads, kv_heads, &a, &interleaved, &axes, &in)) return st;
  if (tokens == 0) return T2V_OK;
  const struct {
    const void* in;
    void* out;
    int64_t stride;
    int heads;
    const char *name, *out_name, *stride_name;
  } t[2] = {{q, q_out, q_stride, heads, "q", "q_out", "q_stride"}, {k, k_out, k_stride, kv_heads, "k", "k_out", "k_stride"}};
  for (int i = 0; i < 2; ++i) {
    a.heads[i] = t[i].heads;
    if (t[i].heads == 0) continue;
    if (int st = check_stride(t[i].stride, t[i].heads, head_dim, t[i].stride_name)) return st;
    in.push_back({t[i].in, rows_bytes(tokens, t[i].stride, t[i].heads, head_dim), t[i].name});
    out.push_back({t[i].out, 2 * tokens * t[i].heads * head_dim, t[i].out_name});
    a.in[i] = static_cast<const bf16*>(t[i].in);
    a.out[i] = static_cast<bf16*>(t[i].out);
    a.stride[i] = t[i].stride;
  }
  a.positions = turn->positions;
  a.tokens = tokens;
  if (int st = check_pointers(a, axes, in, out)) return st;
  set_once(&a, 2 * tokens * (heads + static_cast<int64_t>(kv_heads)) * head_dim);
  const int per = tokens_per_block(tokens, heads + kv_heads, head_dim);
  const int64_t blocks = (tokens + per - 1) / per;
  if (blocks * kThreads > UINT32_MAX)  // a launch counts its threads in 32 bits
    return bad("the call takes " + std::to_string(blocks) + " workgroups of " + std::to_string(per) + " tokens, more than one launch holds");
  with_form(a, head_dim, interleaved, [&](auto d, auto il, auto lds) {
    hipLaunchKernelGGL((norm_rotary_kernel<decltype(d)::value, decltype(il)::value, decltype(lds)::value>), dim3(static_cast<int>(blocks)),
                       dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, per);
  });
  return launched("norm and rotary kernel");
}

int norm_rotary_bwd_impl(const void* q, const void* k, int64_t q_stride, int64_t k_stride, const void* dq_out, const void* dk_out,
                         int64_t dq_out_stride, int64_t dk_out_stride, int64_t tokens, int heads, int kv_heads, int head_dim,
                         const t2v_turn* turn, void* dq, void* dk, void* dq_weight, void* dk_weight, void* ws,
                         uint64_t ws_bytes, uint64_t* need, void* stream) {
  if (need != nullptr) *need = 0;
  if (int st = check_heads(tokens, heads, kv_heads, head_dim)) return st;
  NormArgs a{};
  bool interleaved = false;
  int axes = 0;
  std::vector<Range> in, out;
  if (int st = check_turn(turn, head_dim, heads, kv_heads, &a, &interleaved, &axes, &in)) return st;
  if (!a.norm) return bad("the backward pass needs a norm (eps >= 0); a turn alone is t2v_rotary's inverse");
  const struct {
    const void *in, *grad;
    void *out, *dweight;
    int64_t stride, grad_stride;
    int heads;
    const char *name, *grad_name, *out_name, *dweight_name, *stride_name, *grad_stride_name;
  } t[2] = {{q, dq_out, dq, dq_weight, q_stride, dq_out_stride, heads, "q", "dq_out", "dq", "dq_weight", "q_stride", "dq_out_stride"},
            {k, dk_out, dk, dk_weight, k_stride, dk_out_stride, kv_heads, "k", "dk_out", "dk", "dk_weight", "k_stride", "dk_out_stride"}};
  bool weights = false;
  for (int i = 0; i < 2; ++i) {
    a.heads[i] = t[i].heads;
    if (t[i].dweight != nullptr) {
      if ((i == 0 ? turn->q_weight : turn->k_weight) == nullptr) return bad(std::string(t[i].dweight_name) + " is given without its weight");
      a.dweight[i] = t[i].dweight;
      out.push_back({t[i].dweight, head_dim * (a.weights_f32 ? 4 : 2), t[i].dweight_name});
      weights = true;
    }
    if (tokens == 0 || t[i].heads == 0) continue;
    if (int st = check_stride(t[i].stride, t[i].heads, head_dim, t[i].stride_name)) return st;
    if (int st = check_stride(t[i].grad_stride, t[i].heads, head_dim, t[i].grad_stride_name)) return st;
    in.push_back({t[i].in, rows_bytes(tokens, t[i].stride, t[i].heads, head_dim), t[i].name});
    in.push_back({t[i].grad, rows_bytes(tokens, t[i].grad_stride, t[i].heads, head_dim), t[i].grad_name});
    out.push_back({t[i].out, 2 * tokens * t[i].heads * head_dim, t[i].out_name});
    a.in[i] = static_cast<const bf16*>(t[i].in);
    a.grad[i] = static_cast<const bf16*>(t[i].grad);
    a.out[i] = static_cast<bf16*>(t[i].out);
    a.stride[i] = t[i].stride;
    a.grad_stride[i] = t[i].grad_stride;
  }
  if (tokens == 0 && !weights) return T2V_OK;
  if (ws_bytes > 0) out.push_back({ws, static_cast<int64_t>(ws_bytes), "ws"});
  a.positions = turn->positions;
  a.tokens = tokens;
  if (int st = check_pointers(a, tokens > 0 ? axes : 0, in, out)) return st;
  // At most 512 workgroups (measured: at the top), and fewer, 256 and more, for each to get rows enough to have two in flight in every lane.
  const int64_t rows = kRowsBack * (kThreads * kElems / head_dim), least = (rows + heads + kv_heads - 1) / (heads + kv_heads);
  const int64_t each = std::max<int64_t>((tokens + kMaxBackBlocks - 1) / kMaxBackBlocks, std::min<int64_t>(least, (tokens + 255) / 256));
  const int blocks = tokens == 0 ? 0 : static_cast<int>((tokens + each - 1) / each);
  // One chunk, if the table holds it; else short ones in turn, so that the workgroups go through memory side by side: 116,904 tokens of 24 + 24 heads 819 us, each
  // through a part of its own 872; 60,000 of 30 + 10 heads of 64 182 and 194. (Chunks of 32: 855 and 191, of 5: 799 and 209.)
  const int chunk = each <= 2 * kMaxAngles / head_dim ? static_cast<int>(each) : kChunkBack;
  const uint64_t bytes = weights ? static_cast<uint64_t>(blocks) * 2 * head_dim * sizeof(float) : 0;
  if (need != nullptr) *need = bytes;
  if (ws_bytes < bytes)
    return set_error(T2V_ERR_WORKSPACE, "the call needs " + std::to_string(bytes) + " bytes of workspace, got " + std::to_string(ws_bytes));
  if (weights) a.partial = static_cast<float*>(ws);
  const auto s = static_cast<hipStream_t>(stream);
  if (blocks > 0) {
    with_form(a, head_dim, interleaved, [&](auto d, auto il, auto lds) {
      hipLaunchKernelGGL((norm_rotary_bwd_kernel<decltype(d)::value, decltype(il)::value, decltype(lds)::value>), dim3(blocks),
                         dim3(kThreads), 0, s, a, chunk);
    });
    if (int st = launched("norm and rotary backward kernel")) return st;
  }
  if (!weights) return T2V_OK;
  if (head_dim == 128)
    hipLaunchKernelGGL((norm_weights_kernel<128>), dim3(256), dim3(kThreads), 0, s, a.partial, blocks, a.weights_f32, a.dweight[0], a.dweight[1]);
  else
    hipLaunchKernelGGL((norm_weights_kernel<64>), dim3(128), dim3(kThreads), 0, s, a.partial, blocks, a.weights_f32, a.dweight[0], a.dweight[1]);
  return launched("norm weights kernel");
}

int paged_append_impl(const void* k, const void* v, int64_t k_stride, int64_t v_stride, const void* q, int64_t q_stride, int heads,
                      const int32_t* cu_seqlens, int64_t tokens, const t2v_pages* cache, const t2v_turn* turn, void* q_out,
                      void* stream) {
  if (int st = check_pages(cache)) return st;
  const t2v_pages& g = *cache;
  if (heads < 0) return bad("heads must be >= 0");
  if (int st = check_heads(tokens, heads, 2 * g.kv_heads, g.head_dim)) return st;
  AppendArgs p{};
  NormArgs& a = p.n;
  bool interleaved = false;
  int axes = 0;
  std::vector<Range> in, out;
  if (turn != nullptr) {
    if (int st = check_turn(turn, g.head_dim, heads, g.kv_heads, &a, &interleaved, &axes, &in)) return st;
    a.positions = turn->positions;
  } else if (heads > 0) {
    return bad("q is given without a norm or a turn");
  }
  if (int st = check_stride(k_stride, g.kv_heads, g.head_dim, "k_stride")) return st;
  if (int st = check_stride(v_stride, g.kv_heads, g.head_dim, "v_stride")) return st;
  if (int st = check_stride(q_stride, heads, g.head_dim, "q_stride")) return st;
  if (tokens == 0 || g.nseq == 0) return T2V_OK;
  a.tokens = tokens;
  in.push_back({k, rows_bytes(tokens, k_stride, g.kv_heads, g.head_dim), "k"});
  in.push_back({v, rows_bytes(tokens, v_stride, g.kv_heads, g.head_dim), "v"});
  if (heads > 0) {
    in.push_back({q, rows_bytes(tokens, q_stride, heads, g.head_dim), "q"});
    out.push_back({q_out, 2 * tokens * heads * g.head_dim, "q_out"});
  }
  if (g.pages > 0 && g.k == g.v) return bad("cache.k and cache.v are the same memory");
  // K's and V's pages may lie between each other, so each is checked against the other tensors.
  for (int i = 0; i < 2; ++i) {
    std::vector<Range> o = out;
    if (g.pages > 0)
      o.push_back({i ? g.v : g.k, i ? pages_bytes(g, g.v_strides) : pages_bytes(g, g.k_strides), i ? "cache.v" : "cache.k"});
    if (int st = check_pointers(a, axes, in, o)) return st;
    if (int st = check_tables_apart(g, cu_seqlens, o)) return st;
  }
  a.in[0] = static_cast<const bf16*>(q);
  a.in[1] = static_cast<const bf16*>(k);
  a.out[0] = static_cast<bf16*>(q_out);
  a.stride[0] = q_stride;
  a.stride[1] = k_stride;
  a.heads[0] = heads;
  a.heads[1] = g.kv_heads;
  p.v = static_cast<const bf16*>(v);
  p.v_stride = v_stride;
  p.k_pages = static_cast<bf16*>(g.k);
  p.v_pages = static_cast<bf16*>(g.v);
  p.k_page = g.k_strides[0];
  p.k_token = g.k_strides[1];
  p.k_head = g.k_strides[2];
  p.v_page = g.v_strides[0];
  p.v_token = g.v_strides[1];
  p.v_head = g.v_strides[2];
  p.cu = cu_seqlens;
  p.lengths = g.lengths;
  p.table = g.table;
  p.table_stride = g.table_stride;
  p.nseq = g.nseq;
  p.pages = static_cast<int>(g.pages);
  p.shift = __builtin_ctz(g.page_size);
  p.room = g.width * g.page_size;
  set_once(&a, 2 * tokens * (heads + 2 * static_cast<int64_t>(g.kv_heads)) * g.head_dim);
  const int per = tokens_per_block(tokens, heads + 2 * g.kv_heads, g.head_dim);
  const int64_t blocks = (tokens + per - 1) / per;
  if (blocks * kThreads > UINT32_MAX)
    return bad("the call takes " + std::to_string(blocks) + " workgroups of " + std::to_string(per) + " tokens, more than one launch holds");
  with_form(a, g.head_dim, interleaved, [&](auto d, auto il, auto lds) {
    hipLaunchKernelGGL((paged_append_kernel<decltype(d)::value, decltype(il)::value, decltype(lds)::value>), dim3(static_cast<int>(blocks)),
                       dim3(kThreads), 0, static_cast<hipStream_t>(stream), p, per);
  });
  return launched("paged append kernel");
}

}  // namespace
}  // namespace t2v

extern "C" int t2v_norm_rotary(const void* q, const void* k, int64_t q_stride, int64_t k_stride, int64_t tokens, int heads,
                               int kv_heads, int head_dim, const t2v_turn* turn, void* q_out, void* k_out, void* stream) {
  try {
    return t2v::norm_rotary_impl(q, k, q_stride, k_stride, tokens, heads, kv_heads, head_dim, turn, q_out, k_out, stream);
  } catch (...) {
    return t2v::set_error(T2V_ERR_OOM, "host allocation failed");
  }
}

extern "C" int t2v_norm_rotary_bwd(const void* q, const void* k, int64_t q_stride, int64_t k_stride, const void* dq_out,
                                   const void* dk_out, int64_t dq_out_stride, int64_t dk_out_stride, int64_t tokens, int heads,
                                   int kv_heads, int head_dim, const t2v_turn* turn, void* dq, void* dk, void* dq_weight,
                                   void* dk_weight, void* ws, uint64_t ws_bytes, uint64_t* need, void* stream) {
  try {
    return t2v::norm_rotary_bwd_impl(q, k, q_stride, k_stride, dq_out, dk_out, dq_out_stride, dk_out_stride, tokens, heads, kv_heads,
                                     head_dim, turn, dq, dk, dq_weight, dk_weight, ws, ws_bytes, need, stream);
  } catch (...) {
    return t2v::set_error(T2V_ERR_OOM, "host allocation failed");
  }
}

extern "C" int t2v_paged_append(const void* k, const void* v, int64_t k_stride, int64_t v_stride, const void* q, int64_t q_stride,
                                int heads, const int32_t* cu_seqlens, int64_t tokens, const t2v_pages* cache, const t2v_turn* turn,
                                void* q_out, void* stream) {
  try {
    return t2v::paged_append_impl(k, v, k_stride, v_stride, q, q_stride, heads, cu_seqlens, tokens, cache, turn, q_out, stream);
  } catch (...) {
    return t2v::set_error(T2V_ERR_OOM, "host allocation failed");
  }
}
