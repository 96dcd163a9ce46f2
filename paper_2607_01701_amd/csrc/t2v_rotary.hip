// Rotary positions on the heads of q and k, before attention: y = m R(p f_j) x for pair j of a head's
// first rot_dim dimensions, p the token's position on the pair's axis; the other dimensions are copied. The
// backward pass is the same call with the angles' sign turned.
//
// Bound by memory: every element is read once and written once, at 5.4 TB/s (116,904 tokens of 24 + 24 heads of 128: 502 us; 20,280
// tokens of 24 + 8 heads, 64 dimensions turned: 66 us), 4.8 where vectors are unaligned (36 of 64 dimensions turned, 14,750 tokens
// of 30 + 10 heads: 29 us). Single tokens take a launch. Work is cut into units of 16
// elements, two 16-byte vectors: eight pairs, or 16 dimensions that are copied. A lane has four units in flight
// and loads them before the sines and cosines, which are worked out once a token and shared by
// all heads through LDS. Counts of pairs that are no multiple of 8 take the same path: the last unit is moved
// back to overlap the one before (it writes the same values again), and vectors need not be aligned.
// Angles: t2v_rotary.hpp.
#include <algorithm>
#include <cmath>
#include <string>
#include <vector>

#include "../../include/t2vattn.h"
#include "t2v_device.hpp"
#include "t2v_host.h"
#include "t2v_rotary.hpp"

namespace t2v {
namespace {

constexpr int kThreads = 256;
constexpr int kUnits = 4;  // in flight per lane
constexpr int kMaxAngles = 2048;  // of a workgroup (16 KB of LDS: eight workgroups on a CU)

struct RotaryArgs {
  const bf16* in[2];   // q, k
  bf16* out[2];
  int64_t stride[2];   // elements between tokens of q and k; outputs are contiguous
  int heads[2];
  const int32_t* positions;  // [axes, tokens]
  int64_t tokens;
  int rot_dim;
  float mscale;
  int inverse;
  RotaryAngles angles;
};

// Eight bf16 at any 2-byte address (a global access of 16 bytes needs no alignment).
typedef __attribute__((address_space(1))) bf16 gbf16;  // in global memory
typedef __attribute__((address_space(1))) uint32_t gu32;
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef __attribute__((address_space(1))) u32x4_any gu32x4_any;
T2V_DEV bf16x8 load_any(const gbf16* p) { return __builtin_bit_cast(bf16x8, *(const gu32x4_any*)(p)); }
T2V_DEV void store_any(gbf16* p, const bf16x8& x) { *(gu32x4_any*)(p) = __builtin_bit_cast(u32x4, x); }

// Where a lane is: unit `u` of head `h` (q's heads, then k's) of the workgroup's token `t`.
struct Place {
  int t, h, u;
};

template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a, int tokens_per_block) {
  __shared__ __attribute__((aligned(16))) float2 cs[kMaxAngles];
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * tokens_per_block;
  const int nt = static_cast<int>(min(static_cast<int64_t>(tokens_per_block), a.tokens - t0));
  const int pairs = a.rot_dim / 2;
  const int turned = (pairs + 7) / 8, units = turned + (D - a.rot_dim + 15) / 16;  // of a head
  const int heads = a.heads[0] + a.heads[1];
  const int total = nt * heads * units;
  // A lane's units are kThreads apart: its place moves by (st, sh, su), with carries.
  const int su = kThreads % units, sr = kThreads / units, st = sr / heads, sh = sr - st * heads;
  Place w;
  {
    const int e = threadIdx.x, r = e / units;
    w.u = e - r * units;
    w.t = r / heads;
    w.h = r - w.t * heads;
  }
  auto advance = [&](Place& x) {
    x.u += su;
    int c = x.u >= units;
    x.u -= c ? units : 0;
    x.h += sh + c;
    c = x.h >= heads;
    x.h -= c ? heads : 0;
    x.t += st + c;
  };
  // First elements of the unit's two vectors within the head, and its first pair (-1: copied).
  struct Vectors {
    int first, second, pair;
  };
  auto vectors = [&](int u) -> Vectors {
    if (u < turned) {
      const int j = max(min(8 * u, pairs - 8), 0);
      return INTERLEAVED ? Vectors{2 * j, 2 * j + 8, j} : Vectors{j, j + pairs, j};
    }
    const int d = min(a.rot_dim + 16 * (u - turned), D - 16);
    return {d, d + 8, -1};
  };
  // A lane's tensor is picked from scalar registers: a choice between two arguments would become a
  // load from the argument block at an address of the lane's.
  const int hq = a.heads[0];
  const gbf16 *q = (const gbf16*)(a.in[0]), *k = (const gbf16*)(a.in[1]);
  gbf16 *qo = (gbf16*)(a.out[0]), *ko = (gbf16*)(a.out[1]);
  int64_t qs = a.stride[0], ks = a.stride[1];
  asm volatile("" : "+s"(q), "+s"(k), "+s"(qo), "+s"(ko), "+s"(qs), "+s"(ks));
  auto source = [&](const Place& x) {
    const bool second = x.h >= hq;
    return (second ? k : q) + (t0 + x.t) * (second ? ks : qs) + static_cast<int64_t>(x.h - (second ? hq : 0)) * D;
  };
  auto target = [&](const Place& x) {
    const bool second = x.h >= hq;
    return (second ? ko : qo) + ((t0 + x.t) * (second ? heads - hq : hq) + (x.h - (second ? hq : 0))) * D;
  };
  // With fewer than eight pairs, or 1 .. 15 dimensions to copy, those are taken one by one.
  const bool few_pairs = pairs < 8, few_copied = D - a.rot_dim < 16;
  auto whole = [&](int u) { return u < turned ? !few_pairs : !few_copied; };

  bf16x8 x[kUnits], y[kUnits];
  auto load = [&](Place p, int e0) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      if (e0 + i * kThreads < total && whole(p.u)) {
        const Vectors v = vectors(p.u);
        const gbf16* s = source(p);
        x[i] = load_any(s + v.first);
        y[i] = load_any(s + v.second);
      }
      advance(p);
    }
  };
  load(w, threadIdx.x);
  for (int e = threadIdx.x; e < nt * pairs; e += kThreads) {
    const int t = e / pairs, j = e - t * pairs;
    const float2 k = angle_of(a.angles, j, a.positions[a.angles.axis[j] * a.tokens + t0 + t]);
    cs[e] = make_float2(k.x * a.mscale, (a.inverse ? -k.y : k.y) * a.mscale);
  }
  __syncthreads();
  for (int e0 = threadIdx.x; e0 < total; e0 += kUnits * kThreads) {
    if (e0 != static_cast<int>(threadIdx.x)) load(w, e0);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      if (e0 + i * kThreads < total) {
        gbf16* o = target(w);
        const float2* row = cs + w.t * pairs;
        if (whole(w.u)) {
          const Vectors v = vectors(w.u);
          if (v.pair >= 0) {
            float u0[8], u1[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) {
              u0[n] = static_cast<float>(INTERLEAVED ? (n < 4 ? x[i][2 * n] : y[i][2 * n - 8]) : x[i][n]);
              u1[n] = static_cast<float>(INTERLEAVED ? (n < 4 ? x[i][2 * n + 1] : y[i][2 * n - 7]) : y[i][n]);
            }
#pragma unroll
            for (int n = 0; n < 8; ++n) {
              const float2 k = row[v.pair + n];
              const bf16 z0 = static_cast<bf16>(u0[n] * k.x - u1[n] * k.y);
              const bf16 z1 = static_cast<bf16>(u0[n] * k.y + u1[n] * k.x);
              if constexpr (!INTERLEAVED) {
                x[i][n] = z0;
                y[i][n] = z1;
              } else if (n < 4) {
                x[i][2 * n] = z0;
                x[i][2 * n + 1] = z1;
              } else {
                y[i][2 * n - 8] = z0;
                y[i][2 * n - 7] = z1;
              }
            }
          }
          store_any(o + v.first, x[i]);
          store_any(o + v.second, y[i]);
        } else {
          const gbf16* s = source(w);
          if (w.u < turned) {
            for (int j = 0; j < pairs; ++j) {
              const int d0 = INTERLEAVED ? 2 * j : j, d1 = INTERLEAVED ? 2 * j + 1 : j + pairs;
              const float u0 = static_cast<float>(s[d0]), u1 = static_cast<float>(s[d1]);
              o[d0] = static_cast<bf16>(u0 * row[j].x - u1 * row[j].y);
              o[d1] = static_cast<bf16>(u0 * row[j].y + u1 * row[j].x);
            }
          } else {  // two at a time: rot_dim is even
            for (int d = a.rot_dim; d < D; d += 2)
              *(gu32*)(o + d) = *(const gu32*)(s + d);
          }
        }
      }
      advance(w);
    }
  }
}

template <int D>
void launch(const RotaryArgs& a, bool interleaved, int blocks, int per, hipStream_t s) {
  if (interleaved)
    hipLaunchKernelGGL((rotary_kernel<D, true>), dim3(blocks), dim3(kThreads), 0, s, a, per);
  else
    hipLaunchKernelGGL((rotary_kernel<D, false>), dim3(blocks), dim3(kThreads), 0, s, a, per);
}

// Tokens of a workgroup: as many as give each lane its kUnits units, as long as there are two workgroups a CU
// (fewer tokens are spread over the CUs), and no more than the table of angles holds.
int tokens_per_block(const RotaryArgs& a, int head_dim) {
  const int pairs = a.rot_dim / 2;
  const int64_t units = static_cast<int64_t>(a.heads[0] + a.heads[1]) * ((pairs + 7) / 8 + (head_dim - a.rot_dim + 15) / 16);
  const int64_t per = std::min<int64_t>(kUnits * kThreads / units, a.tokens / 512);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(per, kMaxAngles / pairs)));
}

int rotary_impl(const void* q, const void* k, int64_t q_stride, int64_t k_stride, const int32_t* positions,
                int64_t tokens, int heads, int kv_heads, int head_dim, const double* freqs, const int32_t* sections,
                int n_sections, int layout, float mscale, int inverse, void* q_out, void* k_out, void* stream) {
  auto bad = [](const std::string& what) { return set_error(T2V_ERR_INVALID_ARG, what); };
  if (head_dim != 64 && head_dim != 128)
    return set_error(T2V_ERR_UNSUPPORTED, "head_dim must be 64 or 128, got " + std::to_string(head_dim));
  if (tokens < 0 || tokens > INT32_MAX) return bad("tokens must be in 0 .. 2^31 - 1");
  if (heads < 0 || kv_heads < 0 || heads + static_cast<int64_t>(kv_heads) < 1)
    return bad("heads and kv_heads must be >= 0, and one of them >= 1");
  if ((heads + static_cast<int64_t>(kv_heads)) * head_dim > (int64_t(1) << 22))
    return bad("heads * head_dim is too large");
  int64_t pairs = 0;
  if (int st = check_rotary(freqs, sections, n_sections, layout, mscale, head_dim, &pairs)) return st;
  if (tokens == 0) return T2V_OK;
  const struct {
    const void* in;
    void* out;
    int64_t stride;
    int heads;
    const char *name, *out_name, *stride_name;
  } t[2] = {{q, q_out, q_stride, heads, "q", "q_out", "q_stride"}, {k, k_out, k_stride, kv_heads, "k", "k_out", "k_stride"}};
  std::vector<Range> in, out;
  RotaryArgs a{};
  for (int i = 0; i < 2; ++i) {
    a.heads[i] = t[i].heads;
    if (t[i].heads == 0) continue;
    const int64_t row = static_cast<int64_t>(t[i].heads) * head_dim;
    if (t[i].stride < row || t[i].stride % 8 != 0 || t[i].stride > (int64_t(1) << 22))
      return bad(std::string(t[i].stride_name) + " must be a multiple of 8 between heads * head_dim and 2^22, got " +
                 std::to_string(t[i].stride));
    in.push_back({t[i].in, 2 * ((tokens - 1) * t[i].stride + row), t[i].name});
    out.push_back({t[i].out, 2 * tokens * row, t[i].out_name});
    a.in[i] = static_cast<const bf16*>(t[i].in);
    a.out[i] = static_cast<bf16*>(t[i].out);
    a.stride[i] = t[i].stride;
  }
  if (positions == nullptr) return bad("positions is NULL");
  if (reinterpret_cast<uintptr_t>(positions) % 4 != 0) return bad("positions is not 4-byte aligned");
  if (int st = validate_pointers(in, out)) return st;
  for (const Range& r : out) {
    const auto p0 = reinterpret_cast<uintptr_t>(positions), o0 = reinterpret_cast<uintptr_t>(r.ptr);
    if (p0 < o0 + r.bytes && o0 < p0 + 4 * tokens * n_sections)
      return bad(std::string(r.name) + " overlaps input positions");
  }
  a.positions = positions;
  a.tokens = tokens;
  a.rot_dim = static_cast<int>(2 * pairs);
  a.mscale = mscale;
  a.inverse = inverse != 0;
  fill_angles(&a.angles, freqs, sections, n_sections);
  const int per = tokens_per_block(a, head_dim);
  const int64_t blocks = (tokens + per - 1) / per;
  if (blocks * kThreads > UINT32_MAX)  // a launch counts its threads in 32 bits
    return bad("the call takes " + std::to_string(blocks) + " workgroups of " + std::to_string(per) + " tokens, more than one launch holds");
  const auto s = static_cast<hipStream_t>(stream);
  const bool interleaved = layout == T2V_ROTARY_INTERLEAVED;
  head_dim == 128 ? launch<128>(a, interleaved, static_cast<int>(blocks), per, s)
                  : launch<64>(a, interleaved, static_cast<int>(blocks), per, s);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? T2V_OK : set_error(T2V_ERR_HIP, std::string("rotary kernel launch: ") + hipGetErrorString(e));
}

}  // namespace
}  // namespace t2v

extern "C" int t2v_rotary(const void* q, const void* k, int64_t q_stride, int64_t k_stride, const int32_t* positions,
                          int64_t tokens, int heads, int kv_heads, int head_dim, const double* freqs,
                          const int32_t* sections, int n_sections, int layout, float mscale, int inverse, void* q_out,
                          void* k_out, void* stream) {
  try {
    return t2v::rotary_impl(q, k, q_stride, k_stride, positions, tokens, heads, kv_heads, head_dim, freqs, sections,
                            n_sections, layout, mscale, inverse, q_out, k_out, stream);
  } catch (...) {
    return t2v::set_error(T2V_ERR_OOM, "host allocation failed");
  }
}
