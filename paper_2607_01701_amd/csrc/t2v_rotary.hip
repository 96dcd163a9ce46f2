// Rotary positions on the heads of q and k, before attention: y = m R(p f_j) x for pair j of a head's
// first rot_dim dimensions, p the token's position on the pair's axis; the other dimensions are copied. The
// backward pass is the same call with the angles' sign turned.
//
// Bound by memory: every element is read once and written once, 16 bytes a lane. A workgroup
// takes tokens one after another; the sine and cosine of a pair are worked out once a token and shared by
// all heads through LDS.
//
// Angles. A frequency is held as a 64-bit fraction of a turn, F = f / 2 pi mod 1 in units of 2^-64, so that
// position * F modulo 2^64 is the angle's fraction of a turn, exact to position * 2^-65 turns at any int32
// position: no large angle is ever formed or reduced. Its top 24 bits and sign go to 32-bit sine and cosine.
#include <algorithm>
#include <cmath>
#include <string>
#include <vector>

#include "../../include/t2vattn.h"
#include "t2v_device.hpp"
#include "t2v_host.h"

namespace t2v {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 64;
constexpr int kMaxAxes = 3;

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
  unsigned long long turn[kMaxPairs];  // a position's angle of each pair, in 2^-64 turns
  unsigned char axis[kMaxPairs];
};

// A workgroup's tokens: kTokens of them, their sines and cosines in LDS.
template <int D, bool INTERLEAVED, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a, int tokens_per_block) {
  constexpr int C = D / 8;  // 16-byte chunks of a head
  __shared__ float2 cs[64 * kMaxPairs];
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * tokens_per_block;
  const int nt = static_cast<int>(min(static_cast<int64_t>(tokens_per_block), a.tokens - t0));
  const int pairs = a.rot_dim / 2;
  for (int e = threadIdx.x; e < nt * pairs; e += kThreads) {
    const int t = e / pairs, j = e - t * pairs;
    const int p = a.positions[a.axis[j] * a.tokens + t0 + t];
    const unsigned long long turns = static_cast<unsigned long long>(static_cast<long long>(p)) * a.turn[j];
    // The fraction of a turn in [-1/2, 1/2), in half turns.
    const float half_turns = static_cast<float>(static_cast<long long>(turns)) * 0x1p-63f;
    float s, c;
    sincospif(half_turns, &s, &c);
    cs[e] = make_float2(c * a.mscale, (a.inverse ? -s : s) * a.mscale);
  }
  __syncthreads();
  const int heads = a.heads[0] + a.heads[1];
  const int per_token = heads * C;
  for (int e = threadIdx.x; e < nt * per_token; e += kThreads) {
    const int t = e / per_token, r = e - t * per_token;
    const int h = r / C, c = r % C;
    const int which = h >= a.heads[0];
    const int hh = which ? h - a.heads[0] : h;
    const bf16* x = a.in[which] + (t0 + t) * a.stride[which] + static_cast<int64_t>(hh) * D;
    bf16* y = a.out[which] + ((t0 + t) * a.heads[which] + hh) * D;
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(x + c * 8);
    bf16x8 w = v;
    const float2* row = cs + t * pairs;
    if constexpr (INTERLEAVED) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = c * 4 + i;
        if (j < pairs) {
          const float u0 = static_cast<float>(v[2 * i]), u1 = static_cast<float>(v[2 * i + 1]);
          const float2 k = row[j];
          w[2 * i] = static_cast<bf16>(u0 * k.x - u1 * k.y);
          w[2 * i + 1] = static_cast<bf16>(u0 * k.y + u1 * k.x);
        }
      }
    } else if (c * 8 < a.rot_dim) {
      // The partner of dimension d is d + pairs or d - pairs: another chunk, read through the cache.
      bf16x8 o = v;
      if constexpr (ALIGNED) {
        o = *reinterpret_cast<const bf16x8*>(x + (c * 8 < pairs ? c * 8 + pairs : c * 8 - pairs));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int d = c * 8 + i;
          if (d < a.rot_dim) o[i] = x[d < pairs ? d + pairs : d - pairs];
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = c * 8 + i;
        if (d < a.rot_dim) {
          const float2 k = row[d < pairs ? d : d - pairs];
          const float u = static_cast<float>(v[i]), p = static_cast<float>(o[i]);
          w[i] = static_cast<bf16>(u * k.x + (d < pairs ? -p : p) * k.y);
        }
      }
    }
    *reinterpret_cast<bf16x8*>(y + c * 8) = w;
  }
}

// f radians in 2^-64 turns, modulo a turn. long double holds 64 bits of the quotient.
unsigned long long turn_of(double f) {
  const long double turns = static_cast<long double>(f) / (2.0L * 3.14159265358979323846264338327950288L);
  const long double frac = turns - std::floor(turns);
  const long double scaled = frac * 18446744073709551616.0L;
  return scaled >= 18446744073709551615.0L ? ~0ull : static_cast<unsigned long long>(scaled + 0.5L);
}

template <int D>
void launch(const RotaryArgs& a, bool interleaved, int blocks, int per, hipStream_t s) {
  if (interleaved)
    hipLaunchKernelGGL((rotary_kernel<D, true, true>), dim3(blocks), dim3(kThreads), 0, s, a, per);
  else if (a.rot_dim % 16 == 0)
    hipLaunchKernelGGL((rotary_kernel<D, false, true>), dim3(blocks), dim3(kThreads), 0, s, a, per);
  else
    hipLaunchKernelGGL((rotary_kernel<D, false, false>), dim3(blocks), dim3(kThreads), 0, s, a, per);
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
  if (freqs == nullptr || sections == nullptr) return bad("freqs or sections is NULL");
  if (n_sections < 1 || n_sections > kMaxAxes) return bad("there must be 1 to 3 sections");
  int64_t pairs = 0;
  for (int i = 0; i < n_sections; ++i) {
    if (sections[i] < 0) return bad("sections must be >= 0");
    pairs += sections[i];
  }
  if (pairs < 1 || 2 * pairs > head_dim) return bad("the sections must sum to 1 .. head_dim / 2 pairs");
  if (layout != T2V_ROTARY_HALF && layout != T2V_ROTARY_INTERLEAVED) return bad("unknown layout");
  if (!std::isfinite(mscale)) return bad("mscale must be finite");
  for (int64_t j = 0; j < pairs; ++j)
    if (!std::isfinite(freqs[j])) return bad("freqs must be finite");
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
  for (int i = 0, j = 0; i < n_sections; ++i)
    for (int n = 0; n < sections[i]; ++n, ++j) {
      a.axis[j] = static_cast<unsigned char>(i);
      a.turn[j] = turn_of(freqs[j]);
    }
  const int per = 1;
  const int blocks = static_cast<int>((tokens + per - 1) / per);
  const auto s = static_cast<hipStream_t>(stream);
  const bool interleaved = layout == T2V_ROTARY_INTERLEAVED;
  head_dim == 128 ? launch<128>(a, interleaved, blocks, per, s) : launch<64>(a, interleaved, blocks, per, s);
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
