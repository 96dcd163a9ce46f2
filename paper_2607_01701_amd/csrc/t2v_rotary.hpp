// What the kernels that turn heads by positions share: angles as 64-bit fractions of a turn, and the checks
// of frequencies and sections.
//
// A frequency is held as F = f / 2 pi mod 1 in units of 2^-64, so that position * F modulo 2^64 is the angle's fraction of a
// turn, exact to position * 2^-65 turns at any int32 position: no large angle is ever formed or reduced. Its top 24 bits and
// sign go to 32-bit sine and cosine.
#pragma once

#include <cmath>

#include "../../include/t2vattn.h"
#include "t2v_device.hpp"
#include "t2v_host.h"

namespace t2v {

constexpr int kMaxPairs = 64;
constexpr int kMaxAxes = 3;

struct RotaryAngles {
  unsigned long long turn[kMaxPairs];  // a position's angle of each pair, in 2^-64 turns
  unsigned char axis[kMaxPairs];
};

// (cos, sin) of pair j at position p.
T2V_DEV float2 angle_of(const RotaryAngles& a, int j, int p) {
  const unsigned long long turns = static_cast<unsigned long long>(static_cast<long long>(p)) * a.turn[j];
  // The fraction of a turn in [-1/2, 1/2), in half turns.
  const float half_turns = static_cast<float>(static_cast<long long>(turns)) * 0x1p-63f;
  float s, c;
  sincospif(half_turns, &s, &c);
  return make_float2(c, s);
}

// f radians in 2^-64 turns, modulo a turn. long double holds 64 bits of the quotient. (Usual frequencies are less than a turn: without floor, which takes
// 0.1 us in long double, 64 pairs take 0.5 us for 6.9.)
inline unsigned long long turn_of(double f) {
  const long double turns = static_cast<long double>(f) * 0.159154943091895335768883763372514362L;  // 1 / (2 pi)
  const long double frac = turns >= 0.0L && turns < 1.0L ? turns : turns - std::floor(turns);
  const long double scaled = frac * 18446744073709551616.0L;
  return scaled >= 18446744073709551615.0L ? ~0ull : static_cast<unsigned long long>(scaled + 0.5L);
}

// Checks frequencies, sections, layout and mscale, and counts the pairs.
inline int check_rotary(const double* freqs, const int32_t* sections, int n_sections, int layout, float mscale, int head_dim,
                        int64_t* n_pairs) {
  auto bad = [](const std::string& what) { return set_error(T2V_ERR_INVALID_ARG, what); };
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
  *n_pairs = pairs;
  return T2V_OK;
}

inline void fill_angles(RotaryAngles* a, const double* freqs, const int32_t* sections, int n_sections) {
  for (int i = 0, j = 0; i < n_sections; ++i)
    for (int n = 0; n < sections[i]; ++n, ++j) {
      a->axis[j] = static_cast<unsigned char>(i);
      a->turn[j] = turn_of(freqs[j]);
    }
}

}  // namespace t2v
