// Rotary positions, host side: the angle per position of every pair of channels.  See include/libra.h.
#include <cmath>
#include <cstring>

#include "libra.h"

namespace {

// What the scaling does to the plain angles theta_i = base^(-2 i / R); long double (64 bits of mantissa), so that the
// fixed-point turns below are right to a unit or two of 2^-64 times the number of turns per position.
long double scaled_angle(long double theta, int i, int rotary_dim, long double base, const libra_rope_scaling_t& s) {
  const long double two_pi = 6.283185307179586476925286766559005768L;
  switch (s.kind) {
    case LIBRA_ROPE_SCALE_LINEAR: return theta / s.factor;
    case LIBRA_ROPE_SCALE_BANDS: {
      const long double turns = s.original_len * theta / two_pi;   // turns within the length that was trained on
      long double keep = (turns - s.low) / (static_cast<long double>(s.high) - s.low);
      keep = keep < 0 ? 0 : (keep > 1 ? 1 : keep);
      return theta * keep + theta / s.factor * (1 - keep);
    }
    case LIBRA_ROPE_SCALE_RAMP: {
      // the pair (a real number) that makes `turns` turns within original_len tokens
      const long double ln_base = std::log(base);
      auto pair_of = [&](long double turns) {
        return rotary_dim * std::log(s.original_len / (turns * two_pi)) / (2 * ln_base);
      };
      long double lo = std::floor(pair_of(s.high)), hi = std::ceil(pair_of(s.low));
      if (lo < 0) lo = 0;
      if (hi > rotary_dim - 1) hi = rotary_dim - 1;
      const long double width = (hi - lo > 0.001L) ? hi - lo : 0.001L;
      long double gone = (i - lo) / width;
      gone = gone < 0 ? 0 : (gone > 1 ? 1 : gone);
      return theta * (1 - gone) + theta / s.factor * gone;
    }
    default: return theta;
  }
}

}  // namespace

extern "C" int libra_rope_init(libra_rope_t* rope, int32_t rotary_dim, int32_t layout, double base,
                               const libra_rope_scaling_t* scaling) {
  if (!rope || rotary_dim < 2 || rotary_dim % 2 != 0) return LIBRA_INVALID_ARGUMENT;
  if (layout != LIBRA_ROPE_HALF && layout != LIBRA_ROPE_INTERLEAVED) return LIBRA_INVALID_ARGUMENT;
  if (!(base > 0.0) || !std::isfinite(base)) return LIBRA_INVALID_ARGUMENT;
  if (rotary_dim > 2 * LIBRA_ROPE_MAX_PAIRS) return LIBRA_UNSUPPORTED_SHAPE;
  libra_rope_scaling_t s = {};
  s.kind = LIBRA_ROPE_SCALE_NONE;
  if (scaling) s = *scaling;
  if (s.kind < LIBRA_ROPE_SCALE_NONE || s.kind > LIBRA_ROPE_SCALE_RAMP) return LIBRA_INVALID_ARGUMENT;
  if (!(s.magnitude >= 0.0) || !std::isfinite(s.magnitude)) return LIBRA_INVALID_ARGUMENT;
  if (s.kind != LIBRA_ROPE_SCALE_NONE && (!(s.factor >= 1.0) || !std::isfinite(s.factor))) return LIBRA_INVALID_ARGUMENT;
  if (s.kind == LIBRA_ROPE_SCALE_BASE && rotary_dim == 2) return LIBRA_INVALID_ARGUMENT;   // R / (R - 2)
  if (s.kind == LIBRA_ROPE_SCALE_BANDS || s.kind == LIBRA_ROPE_SCALE_RAMP) {
    if (s.original_len <= 0 || !(s.low > 0.0) || !(s.high > s.low) || !std::isfinite(s.high)) return LIBRA_INVALID_ARGUMENT;
    if (s.kind == LIBRA_ROPE_SCALE_RAMP && !(base > 1.0)) return LIBRA_INVALID_ARGUMENT;   // divides by ln base
  }

  long double b = base;
  if (s.kind == LIBRA_ROPE_SCALE_BASE) {
    b *= std::pow(static_cast<long double>(s.factor), static_cast<long double>(rotary_dim) / (rotary_dim - 2));
  }
  libra_rope_t r;
  std::memset(&r, 0, sizeof(r));
  r.rotary_dim = rotary_dim;
  r.layout = layout;
  r.magnitude = float(s.magnitude > 0.0 ? s.magnitude
                                        : (s.kind == LIBRA_ROPE_SCALE_RAMP ? 0.1 * std::log(s.factor) + 1.0 : 1.0));
  if (!std::isnormal(r.magnitude)) return LIBRA_INVALID_ARGUMENT;   // beyond float32, or flushed to zero by the kernels
  for (int i = 0; i < rotary_dim / 2; ++i) {
    const long double theta =
        scaled_angle(std::pow(b, -2.0L * i / rotary_dim), i, rotary_dim, static_cast<long double>(base), s);
    long double turns = theta / 6.283185307179586476925286766559005768L;
    if (!std::isfinite(turns)) return LIBRA_INVALID_ARGUMENT;
    turns -= std::floor(turns);   // whole turns per position change nothing
    const long double fixed = std::floor(turns * 18446744073709551616.0L + 0.5L);
    r.turns[i] = fixed >= 18446744073709551616.0L ? 0 : uint64_t(fixed);
  }
  *rope = r;
  return LIBRA_OK;
}
