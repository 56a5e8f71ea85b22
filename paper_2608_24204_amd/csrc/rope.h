// Angle steps of a rotary embedding (host).
#pragma once
#include <cmath>

#include "../../include/wici.h"
#include "kv8.h"

namespace wici {

// Whether the specification is one (see wici_rope).
inline bool rope_ok(const wici_rope& r) {
  if (r.dim < 8 || r.dim > 128 || r.dim % 8) return false;
  if (r.layout != WICI_ROPE_HALF && r.layout != WICI_ROPE_PAIRS) return false;
  if (!(r.base > 1.0) || !std::isfinite(r.base)) return false;
  if (r.scaling == WICI_ROPE_PLAIN) return true;
  if (r.scaling < WICI_ROPE_PLAIN || r.scaling > WICI_ROPE_RAMP) return false;
  if (!(r.factor >= 1.0) || !std::isfinite(r.factor)) return false;
  if (r.scaling != WICI_ROPE_BANDS && r.scaling != WICI_ROPE_RAMP) return true;
  if (!(r.original > 0.0) || !std::isfinite(r.original)) return false;
  return (r.low == 0.0 && r.high == 0.0) ||
         (r.low > 0.0 && r.low < r.high && std::isfinite(r.high));
}

inline RopeFreqs rope_freqs(const wici_rope& r) {
  const double tau = 6.283185307179586476925;
  const bool own = r.low != 0.0 || r.high != 0.0;
  const double low = own ? r.low : 1.0,
               high = own ? r.high : r.scaling == WICI_ROPE_BANDS ? 4.0 : 32.0;
  auto clamp01 = [](double v) { return v < 0.0 ? 0.0 : v > 1.0 ? 1.0 : v; };
  auto turns_at = [&](double t) {
    return r.dim * std::log(r.original / (t * tau)) / (2.0 * std::log(r.base));
  };
  RopeFreqs f{};
  f.factor = r.scaling == WICI_ROPE_RAMP ? 1.0 + 0.1 * std::log(r.factor) : 1.0;
  double j_lo = 0.0, j_hi = 0.0;
  if (r.scaling == WICI_ROPE_RAMP) {
    j_lo = std::fmax(std::floor(turns_at(high)), 0.0);
    j_hi = std::fmin(std::ceil(turns_at(low)), r.dim - 1.0);
  }
  for (int j = 0; j < r.dim / 2; ++j) {
    const double e = -2.0 * j / r.dim, b = std::pow(r.base, e);
    double v = b;
    if (r.scaling == WICI_ROPE_LINEAR) {
      v = b / r.factor;
    } else if (r.scaling == WICI_ROPE_BASE) {
      v = std::pow(r.base * std::pow(r.factor, r.dim / (r.dim - 2.0)), e);
    } else if (r.scaling == WICI_ROPE_BANDS) {
      const double k = clamp01((r.original * b / tau - low) / (high - low));
      v = (1.0 - k) * b / r.factor + k * b;
    } else if (r.scaling == WICI_ROPE_RAMP) {
      const double m = clamp01((j - j_lo) / std::fmax(j_hi - j_lo, 0.001));
      v = m * b / r.factor + (1.0 - m) * b;
    }
    f.f[j] = v;
  }
  return f;
}

}  // namespace wici
