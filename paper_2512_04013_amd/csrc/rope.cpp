// Rotary frequencies (host code; the kernels are in rope.hip).

#include <algorithm>
#include <cmath>

#include "aug.h"
#include "status.h"

extern "C" aug_status aug_rope_init(const aug_rope_params* p, aug_rope* out) {
  const char* who = "aug_rope_init";
  if (!p || !out) return aug::fail(AUG_ERR_INVALID, "%s: NULL pointer", who);
  if (p->rotary_dim < 16 || p->rotary_dim > 128 || p->rotary_dim % 16)
    return aug::fail(AUG_ERR_UNSUPPORTED, "%s: rotary_dim %d (supported: multiples of 16 up to 128)", who, p->rotary_dim);
  if (p->interleaved != 0 && p->interleaved != 1)
    return aug::fail(AUG_ERR_INVALID, "%s: interleaved %d (0 or 1)", who, p->interleaved);
  if (p->scaling < AUG_ROPE_NONE || p->scaling > AUG_ROPE_RAMP)
    return aug::fail(AUG_ERR_INVALID, "%s: unknown scaling %d", who, p->scaling);
  if (!(p->base > 1.0) || !std::isfinite(p->base)) return aug::fail(AUG_ERR_INVALID, "%s: base %g (above 1)", who, p->base);
  // float32 holds the magnitude, which scales cosines and sines
  if (!(std::fabs(p->magnitude) <= 1e30)) return aug::fail(AUG_ERR_INVALID, "%s: magnitude %g", who, p->magnitude);
  if (p->scaling != AUG_ROPE_NONE && !(p->factor > 0.0 && std::isfinite(p->factor)))
    return aug::fail(AUG_ERR_INVALID, "%s: factor %g (above 0)", who, p->factor);
  const bool bands = p->scaling == AUG_ROPE_BANDS, ramp = p->scaling == AUG_ROPE_RAMP;
  if ((bands || ramp) && (p->original_len < 1 || !(p->low > 0.0) || !(p->high > p->low) || !std::isfinite(p->high)))
    return aug::fail(AUG_ERR_INVALID, "%s: original_len %d, low %g, high %g (above 0, low below high)", who, p->original_len,
                     p->low, p->high);

  const double two_pi = 6.283185307179586476925286766559;
  const double dim = p->rotary_dim;
  double from = 0.0, to = 0.0;
  if (ramp) {
    const auto pair_of = [&](double turns) { return dim * std::log(p->original_len / (two_pi * turns)) / (2.0 * std::log(p->base)); };
    from = std::max(std::floor(pair_of(p->high)), 0.0);
    to = std::min(std::ceil(pair_of(p->low)), dim - 1.0);
  }
  aug_rope r{};
  r.rotary_dim = p->rotary_dim;
  r.interleaved = p->interleaved;
  r.magnitude = static_cast<float>(p->magnitude);
  for (int i = 0; i < p->rotary_dim / 2; ++i) {
    double w = std::pow(p->base, -2.0 * i / dim);
    if (p->scaling == AUG_ROPE_LINEAR) {
      w /= p->factor;
    } else if (bands) {
      const double m = std::clamp((p->original_len * w / two_pi - p->low) / (p->high - p->low), 0.0, 1.0);
      w = w * m + w / p->factor * (1.0 - m);
    } else if (ramp) {
      const double m = std::clamp((i - from) / std::max(to - from, 0.001), 0.0, 1.0);
      w = w / p->factor * m + w * (1.0 - m);
    }
    // An angle of up to 2^31 positions keeps 20 bits behind the point (float64) below
    // this; nothing real comes near it.
    if (!(w <= 1e3)) return aug::fail(AUG_ERR_INVALID, "%s: %g radians per position", who, w);
    r.turns[i] = w / two_pi;
  }
  *out = r;
  return AUG_OK;
}
