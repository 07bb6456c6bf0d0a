// Host side of the score transforms: a caller's sift_score checked, and its
// constants made.  Not part of the ABI.
#pragma once

#include <cmath>

#include "sift_internal.h"
#include "sift_serve.h"

namespace sift {

constexpr double kUnitLog2e = 1.4426950408889634;

// score == nullptr: the default scale alone.  unit: see ScoreArgs.
inline sift_status make_score(const sift_score* score, int32_t head_dim, double unit,
                              ScoreArgs* out) {
  const sift_score s = score != nullptr ? *score : sift_score{0.f, 0.f, nullptr};
  if (!(s.cap >= 0.f) || s.cap > kMaxCap) return SIFT_E_UNSUPPORTED;
  const double scale = s.softmax_scale > 0.f && std::isfinite(s.softmax_scale)
                           ? static_cast<double>(s.softmax_scale)
                           : 1.0 / std::sqrt(static_cast<double>(head_dim));
  out->c = static_cast<float>(scale * unit);
  out->x = 0.f;
  out->cap2 = 0.f;
  for (float& a : out->a) a = 0.f;
  for (float& b : out->b) b = 0.f;
  out->slopes = s.slopes;
  if (!std::isfinite(out->c)) return SIFT_E_UNSUPPORTED;
  if (s.cap == 0.f) return SIFT_OK;
  const double x = scale / static_cast<double>(s.cap);
  out->x = static_cast<float>(x);
  out->cap2 = static_cast<float>(s.cap * unit);
  double power = scale * unit;  // unit scale (scale / cap)^2i
  for (int i = 0; i < 5; ++i, power *= x * x) {
    out->a[i] = static_cast<float>(kTanhPoly[i] * power);
    if (i < 4) out->b[i] = static_cast<float>(kTanhPolyBf16[i] * power);
  }
  // a factor that fp32 does not hold, or holds as a denormal, would be a cap of another value
  if (!std::isnormal(out->x) || !std::isnormal(out->cap2)) return SIFT_E_UNSUPPORTED;
  // and an infinite coefficient makes a score of 0 none at all
  for (float a : out->a)
    if (!std::isfinite(a)) return SIFT_E_UNSUPPORTED;
  for (float b : out->b)
    if (!std::isfinite(b)) return SIFT_E_UNSUPPORTED;
  return SIFT_OK;
}

}  // namespace sift
