// Host side of the rotary positions: a caller's sift_rotary checked.  Not part of the
// ABI.
#pragma once

#include <cmath>

#include "sift_internal.h"
#include "sift_serve.h"

namespace sift {

inline sift_status make_rotary(const sift_rotary* r, int32_t head_dim, RotaryArgs* out) {
  if (r->rot_dim < 2 || r->rot_dim % 2 != 0 || r->rot_dim > head_dim) return SIFT_E_SHAPE;
  if (r->inv_freq == nullptr) return SIFT_E_NULL;
  if (!(r->magnitude > 0.f) || !std::isfinite(r->magnitude)) return SIFT_E_UNSUPPORTED;
  *out = RotaryArgs{r->inv_freq, r->rot_dim / 2, r->interleaved != 0, 0, r->magnitude};
  return SIFT_OK;
}

}  // namespace sift
