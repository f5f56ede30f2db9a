// The factor by which gradients are scaled down to a largest norm, formed on the device from the squared norms that the
// ranks have found, so that no host waits for the norm.
#pragma once

#include "device_util.h"
#include "kernels.h"

namespace hanayo {
namespace k {

struct ClipScale {
  float norm;   // before clipping
  float scale;  // max_norm / norm where the norm is larger, else 1; 1 where the norm is not finite
  bool finite;
};

// Every thread of every workgroup does the same few steps, in 64 bits, on the same numbers: parts are added in order.
__device__ __forceinline__ ClipScale clip_scale(const ClipArgs& c) {
  double sum = 0.0;
  for (int i = 0; i < c.parts; ++i) sum += c.sumsq[i];
  const double norm = sqrt(sum);
  ClipScale s;
  s.norm = (float)norm;
  s.finite = norm < (double)INFINITY;  // neither infinite nor NaN
  s.scale = s.finite && norm > (double)c.max_norm ? (float)((double)c.max_norm / norm) : 1.f;
  return s;
}

}  // namespace k
}  // namespace hanayo
