// The factor by which gradients are scaled down to a largest norm, formed on the device from the squared norms that the
// ranks have found, so that no host waits for the norm.
#pragma once

#include "device_util.h"
#include "kernels.h"

namespace hanayo {
namespace k {

struct ClipScale {
  float norm;    // before clipping
  // The factor, scale * 2^exponent: max_norm / norm where the norm is larger, else 1; 1 where the norm is not finite.  The exponent is 0
  // unless the factor lies below fp32's normal numbers (norms beyond 8.5e37 max_norm), where it would keep few bits or none, while a
  // gradient that is large enough for such a norm times the factor is an ordinary number: there scale is in [1/2, 1].
  float scale;
  int exponent;
  bool finite;
  __device__ __forceinline__ bool one() const { return scale == 1.f && exponent == 0; }
  __device__ __forceinline__ float operator()(float g) const { return ldexpf(g * scale, exponent); }
};

// Every thread of every workgroup does the same few steps, in 64 bits, on the same numbers: parts are added in order.
__device__ __forceinline__ ClipScale clip_scale(const ClipArgs& c) {
  double sum = 0.0;
  for (int i = 0; i < c.parts; ++i) sum += c.sumsq[i];
  const double norm = sqrt(sum);
  ClipScale s;
  s.norm = (float)norm;
  s.finite = norm < (double)INFINITY;  // neither infinite nor NaN
  double k = s.finite && norm > (double)c.max_norm ? (double)c.max_norm / norm : 1.0;
  s.exponent = 0;
  if (k < 0x1p-126) k = frexp(k, &s.exponent);
  s.scale = (float)k;
  return s;
}

}  // namespace k
}  // namespace hanayo
