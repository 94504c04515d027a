// What the kernels that attend over pages share.
#pragma once

#include "common.h"
#include "tile_ring.h"

namespace lava {
namespace {

// cap * tanh(z / cap): near zero by its series (the quotient of exponentials would cancel), else from e^(-2 |z / cap|).
__device__ __forceinline__ float capped(float z, float cap, float inv_cap) {
  const float y = z * inv_cap, a = fabsf(y), s = y * y;
  float series = fmaf(s, 2.1869489e-2f, -5.3968254e-2f);             // 62 / 2835, -17 / 315
  series = fmaf(s, series, 1.3333333e-1f);
  series = fmaf(s, series, -3.3333333e-1f);
  series = fmaf(a * s, series, a);
  const float t = fast_exp2(a * (-2.0f * kLog2e));
  const float far = (1.0f - t) * __builtin_amdgcn_rcpf(1.0f + t);
  return cap * copysignf(a < 0.25f ? series : far, y);
}

// to * tanh(z / cap) where |z| < cap / 4: the series alone.
__device__ __forceinline__ float capped_near(float z, float to, float inv_cap) {
  const float y = z * inv_cap, s = y * y;
  float series = fmaf(s, 2.1869489e-2f, -5.3968254e-2f);
  series = fmaf(s, series, 1.3333333e-1f);
  series = fmaf(s, series, -3.3333333e-1f);
  return to * fmaf(y * s, series, y);
}

}  // namespace
}  // namespace lava
