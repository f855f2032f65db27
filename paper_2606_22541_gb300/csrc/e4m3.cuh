// e4m3 quantisation shared by the kernels that make activations for the FP8
// products: one scale per 128 channels.
#pragma once

#include <cuda_fp8.h>
#include <stdint.h>

namespace asap {

// Scale of a group and what its quotients need: s = amax times the fp32
// reciprocal of 448 (1 where that is 0).  Quotients of tiny groups are taken with
// value and scale multiplied by 2^100, so that 1 / s is finite.
struct GroupScale {
  float s, up, scaled, inv;
  __device__ __forceinline__ explicit GroupScale(float amax) {
    s = amax * (1.0f / 448.0f);
    if (!(s > 0.f)) s = 1.0f;
    up = s < 0x1p-100f ? 0x1p100f : 1.0f;
    scaled = s * up;
    inv = 1.0f / scaled;
  }
  // v / s, correctly rounded (Markstein 1990: one correction of v * (1/s), whose
  // reciprocal is correctly rounded, by its residual): the quotient is the one a
  // division gives.  bf16 values over amax / 448 fall exactly between two e4m3
  // values for about one element in 500, and those must not depend on how the
  // quotient was taken.  (An infinite s gives NaN.  The residual is rounded
  // down: that of an exact zero is -0, with which a quotient of -0 keeps its sign.)
  __device__ __forceinline__ float operator()(float v) const {
    v *= up;
    const float q = v * inv;
    return fmaf(__fmaf_rd(-q, scaled, v), inv, q);
  }
};

// Four values to e4m3, nearest even, saturated; a in the low byte.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
}
__device__ __forceinline__ uint32_t e4m3x4(const GroupScale& g, float a, float b, float c, float d) {
  return e4m3x4(g(a), g(b), g(c), g(d));
}

}  // namespace asap
