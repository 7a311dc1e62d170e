// E4M3FN codes of fp32 values over a scale, as the cache writes and the
// dense operators make them.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace gambit {

// x / s rounded to fp32, r = 1 / s rounded: a product with the reciprocal and
// one correction by the exact remainder is the rounded quotient (Markstein's
// theorem).  Quotients beyond E4M3FN's range saturate whatever their last bits,
// and so small ones that the remainder underflows have code zero.  (The
// caller keeps the reciprocal inside fp32.)
__device__ inline float quotient(float x, float s, float r) {
  const float q = x * r, e = fmaf(-q, s, x);
  return fabsf(q) < 512.f ? fmaf(e, r, q) : q;
}

// Nearest E4M3FN codes of four quotients (ties to even; beyond 448 saturating;
// NaN stays), one byte each.
__device__ inline uint32_t fp8_codes(float a, float b, float c, float d) {
  const float y[4] = {a, b, c, d};
  float z[4];
  uint32_t nan = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    z[i] = __builtin_amdgcn_fmed3f(y[i], -448.f, 448.f);
    nan |= y[i] != y[i] ? 0xffu << (8 * i) : 0u;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], w, true);
  return ((uint32_t)w & ~nan) | (0x7f7f7f7fu & nan);
}

// Sixteen bytes that no one reads again (the loads' non-temporal hint).
__device__ inline uint4 load_once(const void* p) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 a = __builtin_nontemporal_load(static_cast<const u32x4*>(p));
  return make_uint4(a[0], a[1], a[2], a[3]);
}

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

}  // namespace gambit
