// The position rotation of queries and keys: of a head's first `rot` values,
// pair i - (2i, 2i + 1), or (i, i + rot / 2) - turns by its position's angle,
//     (a, b) -> (a cos - b sin, b cos + a sin),
// with cosines and sines from a table [position][rot] (rot / 2 of each).  Eight
// pairs make a unit: unit u < rot / 16 takes cosines 8u .. 8u + 7 either way.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "fp8_codes.h"

namespace gambit {

struct Turn {
  float c[8], s[8];
};

__device__ inline Turn load_turn(const float* row, int rot, int unit) {
  const float4* c = reinterpret_cast<const float4*>(row + 8 * unit);
  const float4* s = reinterpret_cast<const float4*>(row + rot / 2 + 8 * unit);
  const float4 c0 = c[0], c1 = c[1], s0 = s[0], s1 = s[1];
  return {{c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w}};
}

__device__ inline uint32_t two_bf16(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// Where a unit's two 16-byte chunks of eight values lie in its head.
__device__ inline void unit_chunks(int unit, int rot, int pairs, int* c0, int* c1) {
  const bool halves = !pairs && unit < rot / 16;
  *c0 = halves ? unit : 2 * unit;
  *c1 = halves ? unit + rot / 16 : 2 * unit + 1;
}

// The same in fp32, y[0..7] and y[8..15]; a unit that does not turn as it is.
__device__ inline void turn_unit_f32(uint4 x0, uint4 x1, const Turn& t, int pairs, bool turns, float* y) {
  const uint32_t w0[4] = {x0.x, x0.y, x0.z, x0.w}, w1[4] = {x1.x, x1.y, x1.z, x1.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    y[2 * j] = bf16_lo(w0[j]);
    y[2 * j + 1] = bf16_hi(w0[j]);
    y[8 + 2 * j] = bf16_lo(w1[j]);
    y[8 + 2 * j + 1] = bf16_hi(w1[j]);
  }
  if (!turns) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float& a = pairs ? y[2 * j] : y[j];
    float& b = pairs ? y[2 * j + 1] : y[8 + j];
    const float p = a, q = b;
    a = p * t.c[j] - q * t.s[j];
    b = q * t.c[j] + p * t.s[j];
  }
}

// Sixteen values, a unit's two chunks, turned.  Adjacent pairs lie in one dword, the others in two chunks.
__device__ inline void turn_unit(uint4& x0, uint4& x1, const Turn& t, int pairs) {
  uint32_t* w0 = reinterpret_cast<uint32_t*>(&x0);
  uint32_t* w1 = reinterpret_cast<uint32_t*>(&x1);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t y0 = w0[j], y1 = w1[j];
    if (pairs) {
      const float a0 = bf16_lo(y0), b0 = bf16_hi(y0), a1 = bf16_lo(y1), b1 = bf16_hi(y1);
      w0[j] = two_bf16(a0 * t.c[j] - b0 * t.s[j], b0 * t.c[j] + a0 * t.s[j]);
      w1[j] = two_bf16(a1 * t.c[4 + j] - b1 * t.s[4 + j], b1 * t.c[4 + j] + a1 * t.s[4 + j]);
    } else {
      const float a0 = bf16_lo(y0), a1 = bf16_hi(y0), b0 = bf16_lo(y1), b1 = bf16_hi(y1);
      w0[j] = two_bf16(a0 * t.c[2 * j] - b0 * t.s[2 * j], a1 * t.c[2 * j + 1] - b1 * t.s[2 * j + 1]);
      w1[j] = two_bf16(b0 * t.c[2 * j] + a0 * t.s[2 * j], b1 * t.c[2 * j + 1] + a1 * t.s[2 * j + 1]);
    }
  }
}

}  // namespace gambit
