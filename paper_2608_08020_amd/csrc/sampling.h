// What the sampling kernels share: a call's arguments, a row's values, weights.
#pragma once

#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>
#include <cstdint>

#include "fp8_codes.h"

namespace gambit {

constexpr int kMaxVocab = 1 << 18;
constexpr int kBits = 44;                      // S: 2^18 weights of 2^44 sum to 2^62
constexpr int kSegs = kMaxVocab / 4 / 64 + 1;  // 64 loads (a wave's) of 16 bytes each; rows may start inside one

typedef unsigned long long u64;

struct SampleArgs {
  const void* z;
  int64_t stride;  // values between rows
  int32_t vocab;
  const float* u;
  const float* temperature;  // [n], or null: t_all for every row; the others alike
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  float t_all, p_all, m_all;
  int32_t k_all;
  int32_t* out;
};

// A row's parameters.
struct Filter {
  float p, min_p;
  int k;
  double slope;  // log2(e) / temperature
  bool greedy, use_k, use_p;
  __device__ __forceinline__ Filter(const SampleArgs& A, int r) {
    const float T = A.temperature ? A.temperature[r] : A.t_all;
    p = A.top_p ? A.top_p[r] : A.p_all;
    min_p = A.min_p ? A.min_p[r] : A.m_all;
    k = A.top_k ? A.top_k[r] : A.k_all;
    use_k = k > 0 && k < A.vocab;
    use_p = p < 1.f;
    greedy = !(T > 0.f) || k == 1 || (use_p && p <= 0.f);
    slope = 1.4426950408889634 / (double)T;
  }
  // log2 of what a kept weight has at least
  __device__ __forceinline__ double least() const { return min_p > 0.f ? log2((double)fminf(min_p, 1.f)) : -INFINITY; }
};

__device__ inline uint32_t key_of(float z) {  // ordered as the values are
  const uint32_t b = __float_as_uint(z);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

template <bool kF32>
struct Row {
  static constexpr int kPer = kF32 ? 4 : 8;  // values of a 16-byte load
  const uint8_t* base;                       // of load 0, 16-byte aligned: `lead` values before the row
  int lead, vocab, loads;

  __device__ __forceinline__ Row(const void* z, int64_t at, int vocab_) : vocab(vocab_) {
    const uint8_t* p = static_cast<const uint8_t*>(z) + at * (kF32 ? 4 : 2);
    lead = (int)(reinterpret_cast<uintptr_t>(p) & 15) / (kF32 ? 4 : 2);
    base = p - (reinterpret_cast<uintptr_t>(p) & 15);
    loads = (lead + vocab + kPer - 1) / kPer;
  }
  // NaN counts as -inf, +inf as the largest finite value, -0 as 0.
  __device__ static float clean(float x) { return x == x ? fminf(x, FLT_MAX) + 0.f : -INFINITY; }
  __device__ int index(int load, int i) const { return load * kPer + i - lead; }
  __device__ __forceinline__ bool there(int load) const { return (uint32_t)load < (uint32_t)loads; }
  __device__ __forceinline__ bool whole(int load) const { return there(load) && index(load, 0) >= 0 && index(load, 0) + kPer <= vocab; }
  __device__ __forceinline__ uint4 raw(int load) const { return *reinterpret_cast<const uint4*>(base + (size_t)load * 16); }
  __device__ __forceinline__ static void unpack_as_is(uint4 a, float* z) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kF32) {
        z[i] = __uint_as_float(w[i]);
      } else {
        z[2 * i] = bf16_lo(w[i]);
        z[2 * i + 1] = bf16_hi(w[i]);
      }
    }
  }
  __device__ __forceinline__ static void unpack(uint4 a, float* z) {
    unpack_as_is(a, z);
#pragma unroll
    for (int i = 0; i < kPer; ++i) z[i] = clean(z[i]);
  }
  // The values of a load that the row holds in part or not at all: places outside it are not read and count as -inf.
  __device__ __forceinline__ void edge(int load, float* z) const {
    const uint8_t* p = base + (size_t)load * 16;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = index(load, i);
      z[i] = -INFINITY;
      if (!there(load) || at < 0 || at >= vocab) continue;
      if constexpr (kF32)
        z[i] = clean(reinterpret_cast<const float*>(p)[i]);
      else
        z[i] = clean(__uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16));
    }
  }
  __device__ __forceinline__ void get(int load, float* z) const {
    if (whole(load))
      unpack(raw(load), z);
    else
      edge(load, z);
  }
};

// round(2^44 2^x) for x = q / 64 + r, |r| <= 1 / 128, -64 <= x <= 0, powers[i] = 2^(i / 64).
__device__ inline u64 weight_of(int q, double r, const double* powers) {
  double p = fma(r, 9.6181291076284772e-3, 5.5504108664821580e-2);  // ln(2)^n / n!
  p = fma(r, p, 2.4022650695910071e-1);
  p = fma(r, p, 6.9314718055994531e-1);
  p = fma(r, p, 1.0);
  p *= powers[q & 63];
  // times 2^(q / 64 + 44) in the exponent's bits; 2^52 more leaves the whole number in the last ones
  p = __hiloint2double(__double2hiint(p) + (((q >> 6) + kBits) << 20), __double2loint(p)) + 0x1p52;
  return (u64)__double_as_longlong(p) - 0x4330000000000000ull;
}
constexpr double kTo64ths = 0x1.8p46;  // added to a number below 2^25: its last bit is 1/64

// Maximum over a wave.
template <int kCtrl, int kRows>
__device__ inline float dpp_max(float x) {
  const int o = __builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), kCtrl, kRows, 0xf, false);
  return fmaxf(x, __int_as_float(o));
}
__device__ inline float wave_max(float x) {
  x = dpp_max<0x121, 0xf>(dpp_max<0x122, 0xf>(dpp_max<0x124, 0xf>(dpp_max<0x128, 0xf>(x))));  // rotations by 8, 4, 2, 1 in a row of 16
  x = dpp_max<0x143, 0xc>(dpp_max<0x142, 0xa>(x));  // rows 0 and 2 into 1 and 3, then 1 into 2 and 3
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// What the kept values have at least: a key, and of equal ones an index at most.
struct Cut {
  uint32_t key, index;
  __device__ bool holds(float z, int i) const {
    const uint32_t k = key_of(z);
    return k > key || (k == key && (uint32_t)i <= index);
  }
};

__device__ inline u64 wave_total(u64 x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ inline u64 wave_before(u64 x, int lane) {  // sum of the lanes before
  u64 y = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 z = __shfl_up(y, o);
    if (lane >= o) y += z;
  }
  return y - x;
}
// Sum of x over the threads before this one; *all: over all of them.
template <int kThreads>
__device__ inline u64 block_before(u64 x, u64* lds, u64* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const u64 y = wave_before(x, lane);
  __syncthreads();  // an earlier scan has been read
  if (lane == 63) lds[wave] = y + x;
  __syncthreads();
  u64 before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const u64 z = lds[w];
    if (w < wave) before += z;
    sum += z;
  }
  *all = sum;
  return before + y;
}
// Ascending sort of list[0 .. n), padded to a power of two with the largest
// number.  A wave's 64 pairs a step stay within its own 128 places while they
// are at most 64 apart: such steps need no barrier.
template <int kThreads>
__device__ inline void block_sort(u64* list, int n) {
  int m = 128;
  while (m < n) m <<= 1;
  for (int i = n + threadIdx.x; i < m; i += kThreads) list[i] = ~0ull;
  __syncthreads();
  bool wide = false;
  for (int k = 2; k <= m; k <<= 1)
    for (int j = k >> 1; j; j >>= 1) {
      if (j > 64 || wide)
        __syncthreads();
      else
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      wide = j > 64;
      for (int i = threadIdx.x; i < m / 2; i += kThreads) {
        const int a = 2 * i - (i & (j - 1)), b = a + j;
        const u64 x = list[a], y = list[b];
        if ((x > y) == ((a & k) == 0)) {
          list[a] = y;
          list[b] = x;
        }
      }
    }
  __syncthreads();
}

// A workgroup's LDS, as one of the kernels' or another's.  (Through a function, so
// that every access is seen to be to LDS.)
constexpr int kSampleLds = 80 * 1024;
__device__ __forceinline__ unsigned char* lds_bytes() {
  __shared__ __attribute__((aligned(16))) unsigned char bytes[kSampleLds];
  return bytes;
}
template <class T>
__device__ __forceinline__ T& lds_as() {
  static_assert(sizeof(T) <= kSampleLds, "two workgroups a compute unit");
  return *reinterpret_cast<T*>(lds_bytes());
}

}  // namespace gambit
