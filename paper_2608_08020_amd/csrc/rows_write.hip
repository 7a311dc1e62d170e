// Packed tokens of several traces into one layer's caches.
//
// A workgroup takes the part of one block that a trace's tokens cover: for
// bf16 pools one KV head of it, a 16-byte chunk of K and of V a thread; for
// fp8 pools all heads of K or of V, since a block has one scale of each, the
// largest written magnitude / 448 over tokens and heads (so that it becomes
// E4M3FN's largest value).  Both are bound by HBM: token rows are read whole
// (256 bytes a head), turned in LDS into the caches' tile layout, and stored
// 16 bytes a lane in order.  Measured with 8 KV heads (a large copy: 4.76 TB/s):
// bf16, eight segments of 2048 to 8192 tokens, 374 MB, 71 us, 5.3 TB/s; eight traces of
// one to five tokens 3 us, latency; fp8, sixteen prompts of 256 to 1024 tokens,
// 60 MB, 16 us (26 us with one workgroup for a block's K and V).
#include "rows.h"

namespace gambit {
namespace {

constexpr int kRow = kHeadDim * 2;  // bytes of a token's head in the caller's K or V

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

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

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ inline size_t source_row(const WriteLaunch& L, int tok) { return L.rows ? L.rows[tok] : tok; }

__global__ __launch_bounds__(256) void rows_write_bf16_kernel(DevPool P, WriteLaunch L) {
  constexpr int kVRow = kRow + 8, kKCol = kBlock * 16 + 16;
  __shared__ __attribute__((aligned(16))) uint8_t klds[16 * kKCol], vlds[kBlock * kVRow];
  const int head = blockIdx.x % P.Hkv, t = threadIdx.x;
  const WriteItem U = L.items[blockIdx.x / P.Hkv];
  const int r0 = U.r0, r1 = U.r1;
  {
    const int row = t >> 4, c = t & 15;
    // rows outside the write re-read one inside it (never stored)
    const size_t src = (source_row(L, U.src + min(max(row, r0), r1 - 1) - r0) * P.Hkv + head) * kHeadDim + 8 * c;
    const uint4 kk = *reinterpret_cast<const uint4*>(L.k + src), vv = *reinterpret_cast<const uint4*>(L.v + src);
    *reinterpret_cast<uint4*>(klds + c * kKCol + k_phys(row) * 16) = kk;
    uint2* vd = reinterpret_cast<uint2*>(vlds + row * kVRow + c * 16);
    vd[0] = make_uint2(vv.x, vv.y);
    vd[1] = make_uint2(vv.z, vv.w);
  }
  __syncthreads();
  const size_t tile = ((size_t)U.blk * P.Hkv + head) * kBlock * kRow;
  const int krow = k_phys(t & 15);  // k_phys is its own inverse
  if (krow >= r0 && krow < r1)
    *reinterpret_cast<uint4*>(P.k_cache + tile + t * 16) =
        *reinterpret_cast<const uint4*>(klds + (t >> 4) * kKCol + (t & 15) * 16);
  const int d = t >> 1, f = (t & 1) * 8;  // the chunk's tokens: f .. f + 7 of element d
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    w[e / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(vlds + (f + e) * kVRow + d * 2) << (16 * (e % 2));
  uint8_t* dst = P.v_cache + tile + t * 16;
  if (f >= r0 && f + 8 <= r1) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (f + e >= r0 && f + e < r1) reinterpret_cast<uint16_t*>(dst)[e] = (uint16_t)(w[e / 2] >> (16 * (e % 2)));
  }
}

// blockIdx.y: 0 K, 1 V.  Two heads of the block a pass, a half of the workgroup
// each, four passes in registers (so a block of at most eight heads is read
// once, a larger one twice: magnitudes, then codes).  K: a thread takes 16 d of
// a row, one 16-byte chunk of the tile, in the tile's order, so its stores need
// no turning.  V: four tokens by four d, turned in LDS.
__global__ __launch_bounds__(256) void rows_write_fp8_kernel(DevPool P, WriteLaunch L) {
  constexpr int kPasses = 4, kHeads = 2 * kPasses, kTile = kBlock * kHeadDim;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kHeads * kTile];
  __shared__ uint32_t most_s[4];
  const int t = threadIdx.x, half = t >> 7, u = t & 127;
  const bool is_v = blockIdx.y != 0;
  const WriteItem U = L.items[blockIdx.x];
  const int r0 = U.r0, r1 = U.r1;
  // the thread's rows: K one, V four; rows outside the write re-read one inside it (never stored)
  const int krow = k_phys(u & 15), c = u >> 4;   // K: 16-byte chunk c of row krow
  const int tg = u >> 5, dg = u & 31;            // V: tokens 4 tg .., d 4 dg ..
  size_t src[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = is_v ? 4 * tg + i : krow;
    src[i] = source_row(L, U.src + min(max(row, r0), r1 - 1) - r0) * P.Hkv * kHeadDim + (is_v ? 4 * dg : 16 * c);
  }
  uint4 x[kPasses][2];  // K: 16 values of a row; V: 4 values of 4 rows
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
      if (h0 + 2 * i >= P.Hkv) continue;  // uniform
      const size_t h = (size_t)min(h0 + 2 * i + half, P.Hkv - 1) * kHeadDim;
      if (is_v) {
        u32x2 y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const u32x2*>(L.v + src[j] + h);
        x[i][0] = make_uint4(y[0].x, y[0].y, y[1].x, y[1].y);
        x[i][1] = make_uint4(y[2].x, y[2].y, y[3].x, y[3].y);
      } else {
        x[i][0] = *reinterpret_cast<const uint4*>(L.k + src[0] + h);
        x[i][1] = *reinterpret_cast<const uint4*>(L.k + src[0] + h + 8);
      }
    }
  };
  float* scale_at = P.kv_scale + 2 * (size_t)U.blk + is_v;
  float s;
  load(0);
  if (U.floor > 0.f) {
    // the magnitudes of bf16 values are ordered as their bits; NaN counts for nothing
    uint32_t most = 0;
    for (int h0 = 0; h0 < P.Hkv; h0 += kHeads) {
      if (h0) load(h0);
#pragma unroll
      for (int i = 0; i < 2 * kPasses; ++i) {
        const uint4 y = x[i / 2][i % 2];
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t lo = w[j] & 0x7fffu, hi = (w[j] >> 16) & 0x7fffu;
          most = max(most, lo > 0x7f80u ? 0u : lo);
          most = max(most, hi > 0x7f80u ? 0u : hi);
        }
      }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
    if ((t & 63) == 0) most_s[t >> 6] = most;
    __syncthreads();
    most = max(max(most_s[0], most_s[1]), max(most_s[2], most_s[3]));
    s = fmaxf(__uint_as_float(min(most, 0x7f7fu) << 16) / 448.f, U.floor);
    if (t == 0) *scale_at = s;
    if (P.Hkv > kHeads) load(0);
  } else {
    s = *scale_at;
  }
  // a scale near zero and the values both times 2^64 (exact, or beyond where the
  // quotient saturates); of a scale of zero, zero stays zero and the rest saturates
  const bool tiny = fabsf(s) < 0x1p-64f;  // uniform
  if (tiny) s *= 0x1p64f;
  const float r = fminf(1.f / s, 0x1.fffffep127f);
  auto q = [&](float y) { return quotient(y, s, r); };
  auto grown = [](uint32_t w) {
    return __float_as_uint(bf16_lo(w) * 0x1p64f) >> 16 | (__float_as_uint(bf16_hi(w) * 0x1p64f) & 0xffff0000u);
  };
  uint8_t* cache = (is_v ? P.v_cache : P.k_cache) + (size_t)U.blk * P.Hkv * kTile;
  for (int h0 = 0; h0 < P.Hkv; h0 += kHeads) {
    const int nh = min(kHeads, P.Hkv - h0);
    if (h0) {
      __syncthreads();  // the heads before are stored
      load(h0);
    }
    if (tiny) {
#pragma unroll
      for (int i = 0; i < 2 * kPasses; ++i) {
        uint4& y = x[i / 2][i % 2];
        y = make_uint4(grown(y.x), grown(y.y), grown(y.z), grown(y.w));
      }
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      if (2 * i >= nh) continue;  // uniform
      const int hh = 2 * i + half;
      const uint4 a = x[i][0], b = x[i][1];
      if (!is_v) {
        const uint4 y = make_uint4(fp8_codes(q(bf16_lo(a.x)), q(bf16_hi(a.x)), q(bf16_lo(a.y)), q(bf16_hi(a.y))),
                                   fp8_codes(q(bf16_lo(a.z)), q(bf16_hi(a.z)), q(bf16_lo(a.w)), q(bf16_hi(a.w))),
                                   fp8_codes(q(bf16_lo(b.x)), q(bf16_hi(b.x)), q(bf16_lo(b.y)), q(bf16_hi(b.y))),
                                   fp8_codes(q(bf16_lo(b.z)), q(bf16_hi(b.z)), q(bf16_lo(b.w)), q(bf16_hi(b.w))));
        if (hh < nh && krow >= r0 && krow < r1) *reinterpret_cast<uint4*>(cache + (size_t)(h0 + hh) * kTile + u * 16) = y;
      } else {
        uint32_t* tile = reinterpret_cast<uint32_t*>(lds + hh * kTile) + tg;  // [d][tokens]
        tile[(4 * dg + 0) * 4] = fp8_codes(q(bf16_lo(a.x)), q(bf16_lo(a.z)), q(bf16_lo(b.x)), q(bf16_lo(b.z)));
        tile[(4 * dg + 1) * 4] = fp8_codes(q(bf16_hi(a.x)), q(bf16_hi(a.z)), q(bf16_hi(b.x)), q(bf16_hi(b.z)));
        tile[(4 * dg + 2) * 4] = fp8_codes(q(bf16_lo(a.y)), q(bf16_lo(a.w)), q(bf16_lo(b.y)), q(bf16_lo(b.w)));
        tile[(4 * dg + 3) * 4] = fp8_codes(q(bf16_hi(a.y)), q(bf16_hi(a.w)), q(bf16_hi(b.y)), q(bf16_hi(b.w)));
      }
    }
    if (!is_v) continue;
    __syncthreads();
    for (int d = t; d < nh * kHeadDim; d += 256) {
      uint8_t* dst = cache + (size_t)h0 * kTile + d * kBlock;
      if (r0 == 0 && r1 == kBlock) {
        *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(lds + d * kBlock);
      } else {
        for (int e = r0; e < r1; ++e) dst[e] = lds[d * kBlock + e];
      }
    }
  }
}

}  // namespace

hipError_t launch_rows_write(const DevPool& P, const WriteLaunch& L, hipStream_t s) {
  if (L.n_items <= 0) return hipSuccess;
  if (P.esize == 2)
    hipLaunchKernelGGL(rows_write_bf16_kernel, dim3((unsigned)L.n_items * P.Hkv), dim3(256), 0, s, P, L);
  else
    hipLaunchKernelGGL(rows_write_fp8_kernel, dim3(L.n_items, 2), dim3(256), 0, s, P, L);
  return hipGetLastError();
}

}  // namespace gambit
