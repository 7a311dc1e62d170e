// Packed tokens of several traces into one layer's caches.
//
// A workgroup takes the part of one block that a trace's tokens cover: for
// bf16 pools one KV head of it, a 16-byte chunk of K and of V a thread; for
// fp8 pools all heads of K or of V, since a block has one scale of each, the
// largest written magnitude / 448 over tokens and heads (so that it becomes
// E4M3FN's largest value).  Both are bound by HBM: token rows are read whole
// (256 bytes a head), turned in LDS into the caches' tile layout, and stored
// 16 bytes a lane in order.
#include "rows.h"

namespace gambit {
namespace {

constexpr int kRow = kHeadDim * 2;  // bytes of a token's head in the caller's K or V

// Nearest E4M3FN code of y (ties to even; beyond 448 saturating; NaN stays).
__device__ inline uint32_t fp8_code(float y) {
  const uint32_t u = __float_as_uint(y), sign = (u >> 24) & 0x80u, m = u & 0x7FFFFFFFu;
  const float a = __uint_as_float(m);
  uint32_t c;
  if (m > 0x7F800000u)
    c = 0x7Fu;
  else if (a >= 448.f)
    c = 0x7Eu;
  else if (a < 0.015625f)  // subnormal: steps of 2^-9
    c = (uint32_t)__builtin_rintf(a * 512.f);
  else
    c = ((m + 0x7FFFFu + ((m >> 20) & 1u)) >> 20) - (120u << 3);
  return sign | c;
}

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

// blockIdx.y: 0 K, 1 V.  Heads go eight at a time through registers: their
// tokens are read once where a block has at most eight heads, twice otherwise.
__global__ __launch_bounds__(256) void rows_write_fp8_kernel(DevPool P, WriteLaunch L) {
  constexpr int kHeads = 8, kTile = kBlock * kHeadDim;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kHeads * kTile];
  __shared__ uint32_t most_s[4];
  const int t = threadIdx.x, which = blockIdx.y;
  const WriteItem U = L.items[blockIdx.x];
  const int r0 = U.r0, r1 = U.r1, row = t >> 4, c = t & 15;
  const uint16_t* src = (which ? L.v : L.k) + source_row(L, U.src + min(max(row, r0), r1 - 1) - r0) * P.Hkv * kHeadDim + 8 * c;
  uint4 x[kHeads];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      x[i] = *reinterpret_cast<const uint4*>(src + (size_t)min(h0 + i, P.Hkv - 1) * kHeadDim);
  };
  float* scale_at = P.kv_scale + 2 * (size_t)U.blk + which;
  float s;
  load(0);
  if (U.floor > 0.f) {
    // the magnitudes of bf16 values are ordered as their bits; NaN counts for nothing
    uint32_t most = 0;
    for (int h0 = 0; h0 < P.Hkv; h0 += kHeads) {
      if (h0) load(h0);
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
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
  uint8_t* cache = which ? P.v_cache : P.k_cache;
  for (int h0 = 0; h0 < P.Hkv; h0 += kHeads) {
    const int nh = min(kHeads, P.Hkv - h0);
    if (h0) {
      __syncthreads();  // the tiles of the heads before are stored
      load(h0);
    }
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      if (i >= nh) break;
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
      uint32_t y[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y[2 * j] = fp8_code(__uint_as_float(w[j] << 16) / s);
        y[2 * j + 1] = fp8_code(__uint_as_float(w[j] & 0xffff0000u) / s);
      }
      uint8_t* tile = lds + i * kTile;
      if (which == 0) {  // elements 8 c .. 8 c + 7 of the row: half a 16-byte chunk
        *reinterpret_cast<uint2*>(tile + ((c >> 1) * kBlock + k_phys(row)) * 16 + (c & 1) * 8) =
            make_uint2(y[0] | y[1] << 8 | y[2] << 16 | y[3] << 24, y[4] | y[5] << 8 | y[6] << 16 | y[7] << 24);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[(8 * c + j) * kBlock + row] = (uint8_t)y[j];
      }
    }
    __syncthreads();
    uint8_t* dst = cache + ((size_t)U.blk * P.Hkv + h0) * kTile;
    for (int u = t; u < nh * (kTile / 16); u += 256) {
      const uint4 v = *reinterpret_cast<const uint4*>(lds + u * 16);
      const int krow = k_phys(u & 15);
      if (which == 0 ? (krow >= r0 && krow < r1) : (r0 == 0 && r1 == kBlock)) {
        *reinterpret_cast<uint4*>(dst + u * 16) = v;
      } else if (which == 1) {
        for (int e = r0; e < r1; ++e) dst[u * 16 + e] = lds[u * 16 + e];
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
