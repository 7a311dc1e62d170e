// Rotated queries and keys of new tokens (gambit_rotate), kernel and host
// entry point.  A thread turns one unit of one head, both chunks, so that a head may be turned in
// place.  Bound by HBM at many tokens and by the launch at few: 32 query and 8 key
// heads, 64 tokens 3.2 us, 8192 tokens 27 us (6.1 TB/s; four heads a thread, which read
// the table a quarter as often: 27 us, and 135 against 123 us at 32768 tokens).
#include <hip/hip_runtime.h>

#include "../../include/gambit.h"
#include "kernels.h"
#include "rotary.h"

namespace gambit {
namespace {

struct RotateArgs {
  const uint16_t* x[2];  // queries, keys
  int64_t stride[2];     // values between tokens
  uint16_t* out[2];      // [n][heads][128]
  int32_t heads[2];
  int32_t n;
  const int32_t* pos;
  const float* table;
  int32_t n_pos, rot, pairs;
};

__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs A, uint32_t per_token, uint32_t total) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const uint32_t tok = i / per_token, j = i % per_token;
  const int unit = j & 7, h = j >> 3, side = h >= A.heads[0], hh = h - side * A.heads[0];
  const int pos = A.pos[tok];
  const bool ok = pos >= 0 && pos < A.n_pos, turns = unit < A.rot / 16;
  Turn t = load_turn(A.table + (size_t)(ok ? pos : 0) * A.rot, A.rot, turns ? unit : 0);
  if (!ok) {
#pragma unroll
    for (int e = 0; e < 8; ++e) t.c[e] = t.s[e] = __builtin_nanf("");
  }
  int c0, c1;
  unit_chunks(unit, A.rot, A.pairs, &c0, &c1);
  const uint16_t* p = A.x[side] + (size_t)tok * A.stride[side] + (size_t)hh * kHeadDim;
  uint4 x0 = *reinterpret_cast<const uint4*>(p + 8 * c0), x1 = *reinterpret_cast<const uint4*>(p + 8 * c1);
  if (turns) turn_unit(x0, x1, t, A.pairs);
  uint16_t* to = A.out[side] + ((size_t)tok * A.heads[side] + hh) * kHeadDim;
  *reinterpret_cast<uint4*>(to + 8 * c0) = x0;
  *reinterpret_cast<uint4*>(to + 8 * c1) = x1;
}

bool bad(const void* x, int64_t stride, const void* out) {
  return !x || !out || reinterpret_cast<uintptr_t>(x) % 16 || reinterpret_cast<uintptr_t>(out) % 16 || stride < 0 || stride % 8;
}

}  // namespace
}  // namespace gambit

extern "C" gambit_status gambit_rotate(int32_t n, int32_t q_heads, int32_t k_heads, const void* q, int64_t q_stride,
                                       const void* k, int64_t k_stride, const int32_t* positions, const float* table,
                                       int32_t n_pos, int32_t rot, int32_t pairs, void* q_out, void* k_out,
                                       void* stream) {
  using namespace gambit;
  if (n < 0 || q_heads < 0 || k_heads < 0 || rot < 16 || rot > kHeadDim || rot % 16 || n_pos < 1) return GAMBIT_ERR_INVALID;
  const int64_t heads = (int64_t)q_heads + k_heads;
  if (heads > 4096 || n * heads * 8 > 0x7fffffff) return GAMBIT_ERR_UNSUPPORTED;
  if (n == 0 || heads == 0) return GAMBIT_OK;
  if (!positions || reinterpret_cast<uintptr_t>(positions) % 4 || !table || reinterpret_cast<uintptr_t>(table) % 16) return GAMBIT_ERR_INVALID;
  if ((q_heads && bad(q, q_stride, q_out)) || (k_heads && bad(k, k_stride, k_out))) return GAMBIT_ERR_INVALID;
  RotateArgs A{{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k)},
               {q_stride, k_stride},
               {static_cast<uint16_t*>(q_out), static_cast<uint16_t*>(k_out)},
               {q_heads, k_heads},
               n, positions, table, n_pos, rot, pairs != 0};
  const uint32_t per_token = 8 * (uint32_t)heads, total = n * per_token;
  hipLaunchKernelGGL(rotate_kernel, dim3((total + 255) / 256), dim3(256), 0, static_cast<hipStream_t>(stream), A, per_token, total);
  return hipGetLastError() == hipSuccess ? GAMBIT_OK : GAMBIT_ERR_DEVICE;
}
