// Attention of packed rows over the paged caches for gfx950: prompts (causal,
// grouped heads, sequences of different lengths) and trees of drafted tokens.
//
// A row is a (packed token, query head of the GQA group); a workgroup takes
// up to 128 rows of one KV head, 32 a wave, over a range of cached positions,
// 64 at a time:
//   S^T[token][row] = K[token][:] . Q[row][:]            (A = K, B = Q^T)
//   O^T[d][row]    += V^T[d][token] . P^T[token][row]    (A = V^T, B = P^T)
// on v_mfma_f32_32x32x16_bf16, with the running maximum and sum of a softmax
// (fp32, exp2 domain), so the keys pass once.  The caches' tile layout is the
// operands' own: a stored K row order (bits 2 and 3 of the token swapped) puts
// into a lane's accumulators of S^T exactly the eight tokens that its B
// operand of the second product holds, and V is stored transposed.  So both
// products read 16 bytes a lane, 1 KiB of LDS in lane order, without bank
// conflicts; the tiles get there by direct global-to-LDS loads (bf16), or
// widened on the way (fp8, exact), one key tile ahead.
//
// P is one bf16 operand when the output is bf16 (its rounding, 2^-8 of a
// term, is of the output's own size and averages over the terms; the sum l is
// taken over the rounded values) and hi + lo bf16 parts (16 bits) when the
// output is fp32.
//
// A range that is split, or shared by several traces, leaves unnormalised
// partials that rows_merge_kernel joins by log-sum-exp.
#include <cmath>

#include "lds_dma.h"
#include "rows.h"

namespace gambit {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
#define GAMBIT_CONST __attribute__((address_space(4)))

constexpr int kThreads = 256;
constexpr int kVOff = kKeyTile * kHeadDim * 2;  // V behind K in a stage
constexpr int kStage = 2 * kVOff;
constexpr float kLazy = 8.f;  // a row's reference moves when a score exceeds it by 2^kLazy

__device__ inline uint32_t pack_bf16x2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// Scalar load of an int the launch does not write.
__device__ inline int ld_const(const int32_t* p) {
  return *reinterpret_cast<const GAMBIT_CONST int32_t*>(reinterpret_cast<uintptr_t>(p));
}
__device__ inline float ld_const(const float* p) {
  return *reinterpret_cast<const GAMBIT_CONST float*>(reinterpret_cast<uintptr_t>(p));
}

// One instruction (this source is built without IEEE mode, so the operands
// need no quieting first); a NaN operand is passed over.
__device__ inline float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

__device__ inline float other_half(float x) { return __shfl_xor(x, 32); }

// fp8 E4M3 -> bf16, eight codes (exact).
__device__ inline uint4 widen8(uint32_t w0, uint32_t w1) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, true);
  return make_uint4(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                    __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d));
}

// Keep the first nv of eight bf16 values.
__device__ inline uint4 keep_first(uint4 x, int nv) {
  x.x &= nv >= 2 ? 0xffffffffu : (nv == 1 ? 0xffffu : 0u);
  x.y &= nv >= 4 ? 0xffffffffu : (nv == 3 ? 0xffffu : 0u);
  x.z &= nv >= 6 ? 0xffffffffu : (nv == 5 ? 0xffffu : 0u);
  x.w &= nv >= 8 ? 0xffffffffu : (nv == 7 ? 0xffffu : 0u);
  return x;
}

__device__ inline bool not_finite2(uint32_t x) {
  return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
}

// The running state of a wave's 32 rows.  Lane (half h, row n): acc[db][r] is
// O[n][32 db + 8 (r / 4) + 4 h + r % 4]; l is the half's part of the sum.
struct Rows {
  float m, l;
  f32x16 acc[4];
};

// One stage in LDS:
//  K: [32-token half th][operand kb][d half][block of the two][row] 16 bytes
//  V: [block][32 d][token half][d % 32] 16 bytes
// so lane l's operand is at 16 l of each 1 KiB.
struct KeyScales {
  float k[4], v[4];  // of the tile's blocks (fp8)
};

// One key tile for the wave's rows.  MASKED: bit t of `vis` says whether the
// lane's row sees token t of the tile; tokens from nvalid on hold no values.
template <bool FP8, bool HILO, bool MASKED>
__device__ inline void key_tile(const uint8_t* stage, int lane, const bf16x8 (&q)[8], float c, const KeyScales& sc,
                                uint64_t vis, int nvalid, Rows& st) {
  const int h = lane >> 5;
  const uint8_t* base = stage + lane * 16;
  f32x16 s[2];
#pragma unroll
  for (int th = 0; th < 2; ++th) {
    s[th] = f32x16{};
#pragma unroll
    for (int kb = 0; kb < 8; ++kb)
      s[th] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          *reinterpret_cast<const bf16x8*>(base + (th * 8 + kb) * 1024), q[kb], s[th], 0, 0, 0);
  }
  if constexpr (MASKED) {
    const uint32_t v0 = (uint32_t)vis >> (8 * h), v1 = (uint32_t)(vis >> 32) >> (8 * h);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const uint32_t bit = 1u << (16 * (r / 8) + r % 8);
      s[0][r] = (v0 & bit) ? s[0][r] : -INFINITY;
      s[1][r] = (v1 & bit) ? s[1][r] : -INFINITY;
    }
  }
  float cb[4];
#pragma unroll
  for (int b = 0; b < 4; ++b) cb[b] = FP8 ? fmaxf(c * sc.k[b], 1e-37f) : c;
  float mx;
  if constexpr (FP8) {
    float mb[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const f32x16& x = s[b / 2];
      const int o = 8 * (b % 2);
      mb[b] = max3(max3(x[o], x[o + 1], x[o + 2]), max3(x[o + 3], x[o + 4], x[o + 5]), x[o + 6]);
      mb[b] = max3(mb[b], x[o + 7], x[o + 7]) * cb[b];
    }
    mx = max3(max3(mb[0], mb[1], mb[2]), mb[3], mb[3]);
  } else {
    mx = max3(s[0][0], s[0][1], s[1][0]);
#pragma unroll
    for (int r = 2; r < 16; r += 2) mx = max3(mx, s[0][r], s[0][r + 1]);
#pragma unroll
    for (int r = 1; r < 15; r += 2) mx = max3(mx, s[1][r], s[1][r + 1]);
    mx = max3(mx, s[1][15], s[1][15]) * c;
  }
  if (__builtin_amdgcn_ballot_w64(mx > st.m + kLazy)) {
    mx = max3(mx, other_half(mx), mx);
    const float m_new = mx > st.m + kLazy ? mx : st.m;
    const float alpha = m_new == st.m ? 1.f : __builtin_amdgcn_exp2f(st.m - m_new);
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < 4; ++db) st.acc[db] *= alpha;
    st.m = m_new;
  }
  const float nm = st.m == -INFINITY ? 0.f : -st.m;
  uint4 ph[4], pl[4];
  float l0 = 0.f, l1 = 0.f;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    uint32_t hw[4], lw[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x = __builtin_amdgcn_exp2f(fmaf(s[b / 2][8 * (b % 2) + 2 * j], cb[b], nm));
      float y = __builtin_amdgcn_exp2f(fmaf(s[b / 2][8 * (b % 2) + 2 * j + 1], cb[b], nm));
      if constexpr (FP8 || HILO) {
        l0 += x;
        l1 += y;
      }
      if constexpr (FP8) {
        x *= sc.v[b];
        y *= sc.v[b];
      }
      hw[j] = pack_bf16x2(x, y);
      if constexpr (HILO)
        lw[j] = pack_bf16x2(x - __uint_as_float(hw[j] << 16), y - __uint_as_float(hw[j] & 0xffff0000u));
      if constexpr (!FP8 && !HILO)
        l0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, hw[j]), bf16x2{(__bf16)1.f, (__bf16)1.f}, l0,
                                             false);
    }
    ph[b] = make_uint4(hw[0], hw[1], hw[2], hw[3]);
    if constexpr (HILO) pl[b] = make_uint4(lw[0], lw[1], lw[2], lw[3]);
  }
  st.l += l0 + l1;
  if constexpr (!MASKED) {
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int db = 0; db < 4; ++db) {
        const bf16x8 v = *reinterpret_cast<const bf16x8*>(base + kVOff + (b * 4 + db) * 1024);
        st.acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, ph[b]), st.acc[db], 0, 0, 0);
        if constexpr (HILO)
          st.acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, pl[b]), st.acc[db], 0, 0, 0);
      }
  } else {
    // A value that some rows see may be infinite or NaN where other rows have
    // P = 0, which the product would turn into NaN: such a block is added
    // row by row, from the tokens that the row sees.
#pragma unroll 1
    for (int b = 0; b < 4; ++b) {
      uint4 v[4];
      bool bad = false;
      const int nv = nvalid - 16 * b - 8 * h;
#pragma unroll
      for (int db = 0; db < 4; ++db) {
        v[db] = keep_first(*reinterpret_cast<const uint4*>(base + kVOff + (b * 4 + db) * 1024), nv);
        bad |= not_finite2(v[db].x) || not_finite2(v[db].y) || not_finite2(v[db].z) || not_finite2(v[db].w);
      }
      if (!__builtin_amdgcn_ballot_w64(bad)) {
#pragma unroll
        for (int db = 0; db < 4; ++db) {
          const bf16x8 x = __builtin_bit_cast(bf16x8, v[db]);
          st.acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8, ph[0]), st.acc[db], 0, 0, 0);
          if constexpr (HILO)
            st.acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8, pl[0]), st.acc[db], 0, 0, 0);
        }
      } else {
        uint4 w = ph[0], wl = HILO ? pl[0] : make_uint4(0, 0, 0, 0);
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
          float p = __uint_as_float(w.x << 16);
          if constexpr (HILO) p += __uint_as_float(wl.x << 16);
          const float po = other_half(p);
#pragma unroll 1
          for (int t = 0; t < 2; ++t) {  // the token of the lane's own half, then the other half's
            const int tok = 16 * b + 8 * (t ? 1 - h : h) + e;
            const float pt = t ? po : p;
            const bool sees = tok < nvalid && ((vis >> tok) & 1);
            const uint8_t* col = stage + kVOff + b * 4096 + ((tok >> 3) & 1) * 512 + 2 * e;
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const uint32_t x = *reinterpret_cast<const uint16_t*>(col + db * 1024 + (8 * (r / 4) + 4 * h + r % 4) * 16);
                const float add = pt * __uint_as_float(x << 16);
                st.acc[db][r] += sees ? add : 0.f;
              }
          }
          w = make_uint4(w.x >> 16 | w.y << 16, w.y >> 16 | w.z << 16, w.z >> 16 | w.w << 16, w.w >> 16);
          if constexpr (HILO)
            wl = make_uint4(wl.x >> 16 | wl.y << 16, wl.y >> 16 | wl.z << 16, wl.z >> 16 | wl.w << 16, wl.w >> 16);
        }
      }
      ph[0] = ph[1], ph[1] = ph[2], ph[2] = ph[3];
      if constexpr (HILO) pl[0] = pl[1], pl[1] = pl[2], pl[2] = pl[3];
    }
  }
}

// The drafts of a trace as a stage: tokens in rows there, so V is turned on
// the way.  Tokens past the tree are zeros.
__device__ inline void stage_drafts(const RowsLaunch& A, const RowItem& U, int Hkv, int kvh, int t, uint8_t* stage) {
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int u = t + x * kThreads, j = u >> 4, ch = u & 15;
    uint4 k = make_uint4(0, 0, 0, 0);
    if (j < U.ndraft)
      k = *reinterpret_cast<const uint4*>(A.k_new + ((size_t)(U.draft + j) * Hkv + kvh) * kHeadDim + 8 * ch);
    *reinterpret_cast<uint4*>(stage + ((j >> 5) * 8 + (ch >> 1)) * 1024 + (ch & 1) * 512 + ((j >> 4) & 1) * 256 +
                              k_phys(j & 15) * 16) = k;
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int u = t + x * kThreads, d = u & 127, j0 = (u >> 7) * 8;  // eight tokens of one d
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (j0 + e < U.ndraft)
        w[e / 2] |= (uint32_t)A.v_new[((size_t)(U.draft + j0 + e) * Hkv + kvh) * kHeadDim + d] << (16 * (e % 2));
    *reinterpret_cast<uint4*>(stage + kVOff + (j0 >> 4) * 4096 + (d >> 5) * 1024 + ((j0 >> 3) & 1) * 512 + (d & 31) * 16) =
        make_uint4(w[0], w[1], w[2], w[3]);
  }
}

template <bool FP8, bool HILO, bool DRAFT>
__global__ __launch_bounds__(kThreads, 2) void rows_attn_kernel(DevPool P, RowsLaunch A) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kStage];
  const int kvh = blockIdx.x % P.Hkv;
  const RowItem U = __builtin_bit_cast(
      RowItem, *reinterpret_cast<const GAMBIT_CONST i32x16*>(reinterpret_cast<uintptr_t>(A.items + blockIdx.x / P.Hkv)));
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int h = lane >> 5, gs = A.gshift;
  const int nrows = U.ntok << gs, row = 32 * w + (lane & 31);
  const bool here = row < nrows;
  int tok = 0;
  if (here) tok = U.listed ? A.list[U.tok + (row >> gs)] : U.tok + (row >> gs);
  const int head = (kvh << gs) + (row & ((1 << gs) - 1));

  // the wave's queries, row n of lane (n, h): d = 16 kb + 8 h ..
  bf16x8 q[8];
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) {
    uint4 x = make_uint4(0, 0, 0, 0);
    if (here) x = *reinterpret_cast<const uint4*>(A.q + ((size_t)tok * P.Hq + head) * kHeadDim + 16 * kb + 8 * h);
    x.x = (x.x & A.q_and) ^ A.q_xor, x.y = (x.y & A.q_and) ^ A.q_xor;
    x.z = (x.z & A.q_and) ^ A.q_xor, x.w = (x.w & A.q_and) ^ A.q_xor;
    q[kb] = __builtin_bit_cast(bf16x8, x);
  }
  Rows st;
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db) st.acc[db] = f32x16{};

  // positions the lane's row sees, and the fewest and most that a row of the wave does
  const int t0 = kBlock * U.jb0;
  auto limit = [&](int r) { return U.pos0 == kNoLimit ? U.end : min(U.end, U.pos0 + (r >> gs) + 1); };
  const int lim = limit(min(row, nrows - 1));
  const bool active = 32 * w < nrows;
  const int lim_lo = limit(32 * w), lim_hi = limit(min(32 * w + 31, nrows - 1));
  const int ntiles = U.end > t0 ? (U.end - t0 + kKeyTile - 1) / kKeyTile : 0;
  const int jlast = (U.end - 1) / kBlock;
  const int32_t* brow = P.table + (size_t)U.trace * P.max_blocks;
  const size_t tile_bytes = (size_t)kBlock * kHeadDim * (FP8 ? 1 : 2);

  int ids[4];        // blocks of the next tile to fetch
  KeyScales sc_next, sc;
  uint4 raw[4];      // fp8: the next tile on its way
  auto fetch_ids = [&](int i) {
#pragma unroll
    for (int b = 0; b < 4; ++b) ids[b] = ld_const(brow + min(U.jb0 + 4 * i + b, jlast));
  };
  auto id_of = [&](int b) { return b == 0 ? ids[0] : b == 1 ? ids[1] : b == 2 ? ids[2] : ids[3]; };  // b uniform
  auto tile_at = [&](const uint8_t* cache, int id) { return cache + ((size_t)id * P.Hkv + kvh) * tile_bytes; };
  auto check_ids = [&]() {
#pragma unroll
    for (int b = 0; b < 4; ++b)
      if ((unsigned)ids[b] >= (unsigned)P.num_blocks) {
        if (t == 0) atomicOr(P.err, kErrBadBlock);
        ids[b] = 0;
      }
  };
  // asks for tile i (ids): bf16 straight into the stage, fp8 into registers
  auto fetch = [&](uint8_t* stage) {
    check_ids();
    if constexpr (!FP8) {
      const int th = w >> 1, kb0 = 4 * (w & 1);
      const uint8_t* k = tile_at(P.k_cache, (lane & 16) ? id_of(2 * th + 1) : id_of(2 * th)) +
                         ((2 * kb0 + h) * kBlock + (lane & 15)) * 16;
      const uint8_t* v = tile_at(P.v_cache, id_of(w)) + (2 * (lane & 31) + h) * 16;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        dma16(k + x * 512, stage + (th * 8 + kb0 + x) * 1024);
        dma16(v + x * 1024, stage + kVOff + (w * 4 + x) * 1024);
      }
    } else {
      const int b = w >> 1, u = (t & 127) * 16;
      raw[0] = *reinterpret_cast<const uint4*>(tile_at(P.k_cache, id_of(b)) + u);
      raw[1] = *reinterpret_cast<const uint4*>(tile_at(P.k_cache, id_of(b + 2)) + u);
      raw[2] = *reinterpret_cast<const uint4*>(tile_at(P.v_cache, id_of(b)) + u);
      raw[3] = *reinterpret_cast<const uint4*>(tile_at(P.v_cache, id_of(b + 2)) + u);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        sc_next.k[x] = ld_const(P.kv_scale + 2 * ids[x]);
        sc_next.v[x] = ld_const(P.kv_scale + 2 * ids[x] + 1);
      }
    }
  };
  // fp8: the fetched tile widened into the stage
  auto settle = [&](uint8_t* stage) {
    if constexpr (FP8) {
      const int b = w >> 1, x = t & 127;
#pragma unroll
      for (int y = 0; y < 2; ++y) {  // blocks b and b + 2
        uint8_t* k = stage + (y * 8 + (x >> 4)) * 1024 + b * 256 + (x & 15) * 16;
        *reinterpret_cast<uint4*>(k) = widen8(raw[y].x, raw[y].y);
        *reinterpret_cast<uint4*>(k + 512) = widen8(raw[y].z, raw[y].w);
        uint8_t* v = stage + kVOff + (b + 2 * y) * 4096 + (x >> 5) * 1024 + (x & 31) * 16;
        *reinterpret_cast<uint4*>(v) = widen8(raw[2 + y].x, raw[2 + y].y);
        *reinterpret_cast<uint4*>(v + 512) = widen8(raw[2 + y].z, raw[2 + y].w);
      }
      sc = sc_next;
    }
  };

  if (ntiles > 0) {
    fetch_ids(0);
    fetch(lds);
    if (ntiles > 1) fetch_ids(1);
    settle(lds);
  }
#pragma unroll 1
  for (int i = 0; i < ntiles; ++i) {
    uint8_t* stage = lds + (i & 1) * kStage;
    // the tile is there in every wave, and no wave reads the other stage any more
    if constexpr (FP8)
      __syncthreads();
    else {
      __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt 0, lgkmcnt 0
      barrier_no_fence();
    }
    const KeyScales now = sc;
    if (i + 1 < ntiles) {
      fetch(lds + ((i + 1) & 1) * kStage);
      if (i + 2 < ntiles) fetch_ids(i + 2);
    }
    const int tb = t0 + kKeyTile * i;
    if (active && tb < lim_hi) {
      if (tb + kKeyTile <= lim_lo) {
        key_tile<FP8, HILO, false>(stage, lane, q, A.c, now, 0, kKeyTile, st);
      } else {
        const int k = min(max(lim - tb, 0), kKeyTile);
        const uint64_t vis = k >= 64 ? ~0ull : (1ull << k) - 1;
        key_tile<FP8, HILO, true>(stage, lane, q, A.c, now, vis, U.end - tb, st);
      }
    }
    if (i + 1 < ntiles) settle(lds + ((i + 1) & 1) * kStage);
  }
  if constexpr (DRAFT) {
    if (U.draft >= 0) {  // uniform
      __syncthreads();   // the last tile is read
      stage_drafts(A, U, P.Hkv, kvh, t, lds);
      __syncthreads();
      if (active) {
        KeyScales one;
#pragma unroll
        for (int b = 0; b < 4; ++b) one.k[b] = one.v[b] = 1.f;
        const uint64_t vis = here ? A.anc[tok] : 1;
        key_tile<FP8, HILO, true>(lds, lane, q, A.c, one, vis, kKeyTile, st);
      }
    }
  }
  const float l = st.l + other_half(st.l);
  if (!here) return;
  if (U.kidx < 0) {
    const float inv = 1.f / l;
    const size_t o = ((size_t)tok * P.Hq + head) * kHeadDim + 4 * h;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 x = {st.acc[db][4 * j] * inv, st.acc[db][4 * j + 1] * inv, st.acc[db][4 * j + 2] * inv,
                         st.acc[db][4 * j + 3] * inv};
        const size_t at = o + 32 * db + 8 * j;
        if constexpr (HILO)
          *reinterpret_cast<f32x4*>(static_cast<float*>(A.out) + at) = x;
        else
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(A.out) + at) =
              make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
      }
    return;
  }
  const size_t part = (size_t)(A.off[tok] + U.kidx) * P.Hq + head;
  float* dst = A.part_acc + part * kHeadDim + 4 * h;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<f32x4*>(dst + 32 * db + 8 * j) =
          f32x4{st.acc[db][4 * j], st.acc[db][4 * j + 1], st.acc[db][4 * j + 2], st.acc[db][4 * j + 3]};
  if (h == 0) A.part_ml[part] = float2{st.m, l};
}

// out = sum_k 2^(m_k - M) acc_k / sum_k 2^(m_k - M) l_k, M the largest m_k;
// eight rows a workgroup, 32 lanes of four d a row.  A partial without a seen
// position has m = -inf and counts for nothing.
__global__ __launch_bounds__(256) void rows_merge_kernel(RowsLaunch A, int32_t Hq) {
  const int r = blockIdx.x * 8 + (threadIdx.x >> 5), x = threadIdx.x & 31;
  if (r >= A.n_merge * Hq) return;
  const int tok = A.merge[r / Hq], head = r % Hq;
  const int n = A.nk[tok];
  const size_t p0 = (size_t)A.off[tok] * Hq + head;
  float M = -INFINITY;
  for (int k = 0; k < n; ++k) M = fmaxf(M, A.part_ml[p0 + (size_t)k * Hq].x);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int k = 0; k < n; ++k) {
    const size_t p = p0 + (size_t)k * Hq;
    const float2 ml = A.part_ml[p];
    const f32x4 a = *reinterpret_cast<const f32x4*>(A.part_acc + p * kHeadDim + 4 * x);
    const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    l = fmaf(f, ml.y, l);
    if (f != 0.f)
      for (int e = 0; e < 4; ++e) o[e] = fmaf(f, a[e], o[e]);
  }
  const float inv = 1.f / l;
  const size_t at = ((size_t)tok * Hq + head) * kHeadDim + 4 * x;
  if (A.out_f32)
    *reinterpret_cast<f32x4*>(static_cast<float*>(A.out) + at) = f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(A.out) + at) =
        make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
}

template <bool FP8, bool HILO>
void launch_items(const DevPool& P, const RowsLaunch& L, hipStream_t s) {
  const dim3 grid((unsigned)L.n_items * P.Hkv);
  if (L.anc)
    hipLaunchKernelGGL((rows_attn_kernel<FP8, HILO, true>), grid, dim3(kThreads), 0, s, P, L);
  else
    hipLaunchKernelGGL((rows_attn_kernel<FP8, HILO, false>), grid, dim3(kThreads), 0, s, P, L);
}

}  // namespace

hipError_t launch_rows_attention(const DevPool& P, const RowsLaunch& L, hipStream_t s) {
  if (L.n_items <= 0) return hipSuccess;
  const bool fp8 = P.esize == 1, hilo = L.out_f32;
  if (fp8 && hilo) launch_items<true, true>(P, L, s);
  if (fp8 && !hilo) launch_items<true, false>(P, L, s);
  if (!fp8 && hilo) launch_items<false, true>(P, L, s);
  if (!fp8 && !hilo) launch_items<false, false>(P, L, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || L.n_merge == 0) return e;
  hipLaunchKernelGGL(rows_merge_kernel, dim3(((unsigned)L.n_merge * P.Hq + 7) / 8), dim3(256), 0, s, L, P.Hq);
  return hipGetLastError();
}

}  // namespace gambit
