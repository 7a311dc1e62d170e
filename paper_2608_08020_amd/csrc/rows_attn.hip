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
// taken over the rounded values) and three bf16 planes (24 bits) when the
// output is fp32.
//
// A range that is split, or shared by several traces, leaves unnormalised
// partials that rows_merge_kernel joins by log-sum-exp.
//
// Why 128 rows: a wave reads a key tile's 32 KiB (both operands, bf16) from LDS
// for 32 rows, 1024 cycles of its matrix unit; with fewer rows LDS would bound
// (it is busy 27% of the cycles of a long prompt, the matrix units 52%).  Two
// workgroups a CU leave 256 registers a lane, which hold the wave's queries (32),
// outputs (64) and the scores of two tiles (64), and 80 KiB of LDS each: two
// buffers of K and of V fill 64.
//
// What bounds it, measured (medians of kernel times; a large copy: 4.76 TB/s, a
// large library product: 1.25 PFLOP/s):
//   long prompts, bf16: the matrix units and what issues beside them.  One of
//     8192 tokens, 32 query heads over 8: 505 us, 1.09 PFLOP/s of what is seen
//     (about a fifth longer before the order of plain_tile was written out)
//   long prompts, fp8: the same, and the codes' way to bf16 through registers
//     and LDS, once per workgroup.  Four of 1024 to 4096 tokens, 64 query heads
//     over 8: 522 us, 0.90 PFLOP/s
//   short prompts: a workgroup's start, masked tile and end, over a third of its
//     time at six to seven tiles.  Sixteen of 256 to 1024 tokens: 112 us, 0.62 PFLOP/s
//   trees and inserted tokens over long contexts: HBM while a workgroup's rows are
//     few.  64 trees of eight nodes, four to a prefix: 662 MB in 124 us, 5.3 TB/s;
//     128 fp8 trees: the tiles' widening and products, 244 us, 0.66 PFLOP/s
//   a prompt of 17 tokens: one tile, 7.4 us
//   fp32 output at these sizes: 64 products a tile for 32, in the generic loop;
//     whole calls 1.2 to 1.9 times as long
// All 256 registers are taken, and 15 (bf16 pool and output) to 48 (fp8 pool,
// fp32 output, drafts) more lie in scratch; only the generic loop reloads them.
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
constexpr float kLazy = 8.f;  // a row's reference moves when a score exceeds it by 2^kLazy

__device__ inline uint32_t pack_bf16x2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// Scalar load of an int the launch does not write.
__device__ inline int ld_const(const int32_t* p) {
  return *reinterpret_cast<const GAMBIT_CONST int32_t*>(reinterpret_cast<uintptr_t>(p));
}

// One instruction (this source is built without IEEE mode, so the operands
// need no quieting first); a NaN operand is passed over.
__device__ inline float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

// Four direct loads of 1 KiB each, 16 bytes a lane: from base + off + 1024 k
// (base uniform, off the lane's) into LDS at l + 1024 k + 16 x lane.  An
// instruction's offset counts for both sides.  `once`: nobody else reads these
// bytes (non-temporal hint).
__device__ inline void dma16x4(const uint8_t* base, uint32_t off, uint8_t* l, bool once) {
  uint32_t save;
  const uintptr_t b = reinterpret_cast<uintptr_t>(base);
  const uint64_t sb = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32 |
                      (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
  const uint32_t at = __builtin_amdgcn_readfirstlane(lds_addr(l));
#define GAMBIT_DMA16X4(hint)                                     \
  asm volatile(                                                  \
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\t"     \
      "global_load_lds_dwordx4 %1, %2" hint "\n\t"               \
      "global_load_lds_dwordx4 %1, %2 offset:0x400" hint "\n\t"   \
      "global_load_lds_dwordx4 %1, %2 offset:0x800" hint "\n\t"   \
      "global_load_lds_dwordx4 %1, %2 offset:0xc00" hint "\n\t"   \
      "s_nop 0\n\ts_mov_b32 m0, %0"                              \
      : "=&s"(save)                                              \
      : "v"(off), "s"(sb), "s"(at)                               \
      : "memory")
  if (once)
    GAMBIT_DMA16X4(" nt");
  else
    GAMBIT_DMA16X4("");
#undef GAMBIT_DMA16X4
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ inline uint4 load16(const uint8_t* p, bool once) {
  const u32x4* x = reinterpret_cast<const u32x4*>(p);
  return __builtin_bit_cast(uint4, once ? __builtin_nontemporal_load(x) : *x);
}

// The lane, made anew: what the rare parts derive from it does not then wait for
// them in registers that the loops need (a register reloaded from memory waits
// for every direct load in flight).
__device__ inline int lane_again() {
  uint32_t m = ~0u;
  asm volatile("" : "+s"(m));
  return __builtin_amdgcn_mbcnt_hi(m, __builtin_amdgcn_mbcnt_lo(m, 0));
}

// Every load and LDS access of the wave has ended.
__device__ inline void wait_all() {
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt 0, lgkmcnt 0
  asm volatile("" ::: "memory");
}

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

// The helpers below work on pairs of bf16 and on single bits without
// comparisons: a comparison's result takes two scalar registers, and a tile's
// worth of them pushed the loop's own out of theirs.

// Bit b of x as a mask, all ones or none.
__device__ inline uint32_t bit_mask(uint32_t x, int b) { return (uint32_t)((int32_t)(x << (31 - b)) >> 31); }
__device__ inline float select(uint32_t mask, float a, float b) {
  return __uint_as_float((__float_as_uint(a) & mask) | (__float_as_uint(b) & ~mask));
}
// 0x8000 in each half that is not finite.
__device__ inline uint32_t not_finite2(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
// 0x8000 flags -> 0xffff masks.
__device__ inline uint32_t widen_flags(uint32_t f) { return (f << 1) - (f >> 15); }
// Ones (bf16) in each half that is of the kind (0: +inf, 1: -inf, 2: NaN).
__device__ inline uint32_t ones_of(uint32_t x, int kind) {
  const uint32_t z = x ^ (kind ? 0xff80ff80u : 0x7f807f80u);
  const uint32_t inf = ~(((z & 0x7fff7fffu) + 0x7fff7fffu) | z), nan = (x & 0x7fff7fffu) + 0x007f007fu;
  return (((kind == 2 ? nan : inf) & 0x80008000u) >> 15) * 0x3f80u;
}
template <class F>
__device__ inline uint4 each(uint4 x, F&& f) {
  return make_uint4(f(x.x), f(x.y), f(x.z), f(x.w));
}

// The running state of a wave's 32 rows.  Lane (half h, row n): acc[db][r] is
// O[n][32 db + 8 (r / 4) + 4 h + r % 4]; l is the half's part of the sum.
struct Rows {
  float m, l;
  f32x16 acc[4];
};

// Raw scores of a key tile: s[th][r] of lane (h, n) is row n's score of token
// 32 th + 16 (r / 8) + 8 h + r % 8.
struct Scores {
  f32x16 s[2];
};

// The factors of a tile's blocks.  fp8: in LDS, [quantity][block], one quantity
// of all four blocks read when it is needed (all 16 would stay in registers for
// the tile); bf16: the softmax scale.
struct Factors {
  const float* s;
  float c;
  template <bool FP8>
  __device__ float k(int b) const { return FP8 ? s[b] : c; }  // of the raw scores, in log2 units
  __device__ float v(int b) const { return s[4 + b]; }        // of V, its log2 and reciprocal
  __device__ float log_v(int b) const { return s[8 + b]; }
  __device__ float inv_v(int b) const { return s[12 + b]; }
};

// The operands in LDS, the lane's 16 bytes.  K is the cache's own image of each
// block ([d chunk][row]), V is [block][32 d][token half][d].  A read of either
// has lane l's bytes at 16 l modulo 256, which no bank serves twice a cycle (a
// shift of every second block by 128 bytes cost a third of the LDS cycles).
constexpr int kKBlock = kBlock * kHeadDim * 2;
__host__ __device__ constexpr int k_block_at(int b) { return b * kKBlock; }
__device__ inline int k_lane(int lane) {
  return k_block_at((lane >> 4) & 1) + (lane >> 5) * 256 + (lane & 15) * 16;
}
__device__ inline bf16x8 k_operand(const uint8_t* k, int th, int kb) {
  return *reinterpret_cast<const bf16x8*>(k + k_block_at(2 * th) + kb * 512);
}
__device__ inline bf16x8 v_operand(const uint8_t* v, int b, int db) {
  return *reinterpret_cast<const bf16x8*>(v + (b * 4 + db) * 1024);
}

// S^T of the tile whose K is at `k`.
__device__ inline void qk(const uint8_t* k, const bf16x8 (&q)[8], Scores& x) {
#pragma unroll
  for (int th = 0; th < 2; ++th) x.s[th] = f32x16{};
#pragma unroll
  for (int kb = 0; kb < 8; ++kb)
#pragma unroll
    for (int th = 0; th < 2; ++th)
      x.s[th] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(k, th, kb), q[kb], x.s[th], 0, 0, 0);
}

// The lane's largest score of the tile, scaled.
template <bool FP8>
__device__ inline float tile_max(const Scores& x, const Factors& f) {
  float mb[4];
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const f32x16& s = x.s[b / 2];
    const int o = 8 * (b % 2);
    mb[b] = max3(max3(max3(s[o], s[o + 1], s[o + 2]), s[o + 3], s[o + 4]), s[o + 5], s[o + 6]);
    mb[b] = fmaxf(mb[b], s[o + 7]);
    if constexpr (FP8) mb[b] *= f.k<FP8>(b);
  }
  const float mx = fmaxf(max3(mb[0], mb[1], mb[2]), mb[3]);
  return FP8 ? mx : mx * f.c;
}

// Moves a row's reference when a score exceeds it by more than 2^kLazy; until
// then the weights stay <= 2^kLazy and nothing is rescaled.
__device__ inline void rescale(float mx, Rows& st) {
  if (__builtin_amdgcn_ballot_w64(mx > st.m + kLazy)) {
    mx = fmaxf(mx, other_half(mx));
    const float m_new = mx > st.m + kLazy ? mx : st.m;
    const float alpha = m_new == st.m ? 1.f : __builtin_amdgcn_exp2f(st.m - m_new);
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < 4; ++db) st.acc[db] *= alpha;
    st.m = m_new;
  }
}

__device__ inline float reference(const Rows& st) { return st.m == -INFINITY ? 0.f : -st.m; }

// Weights of tokens 2 j and 2 j + 1 of the lane's eight of block b as part of
// the B operand of P.V: one bf16 plane, or (WIDE) three whose sum is the weight
// to fp32's precision; their sum goes to l.  fp8: the operand holds the weight
// times the block's V scale - in one plane by way of the exponent (nm includes
// log2 of the scale), and l takes the sums as they are, to be divided.
template <bool FP8, bool WIDE>
__device__ inline void weigh_pair(const Scores& x, int b, int j, float cb, float nm, float vs, float& l,
                                  uint32_t (&p)[WIDE ? 3 : 1][4]) {
  float u = __builtin_amdgcn_exp2f(fmaf(x.s[b / 2][8 * (b % 2) + 2 * j], cb, nm));
  float v = __builtin_amdgcn_exp2f(fmaf(x.s[b / 2][8 * (b % 2) + 2 * j + 1], cb, nm));
  if constexpr (WIDE) {
    l += u + v;
    if constexpr (FP8) u *= vs, v *= vs;
  }
  p[0][j] = pack_bf16x2(u, v);
  if constexpr (WIDE) {
#pragma unroll
    for (int k = 1; k < 3; ++k) {  // the remainders are exact
      u -= __uint_as_float(p[k - 1][j] << 16);
      v -= __uint_as_float(p[k - 1][j] & 0xffff0000u);
      p[k][j] = pack_bf16x2(u, v);
    }
  } else {
    l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, p[0][j]), bf16x2{(__bf16)1.f, (__bf16)1.f}, l, false);
  }
}

// What a block's exponents add to the scores, and what its sum counts for.
template <bool FP8, bool WIDE>
__device__ inline float shift(float nm, const Factors& f, int b) {
  return FP8 && !WIDE ? nm + f.log_v(b) : nm;
}
template <bool FP8, bool WIDE>
__device__ inline float share(float l, const Factors& f, int b) {
  return FP8 && !WIDE ? l * f.inv_v(b) : l;
}

__device__ inline bf16x8 operand(const uint32_t (&p)[4]) {
  return __builtin_bit_cast(bf16x8, make_uint4(p[0], p[1], p[2], p[3]));
}

// Keeps what makes x where it is written (sums and maxima that are used later
// otherwise sink to there, with their operands in registers until then).
__device__ inline void stay(float& x) { asm volatile("" : "+v"(x)); }

// A tile that every row of the wave sees whole (scores x), and with it the
// scores y of the next tile.  A wave issues in order and a matrix product
// holds up only what needs its result, so the order is written out: between
// two products the vector units take one step each of two tokens' weights -
// the exponents of a pair, the exponentials of the pair before, the rounding of
// the one before that, its sum - while Q.K of the next tile runs, and a part of
// the next tile's maximum while P.V runs; nothing waits for the instruction in
// front of it, and an operand is read from LDS kAhead products before its use.
template <bool FP8>
__device__ inline void plain_tile(const uint8_t* v, const uint8_t* k_next, const bf16x8 (&q)[8], const Factors& f,
                                  const Factors& f_next, const Scores& x, Scores& y, float& mx, Rows& st) {
  constexpr int kAhead = 6;
  const float nm = reference(st);
  float cb[4], nb[4], l[4] = {0.f, 0.f, 0.f, 0.f}, mb[4];
  uint32_t p[4][4];
  float arg[2][2], e[2][2];  // by pair, every second one at the same place
  bf16x8 ring[kAhead];
  auto load = [&](int n) { return n < 16 ? k_operand(k_next, n % 2, n / 2) : v_operand(v, (n - 16) / 4, n % 4); };
  auto args = [&](int j) {
    const int b = j / 4, o = 8 * (b % 2) + 2 * (j % 4);
    arg[j % 2][0] = fmaf(x.s[b / 2][o], cb[b], nb[b]);
    arg[j % 2][1] = fmaf(x.s[b / 2][o + 1], cb[b], nb[b]);
    stay(arg[j % 2][0]);
    stay(arg[j % 2][1]);
  };
  f32x4 inv = {1.f, 1.f, 1.f, 1.f};
  if constexpr (FP8) {
    const f32x4 fk = *reinterpret_cast<const f32x4*>(f.s), fl = *reinterpret_cast<const f32x4*>(f.s + 8);
#pragma unroll
    for (int b = 0; b < 4; ++b) cb[b] = fk[b], nb[b] = nm + fl[b];
  } else {
#pragma unroll
    for (int b = 0; b < 4; ++b) cb[b] = f.c, nb[b] = nm;
  }
#pragma unroll
  for (int n = 0; n < kAhead; ++n) ring[n] = load(n);
  args(0);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int n = 0; n < 32; ++n) {
    if (n < 16)
      y.s[n % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[n % kAhead], q[n / 2], n < 2 ? f32x16{} : y.s[n % 2], 0, 0, 0);
    else
      st.acc[n % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[n % kAhead], operand(p[n / 4 - 4]), st.acc[n % 4], 0, 0, 0);
    if (n < 16) {
      e[n % 2][0] = __builtin_amdgcn_exp2f(arg[n % 2][0]);
      e[n % 2][1] = __builtin_amdgcn_exp2f(arg[n % 2][1]);
      stay(e[n % 2][0]);
      stay(e[n % 2][1]);
    }
    if (n < 15) args(n + 1);
    if (n >= 1 && n < 17) p[(n - 1) / 4][(n - 1) % 4] = pack_bf16x2(e[(n - 1) % 2][0], e[(n - 1) % 2][1]);
    if (n >= 2 && n < 18) {
      const int b = (n - 2) / 4;
      l[b] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, p[b][(n - 2) % 4]),
                                             bf16x2{(__bf16)1.f, (__bf16)1.f}, l[b], false);
      stay(l[b]);
    }
    if (FP8 && n == 16) inv = *reinterpret_cast<const f32x4*>(f.s + 12);
    if (n >= 28) st.l = FP8 ? fmaf(l[n - 28], inv[n - 28], st.l) : st.l + l[n - 28];
    if (n >= 20 && n < 28) {  // y's four blocks, four scores a time
      const int b = n % 4, o = 8 * (b % 2) + 4 * (n / 4 - 5);
      const f32x16& s = y.s[b / 2];
      mb[b] = n < 24 ? fmaxf(max3(s[o], s[o + 1], s[o + 2]), s[o + 3]) : max3(max3(mb[b], s[o], s[o + 1]), s[o + 2], s[o + 3]);
      stay(mb[b]);
    }
    if (n + kAhead < 32) ring[n % kAhead] = load(n + kAhead);
    __builtin_amdgcn_sched_barrier(0);
  }
  if constexpr (FP8) {
    const f32x4 fk = *reinterpret_cast<const f32x4*>(f_next.s);
#pragma unroll
    for (int b = 0; b < 4; ++b) mb[b] *= fk[b];
  }
  mx = fmaxf(max3(mb[0], mb[1], mb[2]), mb[3]);
  if constexpr (!FP8) mx *= f.c;
}

// Adds the values of one kind (0: +inf, 1: -inf, 2: NaN) in a block's V to the
// rows that see them, whatever their weights: the product of `seen`, ones where
// the row sees the token, with ones where the values are.
__device__ inline void add_not_finite(const uint4 (&v)[4], bf16x8 seen, int kind, Rows& st) {
  const uint32_t what = kind == 2 ? 0x7fc00000u : kind ? 0xff800000u : 0x7f800000u;
#pragma unroll
  for (int db = 0; db < 4; ++db) {
    const uint4 a = each(v[db], [&](uint32_t x) { return ones_of(x, kind); });
    const f32x16 n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), seen, f32x16{}, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      uint32_t add = what & (uint32_t)(-__float_as_int(n[r]) >> 31);  // where the row sees one
      asm("" : "+v"(add));  // the source's arithmetic is compiled as if NaN did not occur
      st.acc[db][r] += __uint_as_float(add);
    }
  }
}

// Scores of tokens that the lane's row does not see (bits of `vis`) become -inf.
__device__ inline void mask_scores(uint64_t vis, int lane, Scores& x) {
  const uint32_t v0 = (uint32_t)vis >> (8 * (lane >> 5)), v1 = (uint32_t)(vis >> 32) >> (8 * (lane >> 5));
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int bit = 16 * (r / 8) + r % 8;
    x.s[0][r] = select(bit_mask(v0, bit), x.s[0][r], -INFINITY);
    x.s[1][r] = select(bit_mask(v1, bit), x.s[1][r], -INFINITY);
  }
}

// A tile without one behind it (WIDE: any): the weights of a block are made
// between the products of the block before.
template <bool FP8, bool WIDE>
__device__ inline void last_tile(const uint8_t* v, const Factors& f, const Scores& x, Rows& st) {
  constexpr int kAhead = 6, kPlanes = WIDE ? 3 : 1;
  const float nm = reference(st);
  float l[4] = {0.f, 0.f, 0.f, 0.f};
  uint32_t p[2][kPlanes][4];
  bf16x8 ring[kAhead];
#pragma unroll
  for (int n = 0; n < kAhead; ++n) ring[n] = v_operand(v, n / 4, n % 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) weigh_pair<FP8, WIDE>(x, 0, j, f.k<FP8>(0), shift<FP8, WIDE>(nm, f, 0), FP8 ? f.v(0) : 1.f, l[0], p[0]);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int n = 0; n < 16; ++n) {
    const int b = n / 4;
#pragma unroll
    for (int k = kPlanes - 1; k >= 0; --k)
      st.acc[n % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[n % kAhead], operand(p[b % 2][k]), st.acc[n % 4], 0, 0, 0);
    if (b < 3) {
      weigh_pair<FP8, WIDE>(x, b + 1, n % 4, f.k<FP8>(b + 1), shift<FP8, WIDE>(nm, f, b + 1), FP8 ? f.v(b + 1) : 1.f, l[b + 1],
                            p[(b + 1) % 2]);
      stay(l[b + 1]);
    }
    if (n + kAhead < 16) ring[n % kAhead] = v_operand(v, (n + kAhead) / 4, (n + kAhead) % 4);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int b = 0; b < 4; ++b) st.l += share<FP8, WIDE>(l[b], f, b);
}

// The same for a tile whose V holds infinities or NaN that not every row sees:
// where a row's weight is zero the product would make them NaN, so they are
// zeros in the product and go to the rows that see them (bits of `vis`) beside it.
template <bool FP8, bool WIDE>
__device__ inline void slow_tile(const uint8_t* vt, const Factors& f, const Scores& x, uint64_t vis, int lane, Rows& st) {
  const float nm = reference(st);
  vis >>= 8 * (lane >> 5);
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    uint32_t p[WIDE ? 3 : 1][4];
    float l = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      weigh_pair<FP8, WIDE>(x, b, j, f.k<FP8>(b), shift<FP8, WIDE>(nm, f, b), FP8 ? f.v(b) : 1.f, l, p);
    st.l += share<FP8, WIDE>(l, f, b);
    uint4 v[4];
#pragma unroll
    for (int db = 0; db < 4; ++db) v[db] = __builtin_bit_cast(uint4, v_operand(vt, b, db));
    uint32_t seen[4];  // ones (bf16) of the lane's eight tokens
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t two = (uint32_t)(vis >> (16 * b + 2 * j));
      seen[j] = (two & 1) * 0x3f80u | (two >> 1 & 1) * 0x3f800000u;
    }
#pragma unroll 1
    for (int kind = 0; kind < 3; ++kind) add_not_finite(v, operand(seen), kind, st);
#pragma unroll
    for (int db = 0; db < 4; ++db) {
      v[db] = each(v[db], [](uint32_t y) { return y & ~widen_flags(not_finite2(y)); });
#pragma unroll
      for (int k = WIDE ? 2 : 0; k >= 0; --k)
        st.acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[db]), operand(p[k]), st.acc[db], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);  // one block's operands at a time
  }
}

// The drafts of a trace as a key tile in LDS: tokens in rows there, so V is
// turned on the way.  Tokens past the tree are zeros.  Returns whether the
// thread's part of V holds infinities or NaN.
__device__ inline uint32_t stage_drafts(const RowsLaunch& A, const RowItem& U, int Hkv, int kvh, int t, uint8_t* kst,
                                        uint8_t* vst) {
  uint32_t bad = 0;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int u = t + x * kThreads, j = u >> 4, ch = u & 15;
    uint4 k = make_uint4(0, 0, 0, 0);
    if (j < U.ndraft)
      k = *reinterpret_cast<const uint4*>(A.k_new + ((size_t)(U.draft + j) * Hkv + kvh) * kHeadDim + 8 * ch);
    *reinterpret_cast<uint4*>(kst + k_block_at(j >> 4) + ch * 256 + k_phys(j & 15) * 16) = k;
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int u = t + x * kThreads, d = u & 127, j0 = (u >> 7) * 8;  // eight tokens of one d
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (j0 + e < U.ndraft)
        w[e / 2] |= (uint32_t)A.v_new[((size_t)(U.draft + j0 + e) * Hkv + kvh) * kHeadDim + d] << (16 * (e % 2));
    *reinterpret_cast<uint4*>(vst + (j0 >> 4) * 4096 + (d >> 5) * 1024 + ((j0 >> 3) & 1) * 512 + (d & 31) * 16) =
        make_uint4(w[0], w[1], w[2], w[3]);
    bad |= not_finite2(w[0]) | not_finite2(w[1]) | not_finite2(w[2]) | not_finite2(w[3]);
  }
  return bad;
}

// A wave's rows times `inv` to their places (`at`: row lane % 32's), fp32 or bf16,
// turned in the wave's part of LDS.  What would be rows past the last one stores
// that one again.
template <class T>
__device__ inline void store_rows(uint8_t* rows, const Rows& st, float inv, T* out, uint32_t at, int last, int lane) {
  constexpr int kLanes = kHeadDim * sizeof(T) / 16, kPer = 64 / kLanes;  // lanes a row, rows an instruction stores
  constexpr int kSteps = 32 / kPer;
  const int n = lane & 31, h = lane >> 5, c = lane % kLanes;
  auto row = [&](int k) { return min(k * kPer + lane / kLanes, last); };
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 v = {st.acc[db][4 * j] * inv, st.acc[db][4 * j + 1] * inv, st.acc[db][4 * j + 2] * inv,
                       st.acc[db][4 * j + 3] * inv};
      if constexpr (sizeof(T) == 4)
        *reinterpret_cast<f32x4*>(rows + n * 512 + ((8 * db + 2 * j + h) ^ n) * 16) = v;
      else
        *reinterpret_cast<uint2*>(rows + n * 256 + ((4 * db + j) ^ (n & 15)) * 16 + 8 * h) =
            make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
  wait_all();
  uint4 v[kSteps];
  uint32_t to[kSteps];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    v[k] = *reinterpret_cast<const uint4*>(rows + (row(k) * kLanes + (c ^ (row(k) % kLanes))) * 16);
    to[k] = __shfl(at, row(k));
  }
#pragma unroll
  for (int k = 0; k < kSteps; ++k) reinterpret_cast<uint4*>(out)[(size_t)to[k] * kLanes + c] = v[k];
}

constexpr int kRowBytes = kHeadDim * 2;  // of a query
constexpr int kKTile = k_block_at(4), kVTile = kKeyTile * kHeadDim * 2;  // of a key tile in LDS

template <bool FP8, bool WIDE, bool DRAFT>
__global__ __launch_bounds__(kThreads, 2) void rows_attn_kernel(DevPool P, RowsLaunch A) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kKTile + 2 * kVTile];
  __shared__ __attribute__((aligned(16))) float scale_s[3][4][4];
  __shared__ uint32_t bad_s[2][4];  // by tile and wave: its block's V is not all finite
  // the quotient in a scalar register, so that what it leads to is read by scalar loads
  const int item = __builtin_amdgcn_readfirstlane(blockIdx.x / P.Hkv), kvh = blockIdx.x - item * P.Hkv;
  const RowItem U = __builtin_bit_cast(
      RowItem, *reinterpret_cast<const GAMBIT_CONST i32x16*>(reinterpret_cast<uintptr_t>(A.items + item)));
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int h = lane >> 5, gs = A.gshift;
  const int nrows = U.ntok << gs;
  // the packed token of a row
  auto token = [&](int row) {
    const int j = U.tok + (row >> gs);
    return U.listed ? A.list[j] : j;
  };

  // positions that a row sees, and the fewest and most that one of the wave does
  const int t0 = kBlock * U.jb0;
  auto limit = [&](int r) { return U.pos0 == kNoLimit ? U.end : min(U.end, U.pos0 + (r >> gs) + 1); };
  const bool active = 32 * w < nrows;
  const int lim_lo = limit(32 * w), lim_hi = limit(min(32 * w + 31, nrows - 1));
  const int ntiles = U.end > t0 ? (U.end - t0 + kKeyTile - 1) / kKeyTile : 0;
  // tiles of which the wave sees something
  const int nt = active && lim_hi > t0 ? (lim_hi - t0 + kKeyTile - 1) / kKeyTile : 0;
  const int jlast = (U.end - 1) / kBlock;
  const int32_t* brow = P.table + (size_t)U.trace * P.max_blocks;
  const size_t tile_bytes = (size_t)kBlock * kHeadDim * (FP8 ? 1 : 2);

  // Wave w moves block w of a tile.  Its id is asked for a tile ahead of its bytes.
  auto id_of = [&](int i, int b) { return ld_const(brow + min(U.jb0 + 4 * i + b, jlast)); };
  bool bad_id = false;
  auto checked = [&](int id) {
    const bool in = (unsigned)id < (unsigned)P.num_blocks;
    bad_id |= !in;
    return in ? id : 0;
  };
  auto block_at = [&](const uint8_t* cache, int id) { return cache + ((size_t)id * P.Hkv + kvh) * tile_bytes; };
  auto kbuf = [&](int i) { return lds + (i & 1) * kKTile; };
  auto vbuf = [&](int i) { return lds + 2 * kKTile + (i & 1) * kVTile; };
  uint4 raw_k[2], raw_v[2];  // fp8: the codes on their way,
  float raw_scale = 0.f;     // and the block's K scale (lane 0) and V scale (lanes 1 to 3)
  auto ask_k = [&](int id, int i, int lane) {
    const uint8_t* src = block_at(P.k_cache, id);
    if constexpr (FP8) {
      raw_k[0] = load16(src + lane * 16, U.once);
      raw_k[1] = load16(src + lane * 16 + 1024, U.once);
      raw_scale = P.kv_scale[2 * (size_t)id + min(lane, 1)];
    } else {
      dma16x4(src, lane * 16, kbuf(i) + k_block_at(w), U.once);
    }
  };
  auto ask_v = [&](int id, int i, int lane) {
    const uint8_t* src = block_at(P.v_cache, id);
    if constexpr (FP8) {
      raw_v[0] = load16(src + lane * 16, U.once);
      raw_v[1] = load16(src + lane * 16 + 1024, U.once);
    } else {
      dma16x4(src, (2 * (lane & 31) + (lane >> 5)) * 16, vbuf(i) + w * kKBlock, U.once);
    }
  };
  auto widen_k = [&](int i, int lane) {  // 16 d of a row -> two chunks of 8
    // lane 0: K's with the softmax scale; lanes 1 to 3: V's, its log2, its reciprocal
    // (bf16 output; instructions of one ulp, at most 2^-17 of a weight that is
    // rounded to bf16 next; fp32 output takes the scale itself)
    const float x = fmaxf(lane ? raw_scale : A.c * raw_scale, lane ? 0x1p-100f : 0x1p-120f);
    const float y = lane == 2 ? __builtin_amdgcn_logf(x) : lane == 3 ? __builtin_amdgcn_rcpf(x) : x;
    if (lane < 4) scale_s[i % 3][lane][w] = y;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      uint8_t* k = kbuf(i) + k_block_at(w) + (2 * (4 * y + (lane >> 4)) * kBlock + (lane & 15)) * 16;
      *reinterpret_cast<uint4*>(k) = widen8(raw_k[y].x, raw_k[y].y);
      *reinterpret_cast<uint4*>(k + kBlock * 16) = widen8(raw_k[y].z, raw_k[y].w);
    }
  };
  auto widen_v = [&](int i, int lane) {  // 16 tokens of a d -> two halves
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      uint8_t* v = vbuf(i) + w * kKBlock + (2 * y + (lane >> 5)) * 1024 + (lane & 31) * 16;
      *reinterpret_cast<uint4*>(v) = widen8(raw_v[y].x, raw_v[y].y);
      *reinterpret_cast<uint4*>(v + 512) = widen8(raw_v[y].z, raw_v[y].w);
    }
  };
  // fp8: the scales of a tile's blocks, put into LDS by the wave that moves the
  // block when it settles the tile's K, two tiles ahead (so three places).
  auto factors = [&](int i) { return Factors{scale_s[i % 3][0], A.c}; };

  // the first loads: tile 0's K, then the queries, tile 0's V and tile 1's K
  int id0 = 0, id1 = 0, id2 = 0;  // wave's blocks of tiles i, i + 1, i + 2 (past the end: the last block, unused)
  if (ntiles > 0) {
    id0 = checked(w < 2 ? (w ? U.first[1] : U.first[0]) : (w > 2 ? U.first[3] : U.first[2]));
    ask_k(id0, 0, lane);
    id1 = id_of(1, w);
  }
  // The wave's queries by way of LDS (V's place), so that whole rows are read:
  // row r's 16-byte chunk c at place c ^ (r % 16).
  uint8_t* mine = lds + 2 * kKTile + w * 32 * kRowBytes;
  if (active) {
    int rt[8];  // rows past the last one read that one again
    auto place = [&](int k) { return min(32 * w + 4 * k + (lane >> 4), nrows - 1); };
#pragma unroll
    for (int k = 0; k < 8; ++k) rt[k] = U.tok + (place(k) >> gs);
    if (U.listed) {
#pragma unroll
      for (int k = 0; k < 8; ++k) rt[k] = A.list[rt[k]];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const size_t at = (size_t)rt[k] * P.Hq + (kvh << gs) + (place(k) & ((1 << gs) - 1));
      dma16(A.q + at * kHeadDim + 8 * ((lane & 15) ^ ((4 * k + (lane >> 4)) & 15)), mine + k * 1024);
    }
  }
  id1 = checked(id1);
  wait_all();
  bf16x8 q[8];
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) {
    uint4 x = *reinterpret_cast<const uint4*>(mine + (lane & 31) * kRowBytes + (((2 * kb + h) ^ (lane & 15)) * 16));
    q[kb] = __builtin_bit_cast(bf16x8, each(x, [&](uint32_t y) { return (y & A.q_and) ^ A.q_xor; }));
  }
  Rows st;
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db) st.acc[db] = f32x16{};
  Scores x, y;
  float mx = -INFINITY;
  if (ntiles > 0) {
    if constexpr (FP8) widen_k(0, lane);
    wait_all();
    barrier_no_fence();
    ask_v(id0, 0, lane);
    if (ntiles > 1) ask_k(id1, 1, lane);
    id2 = id_of(2, w);
    if (nt > 0) {
      qk(kbuf(0) + k_lane(lane), q, x);
      mx = tile_max<FP8>(x, factors(0));
    }
    if constexpr (FP8) {
      widen_v(0, lane);
      if (ntiles > 1) widen_k(1, lane);
    }
  }
  // A tile that ends the range, or that not every row of the workgroup sees
  // whole: its tokens past the end hold anything, and become zeros in V (their
  // weights are zero); bad_s says whether the others hold infinities or NaN.
  const int lim_wg = limit(0);
  auto clean_v = [&](int i) {
    const int lane = lane_again(), h = lane >> 5;
    uint8_t* v = vbuf(i) + w * kKBlock + lane * 16;
    const int n = min(max(U.end - (t0 + kKeyTile * i + kBlock * w + 8 * h), 0), 8);
    const uint32_t there = (1u << n) - 1;
    const uint4 keep = make_uint4((bit_mask(there, 0) & 0xffffu) | (bit_mask(there, 1) & 0xffff0000u),
                                  (bit_mask(there, 2) & 0xffffu) | (bit_mask(there, 3) & 0xffff0000u),
                                  (bit_mask(there, 4) & 0xffffu) | (bit_mask(there, 5) & 0xffff0000u),
                                  (bit_mask(there, 6) & 0xffffu) | (bit_mask(there, 7) & 0xffff0000u));
    uint32_t bad = 0;
#pragma unroll
    for (int db = 0; db < 4; ++db) {
      uint4* at = reinterpret_cast<uint4*>(v + db * 1024);
      const uint4 x = *at, y = make_uint4(x.x & keep.x, x.y & keep.y, x.z & keep.z, x.w & keep.w);
      bad |= not_finite2(y.x) | not_finite2(y.y) | not_finite2(y.z) | not_finite2(y.w);
      *at = y;
    }
    const uint64_t any = __builtin_amdgcn_ballot_w64(bad != 0);
    if (lane == 0) bad_s[i & 1][w] = any != 0;
  };
  auto settle = [&](int i) {
    const bool check = t0 + kKeyTile * (i + 1) > lim_wg;  // uniform over the workgroup
    if (check) {
      wait_all();
      clean_v(i);
    }
    return check;
  };
  auto is_bad = [&](int i) {
    return __builtin_amdgcn_readfirstlane(bad_s[i & 1][0] | bad_s[i & 1][1] | bad_s[i & 1][2] | bad_s[i & 1][3]) != 0;
  };
  // Start of tile i: its V and the K of tile i + 1 are there in every wave, and
  // no wave reads its K or the V of tile i - 1 any more; the next ones are asked for.
  auto begin = [&](int i, int lane) {
    wait_all();
    barrier_no_fence();
    id2 = checked(id2);
    if (i + 2 < ntiles) ask_k(id2, i + 2, lane);
    if (i + 1 < ntiles) ask_v(id1, i + 1, lane);
    id1 = id2;
    id2 = id_of(i + 3, w);
  };
  auto end = [&](int i, int lane) {
    if constexpr (FP8) {
      if (i + 2 < ntiles) widen_k(i + 2, lane);
      if (i + 1 < ntiles) widen_v(i + 1, lane);
    }
  };
  auto plain = [&](int i, int lane, const Scores& a, Scores& b) {
    rescale(mx, st);
    plain_tile<FP8>(vbuf(i) + lane * 16, kbuf(i + 1) + k_lane(lane), q, factors(i), factors(i + 1), a, b, mx, st);
  };
  int i = 0;
  if (nt == 0) {
    // The wave's rows see nothing here: it moves its blocks for the others, in a
    // loop in which nothing else is held in registers.
#pragma unroll 1
    for (; i < ntiles; ++i) {
      settle(i);
      begin(i, lane);
      end(i, lane);
    }
  }
  if constexpr (!WIDE) {
    // tiles that every row of the workgroup sees whole, before the wave's last
    const int np = min(lim_wg > t0 ? (lim_wg - t0) / kKeyTile : 0, nt - 1);
#pragma unroll 1
    for (; i + 1 < np; i += 2) {
      begin(i, lane);
      plain(i, lane, x, y);
      end(i, lane);
      begin(i + 1, lane);
      plain(i + 1, lane, y, x);
      end(i + 1, lane);
    }
  }
#pragma unroll 1
  for (; i < ntiles; ++i) {
    const int tb = t0 + kKeyTile * i;
    const bool check = settle(i);
    const int lane = lane_again();
    begin(i, lane);
    auto seen = [&](int lane) {  // tokens of the tile that the lane's row sees
      const int lim = limit(min(32 * w + (lane & 31), nrows - 1));
      return lim - tb <= 0 ? 0 : ~0ull >> (64 - min(lim - tb, 64));
    };
    if (i < nt) {
      if (tb + kKeyTile > lim_lo) {
        mask_scores(seen(lane), lane, x);
        mx = tile_max<FP8>(x, factors(i));
      }
      const bool more = i + 1 < nt;
      if (check && is_bad(i)) {
        rescale(mx, st);
        const int lane = lane_again();
        slow_tile<FP8, WIDE>(vbuf(i) + lane * 16, factors(i), x, seen(lane), lane, st);
      } else if (!WIDE && more) {
        if constexpr (!WIDE) plain(i, lane, x, y);
        x = y;
      } else {
        rescale(mx, st);
        last_tile<FP8, WIDE>(vbuf(i) + lane * 16, factors(i), x, st);
      }
      if (more && (WIDE || (check && is_bad(i)))) {
        qk(kbuf(i + 1) + k_lane(lane), q, x);
        mx = tile_max<FP8>(x, factors(i + 1));
      }
    }
    end(i, lane);
  }
  if constexpr (DRAFT) {
    if (U.draft >= 0) {  // uniform
      __syncthreads();   // the last tile is read
      const uint32_t bad = stage_drafts(A, U, P.Hkv, kvh, t, kbuf(0), vbuf(0));
      const uint64_t any = __builtin_amdgcn_ballot_w64(bad != 0);
      if (lane == 0) bad_s[0][w] = any != 0;
      if (FP8 && t < 16) scale_s[0][t >> 2][t & 3] = t < 4 ? A.c : t >> 2 == 2 ? 0.f : 1.f;  // the drafts are bf16
      __syncthreads();
      if (active) {
        const Factors one = factors(0);
        qk(kbuf(0) + k_lane(lane), q, x);
        auto seen = [&](int lane) {  // a tree's rows are not listed
          const int row = 32 * w + (lane & 31);
          return row < nrows ? A.anc[U.tok + (row >> gs)] : 1;
        };
        const int lane = lane_again();
        mask_scores(seen(lane), lane, x);
        rescale(tile_max<FP8>(x, one), st);
        if (is_bad(0))
          slow_tile<FP8, WIDE>(vbuf(0) + lane * 16, one, x, seen(lane), lane, st);
        else
          last_tile<FP8, WIDE>(vbuf(0) + lane * 16, one, x, st);
      }
    }
  }
  if (bad_id && lane == 0) atomicOr(P.err, kErrBadBlock);
  // Rows leave by way of LDS, whole ones at a time: a row's 16-byte chunk c at
  // place c ^ (row % chunks), a wave's rows in its own part.
  const float l = st.l + other_half(st.l);
  const bool part = U.kidx >= 0;  // uniform
  const int again = lane_again(), row = 32 * w + (again & 31);
  uint32_t at = 0;  // the row's place in the output or among the partials
  if (row < nrows) {
    const int tok = token(row);
    at = (uint32_t)(part ? A.off[tok] + U.kidx : tok) * P.Hq + (kvh << gs) + (row & ((1 << gs) - 1));
    if (part && again < 32) A.part_ml[at] = float2{st.m, l};
  }
  __syncthreads();  // no wave reads K or V any more
  if (!active) return;
  const float inv = part ? 1.f : 1.f / l;
  if (WIDE || part)
    store_rows<float>(lds + w * 16384, st, inv, part ? A.part_acc : static_cast<float*>(A.out), at, min(31, nrows - 1 - 32 * w), again);
  else
    store_rows<uint16_t>(lds + w * 8192, st, inv, static_cast<uint16_t*>(A.out), at, min(31, nrows - 1 - 32 * w), again);
}

// out = sum_k 2^(m_k - M) acc_k / sum_k 2^(m_k - M) l_k, M the largest m_k;
// eight rows a workgroup, a half-wave a row, four d a lane.  Each lane takes the
// factors of every 32nd partial, four partials' rows are asked for at a time.
// A partial without a seen position has m = -inf and sums of zero.  A factor of
// zero still meets the partial's sums: where a V that its rows see is not finite
// they are not, and so is the result, as in a range that was not cut.
// Bound by HBM, for few partials by latency: 4 us for 40 tokens of 32 heads, 7
// for 512, 22 for 1120 of 64 heads.
__global__ __launch_bounds__(256) void rows_merge_kernel(RowsLaunch A, int32_t Hq) {
  const int r = blockIdx.x * 8 + (threadIdx.x >> 5), x = threadIdx.x & 31;
  if (r >= A.n_merge * Hq) return;
  const int tok = A.merge[r / Hq], head = r % Hq;
  const int n = A.nk[tok];
  const size_t p0 = (size_t)A.off[tok] * Hq + head;
  float M = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < n; k0 += 32) {
    const float2 ml = k0 + x < n ? A.part_ml[p0 + (size_t)(k0 + x) * Hq] : float2{-INFINITY, 0.f};
    float most = fmaxf(M, ml.x);
#pragma unroll
    for (int s = 16; s; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
    if (most != M) {  // uniform over the half-wave
      const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - most);
      l *= f;
      o *= f;
      M = most;
    }
    const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    float sum = f * ml.y;
#pragma unroll
    for (int s = 16; s; s >>= 1) sum += __shfl_xor(sum, s);
    l += sum;
    const int m = min(32, n - k0);
    for (int k = 0; k < m; k += 4) {
      f32x4 a[4];
#pragma unroll
      for (int y = 0; y < 4; ++y)
        a[y] = *reinterpret_cast<const f32x4*>(A.part_acc + (p0 + (size_t)(k0 + min(k + y, m - 1)) * Hq) * kHeadDim + 4 * x);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float g = __shfl(f, (threadIdx.x & 32) + k + y);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = k + y < m ? fmaf(g, a[y][e], o[e]) : o[e];
      }
    }
  }
  const float inv = 1.f / l;
  const size_t at = ((size_t)tok * Hq + head) * kHeadDim + 4 * x;
  if (A.out_f32)
    *reinterpret_cast<f32x4*>(static_cast<float*>(A.out) + at) = f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(A.out) + at) =
        make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
}

template <bool FP8, bool WIDE>
void launch_items(const DevPool& P, const RowsLaunch& L, hipStream_t s) {
  const dim3 grid((unsigned)L.n_items * P.Hkv);
  if (L.anc)
    hipLaunchKernelGGL((rows_attn_kernel<FP8, WIDE, true>), grid, dim3(kThreads), 0, s, P, L);
  else
    hipLaunchKernelGGL((rows_attn_kernel<FP8, WIDE, false>), grid, dim3(kThreads), 0, s, P, L);
}

}  // namespace

hipError_t launch_rows_attention(const DevPool& P, const RowsLaunch& L, hipStream_t s) {
  if (L.n_items <= 0) return hipSuccess;
  const bool fp8 = P.esize == 1, wide = L.out_f32;
  if (fp8 && wide) launch_items<true, true>(P, L, s);
  if (fp8 && !wide) launch_items<true, false>(P, L, s);
  if (!fp8 && wide) launch_items<false, true>(P, L, s);
  if (!fp8 && !wide) launch_items<false, false>(P, L, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || L.n_merge == 0) return e;
  hipLaunchKernelGGL(rows_merge_kernel, dim3(((unsigned)L.n_merge * P.Hq + 7) / 8), dim3(256), 0, s, L, P.Hq);
  return hipGetLastError();
}

}  // namespace gambit
