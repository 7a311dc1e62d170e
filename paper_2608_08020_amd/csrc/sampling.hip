// One token a row of logits from a given random number (gambit_sample),
// kernel and host entry point.
//
//     w_i = 2^((z_i - max z) log2(e) / T)
//     kept: the top_k largest (of equal ones the lower index); of those the
//           shortest front part, largest first, whose weight reaches top_p of
//           theirs; of those the ones with w_i >= min_p
//     token: the first kept one, by index, up to which the kept weights' sum
//            exceeds u times their whole sum
//
// Weights are whole numbers, round(2^S w_i) with S = 62 - log2 of the row's
// length (44 for the longest rows): sums are exact whatever their order, so a
// row's token depends on its inputs alone, and the atomics below change
// nothing.  w is computed in fp64 to 2^-50 (a table of 64 powers and a
// polynomial of degree 5), because a token is one of many neighbours on the
// line from 0 to 1, and an error of fp32's size there would give another one
// in every few thousand draws.
//
// One workgroup a row goes over it as often as the filters ask: the maximum;
// with a filter, a histogram of the weights by 64ths of an octave, sixteen
// octaves at a time from the maximum down, and the row's whole weight; the
// values of the bin where the filter's border falls, listed and sorted in LDS,
// together with the kept weight of every 64 loads of the row; then the 64
// loads that the token is among.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>
#include <cstdint>

#include "../../include/gambit.h"
#include "fp8_codes.h"
#include "kernels.h"

namespace gambit {
namespace {

constexpr int kMaxVocab = 1 << 18;
constexpr int kThreads = 1024;
constexpr int kBins = 1024, kBinsPerOctave = 64;  // a histogram's window: 16 octaves
constexpr int kList = 4096;                       // listed values of one bin
constexpr int kSegs = kMaxVocab / 4 / 64 + 1;     // 64 loads (a wave's) of 16 bytes each; rows may start inside one

struct SampleArgs {
  const void* z;
  int64_t stride;  // values between rows
  int32_t vocab;
  int32_t scale_bits;  // S
  const float* u;
  const float* temperature;  // [n], or null: t_all for every row; the others alike
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  float t_all, p_all, m_all;
  int32_t k_all;
  int32_t* out;
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

  __device__ Row(const void* z, int64_t at, int vocab_) : vocab(vocab_) {
    const uint8_t* p = static_cast<const uint8_t*>(z) + at * (kF32 ? 4 : 2);
    lead = (int)(reinterpret_cast<uintptr_t>(p) & 15) / (kF32 ? 4 : 2);
    base = p - (reinterpret_cast<uintptr_t>(p) & 15);
    loads = (lead + vocab + kPer - 1) / kPer;
  }
  // NaN counts as -inf, +inf as the largest finite value, -0 as 0.
  __device__ static float clean(float x) { return x == x ? fminf(x, FLT_MAX) + 0.f : -INFINITY; }
  __device__ int index(int load, int i) const { return load * kPer + i - lead; }
  // The values of a load; places outside the row are not read and count as -inf.
  __device__ void get(int load, float* z) const {
    const uint8_t* p = base + (size_t)load * 16;
    const int first = index(load, 0);
    if (first >= 0 && first + kPer <= vocab) {
      const uint4 a = *reinterpret_cast<const uint4*>(p);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (kF32) {
          z[i] = clean(__uint_as_float(w[i]));
        } else {
          z[2 * i] = clean(bf16_lo(w[i]));
          z[2 * i + 1] = clean(bf16_hi(w[i]));
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        z[i] = -INFINITY;
        if (first + i < 0 || first + i >= vocab) continue;
        if constexpr (kF32)
          z[i] = clean(reinterpret_cast<const float*>(p)[i]);
        else
          z[i] = clean(__uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16));
      }
    }
  }
};

struct Shared {
  unsigned long long mass[kBins];
  uint32_t count[kBins];
  unsigned long long list[kList];  // ~key, index: ascending is likeliest first
  unsigned long long segs[kSegs + 1];
  double power[64];
  unsigned long long wave_sum[kThreads / 64];
  unsigned long long found_mass, rest;
  uint32_t wave_max[kThreads / 64];
  uint32_t found, found_count, listed, key_lo, key_hi, token;
};

// What the kept values have at least: a key, and of equal ones an index at most.
struct Cut {
  uint32_t key, index;
};

template <bool kF32>
struct Sampler {
  Shared& L;
  const Row<kF32> row;
  static constexpr int kPer = Row<kF32>::kPer;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  float top = 0.f;         // the row's maximum
  double slope = 0.;       // log2(e) / T
  float bin_slope = 0.f;
  double least = -INFINITY;  // log2 of min_p
  int bits;                // S
  unsigned long long total = 0;  // weight of all values
  int window = -1;         // the histogram's

  // log2 of a weight
  __device__ double octaves(float z) const { return ((double)z - (double)top) * slope; }
  // round(2^S w); 0 below half a unit (NaN: of -inf at an infinite temperature)
  __device__ unsigned long long weight(double x) const {
    if (!(x >= -(double)(bits + 1))) return 0;
    constexpr double kShift = 0x1.8p46;  // its last bit is 1/64
    const double y = x + kShift, r = x - (y - kShift);
    const int q = (int)__double_as_longlong(y);
    double p = fma(r, 1.3333558146428443e-3, 9.6181291076284772e-3);  // ln(2)^n / n!
    p = fma(r, p, 5.5504108664821580e-2);
    p = fma(r, p, 2.4022650695910071e-1);
    p = fma(r, p, 6.9314718055994531e-1);
    p = fma(r, p, 1.0);
    p = ldexp(p * L.power[q & 63], (q >> 6) + bits) + 0x1p52;
    return (unsigned long long)__double_as_longlong(p) - 0x4330000000000000ull;
  }
  // Bin of a value, from the maximum down; a huge one for -inf.
  __device__ int bin(float z) const {
    return z > -INFINITY ? (int)fminf(fminf(top - z, FLT_MAX) * bin_slope, 0x1p30f) : 0x7fffffff;
  }
  __device__ bool in(const Cut& c, float z, int index) const {
    const uint32_t k = key_of(z);
    return k > c.key || (k == c.key && (uint32_t)index <= c.index);
  }

  // f(load, values) for every load of the row; a wave's are its segment's.
  template <class F>
  __device__ void each(F&& f) {
    for (int j = t; j < (row.loads + 63) / 64 * 64; j += kThreads) {
      float z[kPer];
      if (j < row.loads) {
        row.get(j, z);
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) z[i] = -INFINITY;
      }
      f(j, z);
    }
  }

  __device__ static unsigned long long wave_total(unsigned long long x) {
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
  }
  // Sum of x over the threads before this one; *all: over all of them.
  __device__ unsigned long long scan(unsigned long long x, unsigned long long* all) {
    unsigned long long y = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const unsigned long long z = __shfl_up(y, o);
      if (lane >= o) y += z;
    }
    __syncthreads();  // an earlier scan has been read
    if (lane == 63) L.wave_sum[wave] = y;
    __syncthreads();
    unsigned long long before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      const unsigned long long z = L.wave_sum[w];
      if (w < wave) before += z;
      sum += z;
    }
    *all = sum;
    return before + y - x;
  }

  __device__ void clear_bins() {
    __syncthreads();
    L.mass[t] = 0;
    L.count[t] = 0;
    __syncthreads();
  }
  // The histogram's bin that takes the running count (or mass) from `above` to
  // `want` or more; false if none does.  *above then stands before that bin.
  __device__ bool crossing(bool by_mass, unsigned long long want, unsigned long long* above_count,
                           unsigned long long* above_mass, uint32_t* at, uint32_t* here) {
    static_assert(kBins == kThreads, "a bin a thread");
    const unsigned long long c = L.count[t], m = L.mass[t];
    unsigned long long all_c, all_m;
    const unsigned long long bc = *above_count + scan(c, &all_c), bm = *above_mass + scan(m, &all_m);
    if (t == 0) L.found = ~0u;
    __syncthreads();
    if (by_mass ? bm < want && bm + m >= want : bc < want && bc + c >= want) {
      L.found = t;
      L.found_count = (uint32_t)bc;
      L.found_mass = bm;
    }
    __syncthreads();
    if (L.found == ~0u) {
      *above_count += all_c;
      *above_mass += all_m;
      return false;
    }
    *at = L.found;
    *here = L.count[*at];
    *above_count = L.found_count;
    *above_mass = L.found_mass;
    return true;
  }

  // The histogram of one window; the first time also the weight of all values.
  __device__ void histogram(int w, bool masses) {
    clear_bins();
    unsigned long long sum = 0;
    each([&](int, const float* z) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int b = bin(z[i]) - w * kBins;
        const unsigned long long m = masses ? weight(octaves(z[i])) : 0;
        sum += m;
        if (b >= 0 && b < kBins) {
          atomicAdd(&L.count[b], 1u);
          if (masses) atomicAdd(&L.mass[b], m);
        }
      }
    });
    if (masses) {
      unsigned long long all;
      scan(sum, &all);
      total = all;
    }
    window = w;
    __syncthreads();
  }

  __device__ void append(uint32_t key, int index) {
    const uint32_t at = atomicAdd(&L.listed, 1u);
    if (at < (uint32_t)kList) L.list[at] = (unsigned long long)~key << 32 | (uint32_t)index;
  }
  // Ascending sort of the list, padded to a power of two.
  __device__ void sort(int n) {
    int m = 64;
    while (m < n) m <<= 1;
    for (int i = n + t; i < m; i += kThreads) L.list[i] = ~0ull;
    for (int k = 2; k <= m; k <<= 1)
      for (int j = k >> 1; j; j >>= 1) {
        __syncthreads();
        for (int i = t; i < m / 2; i += kThreads) {
          const int a = 2 * i - (i & (j - 1)), b = a + j;
          const unsigned long long x = L.list[a], y = L.list[b];
          if ((x > y) == ((a & k) == 0)) {
            L.list[a] = y;
            L.list[b] = x;
          }
        }
      }
    __syncthreads();
  }

  // The cut after the listed values that take the running count or mass from
  // `above` to `want`; *mass: of all values in the cut.
  __device__ Cut cut_list(int n, bool by_mass, unsigned long long want, unsigned long long above_count,
                          unsigned long long above_mass, unsigned long long* mass) {
    sort(n);
    constexpr int kEach = kList / kThreads;
    unsigned long long m[kEach], sum = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int a = t * kEach + i;
      m[i] = a < n ? weight(octaves(value_of(~(uint32_t)(L.list[a] >> 32)))) : 0;
      sum += m[i];
    }
    unsigned long long before = above_mass + scan(sum, &all);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int a = t * kEach + i;
      if (a < n && (by_mass ? before < want && before + m[i] >= want : above_count + a + 1 == want)) {
        L.found = a;
        L.found_mass = before + m[i];
      }
      before += m[i];
    }
    __syncthreads();
    const unsigned long long x = L.list[L.found];
    *mass = L.found_mass;
    return {~(uint32_t)(x >> 32), (uint32_t)x};
  }

  // Too many values in a bin for the list: the bin's range of keys is cut
  // finer, down to a list, or to equal values, of which the first by index count.
  __device__ Cut cut_finer(int b, bool by_mass, bool masses, unsigned long long want, unsigned long long above_count,
                           unsigned long long above_mass, unsigned long long* mass) {
    if (t == 0) {
      L.key_lo = ~0u;
      L.key_hi = 0;
    }
    __syncthreads();
    uint32_t lo = ~0u, hi = 0;
    each([&](int, const float* z) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (bin(z[i]) == b) {
          lo = min(lo, key_of(z[i]));
          hi = max(hi, key_of(z[i]));
        }
    });
    atomicMin(&L.key_lo, lo);
    atomicMax(&L.key_hi, hi);
    __syncthreads();
    lo = L.key_lo;
    hi = L.key_hi;
    uint32_t here = ~0u;
    while (here > (uint32_t)kList && lo < hi) {
      int shift = 0;
      while ((hi - lo) >> shift >= (uint32_t)kBins) ++shift;
      clear_bins();
      each([&](int, const float* z) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const uint32_t k = key_of(z[i]);
          if (k < lo || k > hi) continue;
          atomicAdd(&L.count[(hi - k) >> shift], 1u);
          if (masses) atomicAdd(&L.mass[(hi - k) >> shift], weight(octaves(z[i])));
        }
      });
      __syncthreads();
      uint32_t at;
      if (!crossing(by_mass, want, &above_count, &above_mass, &at, &here)) break;  // never: the bin's sums are these
      hi -= at << shift;
      const uint32_t width = (1u << shift) - 1;
      lo = hi - lo > width ? hi - width : lo;
    }
    window = -1;
    if (here <= (uint32_t)kList) {
      if (t == 0) L.listed = 0;
      __syncthreads();
      each([&](int j, const float* z) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const uint32_t k = key_of(z[i]);
          if (k >= lo && k <= hi) append(k, row.index(j, i));
        }
      });
      __syncthreads();
      return cut_list((int)here, by_mass, want, above_count, above_mass, mass);
    }
    // equal values: `need` of them, the first by index
    const unsigned long long w = weight(octaves(value_of(lo)));
    const unsigned long long need = by_mass ? (want - above_mass + w - 1) / (w ? w : 1) : want - above_count;
    *mass = above_mass + need * w;
    seg_sums([&](float z, int) { return key_of(z) == lo; }, [](float) { return 1ull; });
    const uint32_t index = pick(need - 1, [&](float z, int) { return key_of(z) == lo; }, [](float) { return 1ull; });
    return {lo, index};
  }

  // segs[s] = sum of g over the values of segment s that f keeps
  template <class F, class G>
  __device__ void seg_sums(F&& f, G&& g) {
    __syncthreads();
    each([&](int j, const float* z) {
      unsigned long long sum = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (f(z[i], row.index(j, i))) sum += g(z[i]);
      if (__any(sum != 0)) sum = wave_total(sum);
      if (lane == 0) L.segs[j >> 6] = sum;
    });
    __syncthreads();
  }

  // The index, among what f keeps, of the first value up to which the sum of g exceeds `target` (segs hold the sums).
  template <class F, class G>
  __device__ uint32_t pick(unsigned long long target, F&& f, G&& g) {
    const int n = (row.loads + 63) / 64;
    static_assert(kSegs + 1 <= 2 * kThreads, "two segments a thread");
    const unsigned long long a = 2 * t < n ? L.segs[2 * t] : 0, b = 2 * t + 1 < n ? L.segs[2 * t + 1] : 0;
    unsigned long long all;
    const unsigned long long before = scan(a + b, &all);
    if (before <= target && target < before + a + b) {
      const bool second = target >= before + a;
      L.found = 2 * t + second;
      L.rest = target - before - (second ? a : 0);
    }
    __syncthreads();
    if (wave == 0) {
      const int j = (int)L.found * 64 + lane;
      const unsigned long long rest = L.rest;
      float z[kPer];
      unsigned long long m[kPer], sum = 0;
      if (j < row.loads) row.get(j, z);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        m[i] = j < row.loads && f(z[i], row.index(j, i)) ? g(z[i]) : 0;
        sum += m[i];
      }
      unsigned long long y = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const unsigned long long x = __shfl_up(y, o);
        if (lane >= o) y += x;
      }
      y -= sum;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (y <= rest && rest < y + m[i]) L.token = row.index(j, i);
        y += m[i];
      }
    }
    __syncthreads();
    return L.token;
  }

  __device__ int run(const SampleArgs& A, int r) {
    const float T = A.temperature ? A.temperature[r] : A.t_all, p = A.top_p ? A.top_p[r] : A.p_all;
    const float mp = A.min_p ? A.min_p[r] : A.m_all;
    const int k = A.top_k ? A.top_k[r] : A.k_all;
    if (t < 64) L.power[t] = exp2(t / 64.);
    uint32_t best = 0;
    each([&](int, const float* z) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) best = max(best, key_of(z[i]));
    });
#pragma unroll
    for (int o = 32; o; o >>= 1) best = max(best, (uint32_t)__shfl_xor((int)best, o));
    if (lane == 0) L.wave_max[wave] = best;
    if (t == 0) L.token = ~0u;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) best = max(best, L.wave_max[w]);
    top = value_of(best);
    if (top == -INFINITY) return -1;
    const bool use_k = k > 0 && k < row.vocab, use_p = p < 1.f;
    if (!(T > 0.f) || k == 1 || (use_p && p <= 0.f)) {
      uint32_t first = ~0u;
      each([&](int j, const float* z) {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (z[i] == top) first = min(first, (uint32_t)row.index(j, i));
      });
      if (first != ~0u) atomicMin(&L.token, first);
      __syncthreads();
      return (int)L.token;
    }
    slope = 1.4426950408889634 / (double)T;
    bin_slope = fminf((float)(slope * kBinsPerOctave), FLT_MAX);
    if (mp > 0.f) least = log2((double)fminf(mp, 1.f));
    Cut cut{0, ~0u};
    bool summed = false;  // segs hold the kept weights
    auto weigh = [&](float z) { return weight(octaves(z)); };
    auto likely = [&](float z) { return octaves(z) >= least; };
    for (int by_mass = use_k ? 0 : 1; by_mass <= (use_p ? 1 : 0); ++by_mass) {
      const bool last = by_mass == (use_p ? 1 : 0);
      unsigned long long want = k, above_count = 0, above_mass = 0, mass = 0;
      uint32_t at = 0, here = 0;
      if (by_mass) {
        if (window != 0) histogram(0, true);
        want = (unsigned long long)ceil((double)p * (double)total_kept(use_k));
        want = want ? want : 1;
      }
      const int windows = ((bits + 1) * kBinsPerOctave + kBins - 1) / kBins;
      bool found = false;
      int w = 0;
      for (; w < windows; ++w) {
        if (window != w) histogram(w, use_p);
        if ((found = crossing(by_mass, want, &above_count, &above_mass, &at, &here))) break;
      }
      if (!found) {  // the border lies among values of weight zero
        kept_mass = total;
        continue;
      }
      const int b = w * kBins + (int)at;
      if (here <= (uint32_t)kList) {
        if (t == 0) L.listed = 0;
        __syncthreads();
        each([&](int j, const float* z) {
          unsigned long long sum = 0;
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            const int zb = bin(z[i]);
            if (zb == b)
              append(key_of(z[i]), row.index(j, i));
            else if (last && zb < b && likely(z[i]))
              sum += weigh(z[i]);
          }
          if (last) {
            if (__any(sum != 0)) sum = wave_total(sum);
            if (lane == 0) L.segs[j >> 6] = sum;
          }
        });
        __syncthreads();
        cut = cut_list((int)here, by_mass, want, above_count, above_mass, &mass);
        if (last) {
          for (int i = t; i < (int)here; i += kThreads) {
            const unsigned long long x = L.list[i];
            const float z = value_of(~(uint32_t)(x >> 32));
            const int load = ((int)(uint32_t)x + row.lead) / kPer;
            if (in(cut, z, (int)(uint32_t)x) && likely(z)) atomicAdd(&L.segs[load >> 6], weigh(z));
          }
          summed = true;
          __syncthreads();
        }
      } else {
        cut = cut_finer(b, by_mass, use_p, want, above_count, above_mass, &mass);
      }
      kept_mass = mass;
    }
    auto kept = [&](float z, int index) { return z > -INFINITY && in(cut, z, index) && likely(z); };
    if (!summed) seg_sums(kept, weigh);
    const int n = (row.loads + 63) / 64;
    unsigned long long all;
    scan((2 * t < n ? L.segs[2 * t] : 0) + (2 * t + 1 < n ? L.segs[2 * t + 1] : 0), &all);
    const double u = fmax((double)A.u[r], 0.);
    unsigned long long target = (unsigned long long)fmin(u * (double)all, 0x1p63);
    target = target < all ? target : all - 1;
    return (int)pick(target, kept, weigh);
  }

  unsigned long long kept_mass = 0;  // of the values that top_k keeps
  __device__ unsigned long long total_kept(bool use_k) const { return use_k ? kept_mass : total; }
};

template <bool kF32>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs A) {
  __shared__ Shared lds;
  const int r = blockIdx.x;
  Sampler<kF32> s{lds, Row<kF32>(A.z, r * A.stride, A.vocab)};
  s.bits = A.scale_bits;
  const int token = s.run(A, r);
  if (threadIdx.x == 0) A.out[r] = token;
}

}  // namespace
}  // namespace gambit

extern "C" gambit_status gambit_sample(int32_t n, int32_t vocab, const void* logits, int32_t dtype, int64_t row_stride,
                                       const float* u, const float* temperature, float temperature_all,
                                       const int32_t* top_k, int32_t top_k_all, const float* top_p, float top_p_all,
                                       const float* min_p, float min_p_all, int32_t* ids_out, void* stream) {
  using namespace gambit;
  if (n < 0 || vocab < 1 || (dtype != GAMBIT_BF16 && dtype != GAMBIT_F32) || row_stride < 0) return GAMBIT_ERR_INVALID;
  if (vocab > kMaxVocab) return GAMBIT_ERR_UNSUPPORTED;
  if (n == 0) return GAMBIT_OK;
  if (!logits || !u || !ids_out || reinterpret_cast<uintptr_t>(logits) % (dtype == GAMBIT_F32 ? 4 : 2)) return GAMBIT_ERR_INVALID;
  for (const void* p : {(const void*)u, (const void*)temperature, (const void*)top_k, (const void*)top_p, (const void*)min_p, (const void*)ids_out})
    if (reinterpret_cast<uintptr_t>(p) % 4) return GAMBIT_ERR_INVALID;
  SampleArgs A{};
  A.z = logits;
  A.stride = row_stride;
  A.vocab = vocab;
  int log2v = 0;
  while ((1 << log2v) < vocab) ++log2v;
  A.scale_bits = 62 - log2v < 50 ? 62 - log2v : 50;
  A.u = u;
  A.temperature = temperature;
  A.top_k = top_k;
  A.top_p = top_p;
  A.min_p = min_p;
  A.t_all = temperature_all;
  A.k_all = top_k_all;
  A.p_all = top_p_all;
  A.m_all = min_p_all;
  A.out = ids_out;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == GAMBIT_F32)
    hipLaunchKernelGGL(sample_kernel<true>, dim3(n), dim3(kThreads), 0, s, A);
  else
    hipLaunchKernelGGL(sample_kernel<false>, dim3(n), dim3(kThreads), 0, s, A);
  return hipGetLastError() == hipSuccess ? GAMBIT_OK : GAMBIT_ERR_DEVICE;
}
