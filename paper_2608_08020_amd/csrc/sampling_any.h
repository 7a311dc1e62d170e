// The draw of a token from any row of logits (see sampling.hip): short rows, and
// those that the kernels there leave.  One workgroup a row goes over it as
// often as the filters ask: the maximum; with a filter, a histogram of the
// weights by 64ths of an octave, eight octaves at a time from the maximum down,
// and the row's whole weight; the values of the bin where the filter's border
// falls, listed and sorted in LDS, or, of too many, a finer histogram of their
// keys, down to equal values; the kept weight of every 64 loads; then the 64 loads
// that the token is among.
#pragma once

#include "sampling.h"

namespace gambit {

constexpr int kAnyThreads = 512;
constexpr int kAnyBins = 512, kAnyPerOctave = 64;  // a histogram's window: 8 octaves
constexpr int kAnyList = 4096;                       // listed values of one bin

struct AnyShared {
  u64 mass[kAnyBins];
  uint32_t count[kAnyBins];
  u64 list[kAnyList];  // ~key, index: ascending is likeliest first
  u64 segs[kSegs + 1];
  double power[64];
  u64 wave_sum[kAnyThreads / 64];
  u64 found_mass, rest;
  uint32_t wave_max[kAnyThreads / 64];
  uint32_t found, found_count, listed, key_lo, key_hi, token;
};

#define L lds_as<AnyShared>()

template <bool kF32>
struct Sampler {
  const Row<kF32> row;
  static constexpr int kPer = Row<kF32>::kPer;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  float top = 0.f;         // the row's maximum
  double slope = 0.;       // log2(e) / T
  float bin_slope = 0.f;
  double least = -INFINITY;  // log2 of min_p
  u64 total = 0;  // weight of all values
  int window = -1;         // the histogram's

  // log2 of a weight
  __device__ __forceinline__ double octaves(float z) const { return ((double)z - (double)top) * slope; }
  // 2^44 times the weight, rounded; 0 below half a unit (NaN: of -inf at an infinite temperature)
  __device__ __forceinline__ u64 weight(double x) const {
    if (!(x >= -(double)(kBits + 1))) return 0;
    const double y = x + kTo64ths;
    return weight_of((int)__double_as_longlong(y), x - (y - kTo64ths), L.power);
  }
  // Bin of a value, from the maximum down; a huge one for -inf.
  __device__ __forceinline__ int bin(float z) const {
    return z > -INFINITY ? (int)fminf(fminf(top - z, FLT_MAX) * bin_slope, 0x1p30f) : 0x7fffffff;
  }
  // f(load, values) for every load of the row; a wave's are its segment's.
  template <class F>
  __device__ __forceinline__ void each(F&& f) {
    for (int j = t; j < (row.loads + 63) / 64 * 64; j += kAnyThreads) {
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

  __device__ __forceinline__ u64 scan(u64 x, u64* all) { return block_before<kAnyThreads>(x, L.wave_sum, all); }

  __device__ __forceinline__ void clear_bins() {
    __syncthreads();
    L.mass[t] = 0;
    L.count[t] = 0;
    __syncthreads();
  }
  // The histogram's bin that takes the running count (or mass) from `above` to
  // `want` or more; false if none does.  *above then stands before that bin.
  __device__ __forceinline__ bool crossing(bool by_mass, u64 want, u64* above_count,
                           u64* above_mass, uint32_t* at, uint32_t* here) {
    static_assert(kAnyBins == kAnyThreads, "a bin a thread");
    const u64 c = L.count[t], m = L.mass[t];
    u64 all_c, all_m;
    const u64 bc = *above_count + scan(c, &all_c), bm = *above_mass + scan(m, &all_m);
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
  __device__ __forceinline__ void histogram(int w, bool masses) {
    clear_bins();
    u64 sum = 0;
    each([&](int, const float* z) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int b = bin(z[i]) - w * kAnyBins;
        const u64 m = masses ? weight(octaves(z[i])) : 0;
        sum += m;
        if (b >= 0 && b < kAnyBins) {
          atomicAdd(&L.count[b], 1u);
          if (masses) atomicAdd(&L.mass[b], m);
        }
      }
    });
    if (masses) {
      u64 all;
      scan(sum, &all);
      total = all;
    }
    window = w;
    __syncthreads();
  }

  __device__ __forceinline__ void append(uint32_t key, int index) {
    const uint32_t at = atomicAdd(&L.listed, 1u);
    if (at < (uint32_t)kAnyList) L.list[at] = (u64)~key << 32 | (uint32_t)index;
  }
  // The cut after the listed values that take the running count or mass from
  // `above` to `want`; *mass: of all values in the cut.
  __device__ __forceinline__ Cut cut_list(int n, bool by_mass, u64 want, u64 above_count,
                          u64 above_mass, u64* mass) {
    block_sort<kAnyThreads>(L.list, n);
    constexpr int kEach = kAnyList / kAnyThreads;
    u64 m[kEach], sum = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int a = t * kEach + i;
      m[i] = a < n ? weight(octaves(value_of(~(uint32_t)(L.list[a] >> 32)))) : 0;
      sum += m[i];
    }
    u64 before = above_mass + scan(sum, &all);
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
    const u64 x = L.list[L.found];
    *mass = L.found_mass;
    return {~(uint32_t)(x >> 32), (uint32_t)x};
  }

  // Too many values in a bin for the list: the bin's range of keys is cut
  // finer, down to a list, or to equal values, of which the first by index count.
  __device__ __forceinline__ Cut cut_finer(int b, bool by_mass, bool masses, u64 want, u64 above_count,
                           u64 above_mass, u64* mass) {
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
    while (here > (uint32_t)kAnyList && lo < hi) {
      int shift = 0;
      while ((hi - lo) >> shift >= (uint32_t)kAnyBins) ++shift;
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
    if (here <= (uint32_t)kAnyList) {
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
    const u64 w = weight(octaves(value_of(lo)));
    const u64 need = by_mass ? (want - above_mass + w - 1) / (w ? w : 1) : want - above_count;
    *mass = above_mass + need * w;
    seg_sums([&](float z, int) { return key_of(z) == lo; }, [](float) { return 1ull; });
    const uint32_t index = pick(need - 1, [&](float z, int) { return key_of(z) == lo; }, [](float) { return 1ull; });
    return {lo, index};
  }

  // segs[s] = sum of g over the values of segment s that f keeps
  template <class F, class G>
  __device__ __forceinline__ void seg_sums(F&& f, G&& g) {
    __syncthreads();
    each([&](int j, const float* z) {
      u64 sum = 0;
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
  __device__ __forceinline__ uint32_t pick(u64 target, F&& f, G&& g) {
    const int n = (row.loads + 63) / 64;
    constexpr int kEach = (kSegs + kAnyThreads - 1) / kAnyThreads;
    u64 seg[kEach], part = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) part += seg[i] = kEach * t + i < n ? L.segs[kEach * t + i] : 0;
    u64 before = scan(part, &all);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (before <= target && target < before + seg[i]) {
        L.found = kEach * t + i;
        L.rest = target - before;
      }
      before += seg[i];
    }
    __syncthreads();
    if (wave == 0) {
      const int j = (int)L.found * 64 + lane;
      const u64 rest = L.rest;
      float z[kPer];
      u64 m[kPer], sum = 0;
      if (j < row.loads) row.get(j, z);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        m[i] = j < row.loads && f(z[i], row.index(j, i)) ? g(z[i]) : 0;
        sum += m[i];
      }
      u64 y = wave_before(sum, lane);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (y <= rest && rest < y + m[i]) L.token = row.index(j, i);
        y += m[i];
      }
    }
    __syncthreads();
    return L.token;
  }

  __device__ __forceinline__ int run(const SampleArgs& A, int r) {
    const Filter F(A, r);
    const bool use_k = F.use_k, use_p = F.use_p;
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
    for (int w = 0; w < kAnyThreads / 64; ++w) best = max(best, L.wave_max[w]);
    top = value_of(best);
    if (top == -INFINITY) return -1;
    if (F.greedy) {
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
    slope = F.slope;
    bin_slope = fminf((float)(slope * kAnyPerOctave), FLT_MAX);
    least = F.least();
    Cut cut{0, ~0u};
    bool summed = false;  // segs hold the kept weights
    auto weigh = [&](float z) { return weight(octaves(z)); };
    auto likely = [&](float z) { return octaves(z) >= least; };
    for (int by_mass = use_k ? 0 : 1; by_mass <= (use_p ? 1 : 0); ++by_mass) {
      const bool last = by_mass == (use_p ? 1 : 0);
      u64 want = F.k, above_count = 0, above_mass = 0, mass = 0;
      uint32_t at = 0, here = 0;
      if (by_mass) {
        if (window != 0) histogram(0, true);
        want = (u64)ceil((double)F.p * (double)total_kept(use_k));
        want = want ? want : 1;
      }
      const int windows = ((kBits + 1) * kAnyPerOctave + kAnyBins - 1) / kAnyBins;
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
      const int b = w * kAnyBins + (int)at;
      if (here <= (uint32_t)kAnyList) {
        if (t == 0) L.listed = 0;
        __syncthreads();
        each([&](int j, const float* z) {
          u64 sum = 0;
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
          for (int i = t; i < (int)here; i += kAnyThreads) {
            const u64 x = L.list[i];
            const float z = value_of(~(uint32_t)(x >> 32));
            const int load = ((int)(uint32_t)x + row.lead) / kPer;
            if (cut.holds(z, (int)(uint32_t)x) && likely(z)) atomicAdd(&L.segs[load >> 6], weigh(z));
          }
          summed = true;
          __syncthreads();
        }
      } else {
        cut = cut_finer(b, by_mass, use_p, want, above_count, above_mass, &mass);
      }
      kept_mass = mass;
    }
    auto kept = [&](float z, int index) { return z > -INFINITY && cut.holds(z, index) && likely(z); };
    if (!summed) seg_sums(kept, weigh);
    const int n = (row.loads + 63) / 64;
    u64 all;
    u64 mine = 0;
    for (int i = t; i < n; i += kAnyThreads) mine += L.segs[i];
    scan(mine, &all);
    const double u = fmax((double)A.u[r], 0.);
    u64 target = (u64)fmin(u * (double)all, 0x1p63);
    target = target < all ? target : all - 1;
    return (int)pick(target, kept, weigh);
  }

  u64 kept_mass = 0;  // of the values that top_k keeps
  __device__ __forceinline__ u64 total_kept(bool use_k) const { return use_k ? kept_mass : total; }
};

#undef L

}  // namespace gambit
