// One token for every row of logits: temperature, top-k, top-p, min-p, and the token that a given random number falls on.
//
// All limits leave the first so many of the row's tokens in the order of falling logits (equal ones by their numbers), so what is left is told by the least
// logit and how many of those that equal it.  Both are found without sorting: logits become integers of the same order, and their bits are looked at from the
// highest on, eleven at a time, by counts (top-k) or sums of probabilities (top-p) of all that agree in the bits so far.  Then the row is walked in the order of its numbers.
//
// Probabilities w = exp((l - l_max) / T) are compared with shares of their sum, and near a border the last bits decide which token comes out; 50000 of them in fp32 would put
// one row in a hundred on the wrong token.  So they are taken in 64 bits and added as integers w 2^s, s as large as vocab of them fit into 62 bits (sums
// do not depend on their order then, in LDS atomics neither).
#include <math.h>
#include <algorithm>

#include "common.h"
#include "launch.h"

namespace sif {

constexpr uint32_t SM_THREADS = 1024, SM_WAVES = SM_THREADS / 64, SM_BINS = 2048;
constexpr uint32_t kKeyNone = 0x007FFFFFu;      // of -inf

struct SampleArgs {
  const void* logits;
  const float* temperature_list;
  const int32_t* top_k_list;
  const float* top_p_list;
  const float* min_p_list;
  const float* random;
  int32_t* token;
  float* logprob;
  int32_t* kept;
  uint32_t vocab, ld, shift;
  float temperature, top_p, min_p;
  int32_t top_k;
};

// An integer of the same order; 0 for both zeros, -inf for NaN.
__device__ __forceinline__ uint32_t sm_key(float x) {
  x = x != x ? -INFINITY : x + 0.0f;
  const uint32_t u = __float_as_uint(x);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float sm_value(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// exp(x), x <= 0 (NaN counts as far below): 2^n times 2^f with |f| <= 1/2, whose Taylor series to the 13th power is right to 2^-54.
__device__ __forceinline__ double sm_exp(double x) {
  const double t = fmax(x * 1.44269504088896340736, -1100.0), n = rint(t), r = (t - n) * 0.693147180559945309417;
  double p = 1.0 / 6227020800.0;
  p = fma(p, r, 1.0 / 479001600.0);
  p = fma(p, r, 1.0 / 39916800.0);
  p = fma(p, r, 1.0 / 3628800.0);
  p = fma(p, r, 1.0 / 362880.0);
  p = fma(p, r, 1.0 / 40320.0);
  p = fma(p, r, 1.0 / 5040.0);
  p = fma(p, r, 1.0 / 720.0);
  p = fma(p, r, 1.0 / 120.0);
  p = fma(p, r, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  return ldexp(p, (int)n);
}

struct SampleScale {
  float top;
  double inv_t, unit;
  __device__ __forceinline__ double x(float l) const { return l == top ? 0.0 : ((double)l - (double)top) * inv_t; }
  __device__ __forceinline__ double w(float l) const { return sm_exp(x(l)); }
  __device__ __forceinline__ uint64_t whole(double w) const {      // w 2^s, to the nearest (below 2^52: added to 2^52 it is the sum's mantissa)
    return (uint64_t)__double_as_longlong(fma(w, unit, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
  }
};

// A row's logits, sixteen bytes at a time: the wavefronts take one piece each, in order, the lanes of a wavefront neighbouring vectors.
template <typename E>
struct SampleRow {
  static constexpr uint32_t N = 16 / sizeof(E);
  const E* row;
  uint32_t vocab, per_wave;           // elements of a wavefront, a multiple of 64 * N
  // f(index of the first, N values): values past the end are -inf
  template <typename F> __device__ __forceinline__ void each(uint32_t wave, F&& f) const {
    const uint32_t lane = threadIdx.x & 63, end = std::min((wave + 1) * per_wave, vocab);
    for (uint32_t at = wave * per_wave; at < end; at += 64 * N) f(at + lane * N, load(at + lane * N));
  }
  struct Vec { float x[N]; };
  __device__ __forceinline__ Vec load(uint32_t i) const {
    Vec v;
    uint4 u = make_uint4(0, 0, 0, 0);
    if (i < vocab) u = *reinterpret_cast<const uint4*>(row + i);       // (rows are padded to whole vectors)
    if constexpr (N == 4) { v.x[0] = __uint_as_float(u.x); v.x[1] = __uint_as_float(u.y); v.x[2] = __uint_as_float(u.z); v.x[3] = __uint_as_float(u.w); }
    else { v.x[0] = bflo(u.x); v.x[1] = bfhi(u.x); v.x[2] = bflo(u.y); v.x[3] = bfhi(u.y); v.x[4] = bflo(u.z); v.x[5] = bfhi(u.z); v.x[6] = bflo(u.w); v.x[7] = bfhi(u.w); }
#pragma unroll
    for (uint32_t e = 0; e < N; ++e)
      if (i + e >= vocab) v.x[e] = -INFINITY;
    return v;
  }
};

__device__ __forceinline__ uint64_t sm_up64(uint64_t x, int o) {
  return (uint64_t)(uint32_t)__shfl_up((uint32_t)(x >> 32), o, 64) << 32 | (uint32_t)__shfl_up((uint32_t)x, o, 64);
}
__device__ __forceinline__ uint64_t sm_scan64(uint64_t v) {            // inclusive, over a wavefront
  const uint32_t lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t t = sm_up64(v, o);
    if (lane >= (uint32_t)o) v += t;
  }
  return v;
}

struct SampleShared {
  uint64_t bins[SM_BINS];
  uint64_t wave[SM_WAVES];
  uint64_t above;                     // what lies above the bin that was found
  uint32_t bin, ties[SM_WAVES], kept[SM_WAVES];
  float red[SM_WAVES];
  uint64_t picked[2];
};

// The bin, from the highest on, at which the running sum of the bins reaches `target` (asked(sum): whether it does); sh.above gets the sum of those above it.
// Returns the sum of all bins.
template <typename A>
__device__ __forceinline__ uint64_t sm_find(SampleShared& sh, uint64_t above, A&& asked_of) {
  const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const uint64_t hi = sh.bins[SM_BINS - 1 - 2 * t], lo = sh.bins[SM_BINS - 2 - 2 * t];
  uint64_t upto = sm_scan64(hi + lo);
  if (lane == 63) sh.wave[wave] = upto;
  if (t == 0) sh.bin = 0;
  __syncthreads();
  uint64_t before = 0, all = 0;
  for (uint32_t w = 0; w < SM_WAVES; ++w) {
    before += w < wave ? sh.wave[w] : 0;
    all += sh.wave[w];
  }
  upto += before;
  const uint64_t start = upto - hi - lo;
  auto asked = asked_of(all);
  const bool s0 = asked(above + start), s1 = asked(above + start + hi), s2 = asked(above + upto);
  if (!s0 && s2) {                               // one thread, or none where all bins together do not reach it
    sh.bin = s1 ? SM_BINS - 1 - 2 * t : SM_BINS - 2 - 2 * t;
    sh.above = above + (s1 ? start : start + hi);
  }
  __syncthreads();
  return all;
}

template <typename E>
__global__ __launch_bounds__(SM_THREADS) void sample_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6, i = blockIdx.x;
  SampleRow<E> row;
  row.row = (const E*)a.logits + (size_t)i * a.ld;
  row.vocab = a.vocab;
  constexpr uint32_t N = SampleRow<E>::N, STEP = 64 * N;
  row.per_wave = ((a.vocab + SM_WAVES - 1) / SM_WAVES + STEP - 1) / STEP * STEP;
  const float temperature = a.temperature_list != nullptr ? a.temperature_list[i] : a.temperature;
  const int32_t top_k = a.top_k_list != nullptr ? a.top_k_list[i] : a.top_k;
  const float top_p = a.top_p_list != nullptr ? a.top_p_list[i] : a.top_p;
  const float min_p = std::min(a.min_p_list != nullptr ? a.min_p_list[i] : a.min_p, 1.f);

  // the largest logit, and how many there are
  uint32_t best = 0, some = 0;
  row.each(wave, [&](uint32_t, const typename SampleRow<E>::Vec& v) {
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) {
      const uint32_t key = sm_key(v.x[e]);
      best = std::max(best, key);
      some += key > kKeyNone ? 1u : 0u;
    }
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    best = std::max(best, (uint32_t)__shfl_xor(best, o, 64));
    some += __shfl_xor(some, o, 64);
  }
  if (lane == 0) { sh.ties[wave] = best; sh.kept[wave] = some; }
  __syncthreads();
  best = some = 0;
  for (uint32_t w = 0; w < SM_WAVES; ++w) { best = std::max(best, sh.ties[w]); some += sh.kept[w]; }
  __syncthreads();
  if (best <= kKeyNone) {
    if (t == 0) {
      a.token[i] = -1;
      if (a.logprob != nullptr) a.logprob[i] = -INFINITY;
      if (a.kept != nullptr) a.kept[i] = 0;
    }
    return;
  }
  const bool greedy = !(temperature > 0.f);
  SampleScale sc;
  sc.top = sm_value(best);
  sc.inv_t = greedy ? 1.0 : 1.0 / (double)temperature;
  sc.unit = ldexp(1.0, (int)a.shift);

  // what is left: keys above `least`, and the first `equal` of those that are equal to it
  uint32_t least = kKeyNone, equal = 0;
  if (greedy) {
    least = best;
    equal = 1;
  } else {
    if (top_k > 0 && (uint32_t)top_k < some) {
      uint32_t known = 0, mask = 0;
      uint64_t above = 0;
#pragma unroll 1
      for (int level = 0; level < 3; ++level) {
        const int low = level == 0 ? 21 : level == 1 ? 10 : 0;
        const uint32_t bits = level == 2 ? 1023u : 2047u;
        for (uint32_t b = t; b < SM_BINS; b += SM_THREADS) sh.bins[b] = 0;
        __syncthreads();
        row.each(wave, [&](uint32_t, const typename SampleRow<E>::Vec& v) {
#pragma unroll
          for (uint32_t e = 0; e < N; ++e) {
            const uint32_t key = sm_key(v.x[e]);
            if (key > kKeyNone && (key & mask) == known) atomicAdd((unsigned long long*)&sh.bins[key >> low & bits], 1ull);
          }
        });
        __syncthreads();
        sm_find(sh, above, [&](uint64_t) { return [&](uint64_t sum) { return sum >= (uint64_t)top_k; }; });
        above = sh.above;
        known |= sh.bin << low;
        mask |= bits << low;
        __syncthreads();
      }
      least = known;
      equal = (uint32_t)top_k - (uint32_t)above;
    }
    if (top_p < 1.f) {
      uint32_t known = 0, mask = 0;
      uint64_t above = 0;
      double target = 0.0;
#pragma unroll 1
      for (int level = 0; level < 3; ++level) {
        const int low = level == 0 ? 21 : level == 1 ? 10 : 0;
        const uint32_t bits = level == 2 ? 1023u : 2047u;
        for (uint32_t b = t; b < SM_BINS; b += SM_THREADS) sh.bins[b] = 0;
        __syncthreads();
        row.each(wave, [&](uint32_t, const typename SampleRow<E>::Vec& v) {
#pragma unroll
          for (uint32_t e = 0; e < N; ++e) {
            const uint32_t key = sm_key(v.x[e]);
            if (key > least && (key & mask) == known) atomicAdd((unsigned long long*)&sh.bins[key >> low & bits], (unsigned long long)sc.whole(sc.w(sm_value(key))));
          }
        });
        if (t == 0 && equal != 0 && (least & mask) == known) atomicAdd((unsigned long long*)&sh.bins[least >> low & bits], (unsigned long long)(equal * sc.whole(sc.w(sm_value(least)))));
        __syncthreads();
        const int at_level = level;
        sm_find(sh, above, [&](uint64_t all) {
          if (at_level == 0) target = fmax((double)top_p * (double)all, 0.5);      // (at least one token)
          return [&](uint64_t sum) { return (double)sum >= target; };
        });
        above = sh.above;
        known |= sh.bin << low;
        mask |= bits << low;
        __syncthreads();
      }
      // of those equal to `known` as many as it takes
      const uint64_t w = sc.whole(sc.w(sm_value(known)));
      uint64_t need = 1;
      if (w != 0) {
        need = (uint64_t)fmax((target - (double)above) / (double)w, 1.0);
        while (need > 1 && (double)(above + (need - 1) * w) >= target) --need;
        while ((double)(above + need * w) < target) ++need;
      }
      if (known == least) {
        equal = (uint32_t)std::min<uint64_t>(equal, need);
      } else {
        least = known;
        equal = (uint32_t)std::min<uint64_t>(need, a.vocab);
      }
    }
  }

  // The row in the order of its numbers.  First each wavefront's ties, then its sum.
  uint32_t ties = 0;
  if (equal != 0)
    row.each(wave, [&](uint32_t, const typename SampleRow<E>::Vec& v) {
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) ties += sm_key(v.x[e]) == least ? 1u : 0u;
    });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) ties += __shfl_xor(ties, o, 64);
  if (lane == 0) sh.ties[wave] = ties;
  __syncthreads();
  uint32_t ties_before = 0;
  for (uint32_t w = 0; w < wave; ++w) ties_before += sh.ties[w];
  // which of a vector's tokens are left, and what they weigh; `seen`: ties up to here in this wavefront
  auto weigh = [&](const typename SampleRow<E>::Vec& v, uint32_t& seen, uint64_t (&w)[N]) {
    uint32_t left = 0, mine = 0, key[N];
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) {
      key[e] = sm_key(v.x[e]);
      mine += equal != 0 && key[e] == least ? 1u : 0u;
    }
    uint32_t upto = mine;
    if (__any(mine != 0)) {
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(upto, o, 64);
        if (lane >= (uint32_t)o) upto += x;
      }
    }
    uint32_t rank = seen + upto - mine;
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) {
      bool keep = key[e] > least;
      if (equal != 0 && key[e] == least) keep = rank++ < equal;
      w[e] = 0;
      if (keep) {
        const double x = sc.w(sm_value(key[e]));
        if (!(x < (double)min_p)) {
          w[e] = sc.whole(x);
          ++left;
        }
      }
    }
    seen += __shfl(upto, 63, 64);
    return left;
  };
  uint64_t sum = 0;
  uint32_t left = 0, seen = ties_before;
  row.each(wave, [&](uint32_t, const typename SampleRow<E>::Vec& v) {
    uint64_t w[N];
    left += weigh(v, seen, w);
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) sum += w[e];
  });
  sum = sm_scan64(sum);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) left += __shfl_xor(left, o, 64);
  if (lane == 63) sh.wave[wave] = sum;
  if (lane == 0) sh.kept[wave] = left;
  __syncthreads();
  uint64_t before = 0, all = 0;
  uint32_t kept = 0;
  for (uint32_t w = 0; w < SM_WAVES; ++w) {
    before += w < wave ? sh.wave[w] : 0;
    all += sh.wave[w];
    kept += sh.kept[w];
  }
  float u = a.random != nullptr ? a.random[i] : 0.f;
  u = u > 0.f ? std::min(u, 0.99999994f) : 0.f;
  const double target = (double)u * (double)all;
  // the wavefront on whose piece it falls looks again
  if ((double)before > target || !((double)(before + sh.wave[wave]) > target)) return;
  seen = ties_before;
  uint64_t at = before;
  bool found = false;
  row.each(wave, [&](uint32_t first, const typename SampleRow<E>::Vec& v) {
    if (found) return;
    uint64_t w[N], mine = 0;
    weigh(v, seen, w);
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) mine += w[e];
    const uint64_t upto = at + sm_scan64(mine);
    const uint64_t hits = __ballot((double)upto > target);
    if (hits != 0) {
      found = true;
      if (lane == (uint32_t)__ffsll((unsigned long long)hits) - 1) {
        uint64_t x = upto - mine;
        uint32_t e = 0;
        for (; e + 1 < N; ++e) {
          x += w[e];
          if ((double)x > target) break;
        }
        a.token[i] = (int32_t)(first + e);
        if (a.logprob != nullptr) {
          float l = v.x[0];
#pragma unroll
          for (uint32_t z = 1; z < N; ++z) l = e == z ? v.x[z] : l;
          a.logprob[i] = greedy ? 0.f : (float)(sc.x(l) - log((double)all / sc.unit));
        }
        if (a.kept != nullptr) a.kept[i] = (int32_t)kept;
      }
      return;
    }
    at = (uint64_t)(uint32_t)__shfl((uint32_t)(upto >> 32), 63, 64) << 32 | (uint32_t)__shfl((uint32_t)upto, 63, 64);
  });
}

}  // namespace sif

using namespace sif;

extern "C" {

sif_status sif_k_sample(const sif_sample_args* a, void* stream) {
  if (!a) return fail(SIF_E_INVAL, "sample: null arguments");
  if (a->struct_size != sizeof(sif_sample_args)) return fail(SIF_E_INVAL, "sample: struct_size");
  if (a->dtype != SIF_F32 && a->dtype != SIF_BF16) return fail(SIF_E_INVAL, "sample: dtype must be SIF_F32 or SIF_BF16");
  if (a->n == 0 || a->n > 1u << 20 || a->vocab == 0 || a->vocab > 1u << 18) return fail(SIF_E_INVAL, "sample: rows outside 1 .. 2^20 or tokens outside 1 .. 2^18");
  if (a->ld < a->vocab || (a->ld & 7)) return fail(SIF_E_INVAL, "sample: bad leading dimension");
  if (!a->logits_dev || !a->token_dev) return fail(SIF_E_INVAL, "sample: null operand");
  if (!a->temperature_dev && !(a->temperature >= 0.f)) return fail(SIF_E_INVAL, "sample: temperature must not be negative");
  if (!a->random_dev && (a->temperature_dev || a->temperature > 0.f)) return fail(SIF_E_INVAL, "sample: no random numbers");
  if ((uintptr_t)a->logits_dev & 15) return fail(SIF_E_INVAL, "sample: logits must be 16-byte aligned");
  if (((uintptr_t)a->temperature_dev | (uintptr_t)a->top_k_dev | (uintptr_t)a->top_p_dev | (uintptr_t)a->min_p_dev | (uintptr_t)a->random_dev | (uintptr_t)a->token_dev |
       (uintptr_t)a->logprob_dev | (uintptr_t)a->kept_dev) & 3) return fail(SIF_E_INVAL, "sample: misaligned list");
  SampleArgs x;
  x.logits = a->logits_dev;
  x.temperature_list = a->temperature_dev;
  x.top_k_list = a->top_k_dev;
  x.top_p_list = a->top_p_dev;
  x.min_p_list = a->min_p_dev;
  x.random = a->random_dev;
  x.token = a->token_dev;
  x.logprob = a->logprob_dev;
  x.kept = a->kept_dev;
  x.vocab = a->vocab;
  x.ld = a->ld;
  x.shift = 51;
  while ((uint64_t)a->vocab << x.shift > 1ull << 62) --x.shift;
  x.temperature = a->temperature;
  x.top_k = a->top_k;
  x.top_p = a->top_p;
  x.min_p = a->min_p;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (a->dtype == SIF_BF16) hipLaunchKernelGGL((sample_kernel<bf16_t>), dim3(a->n), dim3(SM_THREADS), 0, s, x);
  else hipLaunchKernelGGL((sample_kernel<float>), dim3(a->n), dim3(SM_THREADS), 0, s, x);
  return check_launch("sample");
}

}  // extern "C"
