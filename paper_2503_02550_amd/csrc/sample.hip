// One token for every row of logits: temperature, top-k, top-p, min-p, and the token that a given random number falls on.
//
// All limits leave the first so many of the row's tokens in the order of falling logits (equal ones by their numbers), so what is left is told by the least
// logit and how many of those that equal it.  A block of sixteen wavefronts takes a row:
//   the largest logit (a temperature of 0 ends here);
//   a bound that what is left must reach: for a top-k of up to 512 that of the k-th largest of the threads' own largest logits, else of a histogram of counts or, for top-p, of
//     probabilities over equal steps of the logit;
//   a list of tokens, up to 1024.  For a top-k all that reach the bound, where they fit: then all else happens on that list, sums over ranks decide about top-p, sums over the list
//     about the token.  For a top-p, and a top-k of more, only those of the bound's own bin: it gives the least logit that is left.  Where they do not fit (many equal logits) the least logit
//     is found from the bits of the logits, eleven at a time;
//   the sums of what is left in sixteen parts of the row (for a top-p they were added up while the bin was listed), which say in which part the token lies, and so on in there.
// A row is read from memory once; a part of it stays in LDS, later walks find the rest in the L2.
//
// What bounds it is not the row's bytes (256 rows of 50304 fp32 logits: 6.5 of 44 us) but the walks of one CU over its row: 3 us for a walk that compares, 10 for one that adds up a histogram of probabilities,
// 11 for the sums of what is left (some 25 vector instructions an element, four cycles each, on 1/256 of the chip), 15 where it lists as well, 1 to 2 for a phase with barriers. One row of 50256 in bf16:
// greedy 5.1 us, top-k 50 11, 200 16, 900 26, nothing but the temperature 19, top-p 0.9 of which 953 are left 36, 21180 38; 256 rows of 50304 in fp32: 11, 19, 23, 35, 24, 41, 44.
//
// Probabilities w = exp((l - l_max) / T) are compared with shares of their sum, and near a border the last bits decide which token comes out; 50000 of them in fp32 would put
// one row in a hundred on the wrong token.  So they are taken in 64 bits and added as integers w 2^s, s as large as vocab of them fit into 62 bits (sums
// do not depend on their order then, in LDS atomics neither).
#include <math.h>
#include <algorithm>

#include "common.h"
#include "launch.h"

namespace sif {

constexpr uint32_t SM_THREADS = 1024, SM_WAVES = SM_THREADS / 64, SM_BINS = 4096, SM_LIST = 1024, SM_COUNTED = 384;
constexpr uint32_t SM_FEW = 512;       // a top-k that the threads' largest bound
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

// 2^x for |x| <= 1: the Taylor series of exp(x ln 2) to the 18th power, right to 2^-52.
__device__ __forceinline__ double sm_exp2(double x) {
  const double r = x * 0.693147180559945309417;
  double p = 1.0 / 6402373705728000.0;
  p = fma(p, r, 1.0 / 355687428096000.0);
  p = fma(p, r, 1.0 / 20922789888000.0);
  p = fma(p, r, 1.0 / 1307674368000.0);
  p = fma(p, r, 1.0 / 87178291200.0);
  p = fma(p, r, 1.0 / 6227020800.0);
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
  return fma(p, r, 1.0);
}

// A logit as a number of steps below the largest one, NaN and what is further as the last: t, the nearest whole number n and the rest r.  (2^52 + 2^51 in front of the point
// leaves no bits behind it.)  Differences, products, cuts and roundings keep the order, so steps of steps do.
struct SampleStep { int n; double r; };
struct SampleSteps {
  double top, per;
  __device__ __forceinline__ SampleStep of(float l, double last = -65504.0) const {
    const double t = fmax(((double)l - top) * per, last), m = t + 6755399441055744.0;
    return {(int)(uint32_t)__double_as_longlong(m), t - (m - 6755399441055744.0)};
  }
  __device__ __forceinline__ static uint32_t bin(int n) { return (uint32_t)(SM_BINS - 1 + (n >> 4)); }      // 1 .. 4095
};

// A token's probability over the largest one's, times 2^s: 2^(t / 1024) from a table of 2^(i / 1024) and three terms of a series (the next one is 2^-50 at most).  2^-63.97 is as
// good as nothing, and below a half as an integer.
struct SampleScale {
  SampleSteps steps;
  const double* table;                // in LDS: 2^(s + i / 1024)
  __device__ __forceinline__ double scaled(const SampleStep& x) const {
    constexpr double k = 0.693147180559945309417 / 1024.0;
    const double p = fma(fma(fma(k * k * k / 6.0, x.r, k * k / 2.0), x.r, k), x.r, 1.0);
    const double y = table[x.n & 1023] * p;        // (no less than 2^s, s from 30 on, so the exponent takes n's whole part as it is)
    return __hiloint2double(__double2hiint(y) + (x.n >> 10 << 20), __double2loint(y));
  }
  // To the nearest whole number: below 2^52 it is the mantissa of the sum with 2^52, whose other bits sums may leave in and take away once.
  static constexpr uint64_t kRaw = 0x4330000000000000ull;
  __device__ __forceinline__ static uint64_t raw(double y) { return (uint64_t)__double_as_longlong(y + 4503599627370496.0); }
  __device__ __forceinline__ static uint64_t whole(double y) { return raw(y) & 0xFFFFFFFFFFFFFull; }
  __device__ __forceinline__ uint64_t mass(float l) const { return whole(scaled(steps.of(l))); }
};

// A row's logits, sixteen bytes at a time, neighbouring lanes neighbouring vectors, a piece of the row to each wavefront in order.  What stands behind the row reads as -inf.
// The first vectors of every lane stay in LDS, the others are read again for every walk: 256 rows of 50304 fp32 logits are more than the L2s hold, half of them is not.
constexpr uint32_t SM_HELD = 6;
template <typename E>
struct SampleRow {
  static constexpr uint32_t N = 16 / sizeof(E), STEP = 64 * N;
  const E* row;
  uint4* held;                        // in LDS: [wavefront][SM_HELD][lane]
  uint32_t vocab;
  bool infinite;                      // there are logits of +inf: they read as 0 and the others as -inf
  struct Vec { float x[N]; };
  __device__ __forceinline__ static Vec values(const uint4& u) {
    Vec v;
    if constexpr (N == 4) { v.x[0] = __uint_as_float(u.x); v.x[1] = __uint_as_float(u.y); v.x[2] = __uint_as_float(u.z); v.x[3] = __uint_as_float(u.w); }
    else { v.x[0] = bflo(u.x); v.x[1] = bfhi(u.x); v.x[2] = bflo(u.y); v.x[3] = bfhi(u.y); v.x[4] = bflo(u.z); v.x[5] = bfhi(u.z); v.x[6] = bflo(u.w); v.x[7] = bfhi(u.w); }
    return v;
  }
  __device__ __forceinline__ static float largest(const Vec& v) {
    float x = v.x[0];
#pragma unroll
    for (uint32_t e = 1; e < N; ++e) x = fmaxf(x, v.x[e]);
    return x;
  }
  __device__ __forceinline__ uint4 raw(uint32_t i, uint32_t end) const {      // (rows are padded to whole vectors)
    constexpr uint32_t none = N == 4 ? 0xFF800000u : 0xFF80FF80u;
    return i < end ? *reinterpret_cast<const uint4*>(row + i) : make_uint4(none, none, none, none);
  }
  __device__ __forceinline__ uint32_t piece() const { return ((vocab + SM_WAVES - 1) / SM_WAVES + STEP - 1) / STEP * STEP; }
  __device__ __forceinline__ Vec cleaned(Vec v, uint32_t at, uint32_t i) const {
    if (at + STEP > vocab) {          // the row's end: the last vector may go beyond it
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) v.x[e] = i + e < vocab ? v.x[e] : -INFINITY;
    }
    if (infinite) {
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) v.x[e] = v.x[e] == INFINITY ? 0.f : -INFINITY;
    }
    return v;
  }
  // Elements `first` (a multiple of N) to `end`, by one wavefront: f(index of the lane's first value, values).  Four vectors of a lane are on the way ahead of the one in use.
  template <typename F> __device__ __forceinline__ void read(uint32_t first, uint32_t end, F&& f) const {
    const uint32_t lane = threadIdx.x & 63;
    if (first >= end) return;
    uint32_t i = first + lane * N;
    uint4 a = raw(i, end), b = raw(i + STEP, end), c = raw(i + 2 * STEP, end), d = raw(i + 3 * STEP, end);
#pragma unroll 1
    for (uint32_t at = first; at < end; at += STEP, i += STEP) {
      const Vec v = cleaned(values(a), at, i);
      a = b;
      b = c;
      c = d;
      d = raw(i + 4 * STEP, end);
      f(i, v);
    }
  }
  // A part of one wavefront's piece, by any wavefront: a vector for each lane from LDS, where it is there.
  template <typename F> __device__ __forceinline__ void again(uint32_t first, uint32_t end, uint32_t piece_of, F&& f) const {
    const uint32_t lane = threadIdx.x & 63, j = (first - piece_of * piece()) / STEP;
    if (first >= end || end - first > STEP || j >= SM_HELD) return read(first, end, f);
    f(first + lane * N, cleaned(values(held[(piece_of * SM_HELD + j) * 64 + lane]), first, first + lane * N));
  }
  // The whole row.  FIRST: the first time, when the vectors come into LDS.
  template <bool FIRST, typename F> __device__ __forceinline__ void walk(F&& f) const {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = wave * piece(), end = std::min(first + piece(), vocab);
    uint4* mine = held + wave * SM_HELD * 64 + lane;
    if constexpr (FIRST) {
      // (eight vectors of a lane on the way: a row of 50000 bf16 logits has seven)
      uint32_t i = first + lane * N, j = 0;
      uint4 next[8];
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u) next[u] = raw(i + u * STEP, end);
#pragma unroll 1
      for (uint32_t at = first; at < end; at += 8 * STEP) {
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u, i += STEP, ++j) {
          if (at + u * STEP >= end) break;
          const uint4 now = next[u];
          next[u] = raw(i + 8 * STEP, end);
          if (j < SM_HELD) mine[j * 64] = now;
          f(i, cleaned(values(now), at + u * STEP, i));
        }
      }
    } else {
      // (the first ones that are read again are asked for in front of those in LDS)
      const uint32_t again = first + SM_HELD * STEP;
      uint32_t i = again + lane * N;
      uint4 a = raw(i, end), b = raw(i + STEP, end), c = raw(i + 2 * STEP, end), d = raw(i + 3 * STEP, end);
      const uint32_t till = std::min(end, again);
      if (first < till) {
        uint32_t k = first + lane * N;
        uint4 u = mine[0];
#pragma unroll 1
        for (uint32_t at = first, j = 1; at < till; at += STEP, k += STEP, ++j) {
          const Vec v = cleaned(values(u), at, k);
          if (j < SM_HELD) u = mine[j * 64];
          f(k, v);
        }
      }
#pragma unroll 1
      for (uint32_t at = again; at < end; at += STEP, i += STEP) {
        const Vec v = cleaned(values(a), at, i);
        a = b;
        b = c;
        c = d;
        d = raw(i + 4 * STEP, end);
        f(i, v);
      }
    }
  }
};

// Inclusive sums over a wavefront: within sixteen lanes by row shifts, then the rows' last lanes to the rows behind them.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t sm_dpp(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t sm_dpp(uint64_t x) { return (uint64_t)sm_dpp<CTRL, ROWS>((uint32_t)(x >> 32)) << 32 | sm_dpp<CTRL, ROWS>((uint32_t)x); }
template <typename T>
__device__ __forceinline__ T sm_row_scan(T x) {
  x += sm_dpp<0x111, 0xF>(x);
  x += sm_dpp<0x112, 0xF>(x);
  x += sm_dpp<0x114, 0xF>(x);
  x += sm_dpp<0x118, 0xF>(x);
  return x;
}
template <typename T>
__device__ __forceinline__ T sm_scan(T x) {
  x = sm_row_scan(x);
  x += sm_dpp<0x142, 0xA>(x);
  x += sm_dpp<0x143, 0xC>(x);
  return x;
}
// The largest of a wavefront's, in all lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ float sm_dpp_max(float x) { return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), CTRL, ROWS, 0xF, false))); }
__device__ __forceinline__ float sm_max(float x) {
  x = sm_dpp_max<0x111, 0xF>(x);
  x = sm_dpp_max<0x112, 0xF>(x);
  x = sm_dpp_max<0x114, 0xF>(x);
  x = sm_dpp_max<0x118, 0xF>(x);
  x = sm_dpp_max<0x142, 0xA>(x);
  x = sm_dpp_max<0x143, 0xC>(x);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ uint32_t sm_last(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); }
__device__ __forceinline__ uint64_t sm_lane(uint64_t x, uint32_t l) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), (int)l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, (int)l);
}
__device__ __forceinline__ uint32_t sm_sum(uint32_t x) { return sm_last(sm_scan(x)); }

struct SampleShared {
  union {
    uint64_t bins[SM_BINS];           // counts or sums of probabilities
    struct {                          // (when a list is made its bin is found)
      uint64_t sorted[SM_LIST], weight[SM_LIST];      // by rank; by place among the listed ones' numbers
      uint32_t turn[SM_LIST], number[SM_LIST], rank[SM_LIST];      // as it was listed: its turn in its wavefront; by place
    };
  };
  double table[1024];
  uint64_t order[SM_LIST];            // a listed token's key, turned over, and its number: in this order they are sorted
  uint64_t wave[SM_WAVES];
  uint64_t above;                     // what lies above the bin that was found
  uint64_t part_sum[SM_WAVES];        // of the row's sixteen parts what is left, their tokens and those that equal the least one
  uint32_t part_left[SM_WAVES], part_ties[SM_WAVES];
  uint32_t bin, some[SM_WAVES], more[SM_WAVES];
  float best[SM_WAVES];
  uint32_t listed;
  uint4 held[SM_WAVES * SM_HELD * 64];
};

// What a wavefront's lanes have written to LDS, its other lanes may read.
__device__ __forceinline__ void sm_wait() { __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront"); __builtin_amdgcn_wave_barrier(); __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront"); }

// Sums over the block.  Every thread gets the whole; barriers on both sides.
__device__ __forceinline__ uint32_t sm_count(SampleShared& sh, uint32_t x) {
  x = sm_sum(x);
  if ((threadIdx.x & 63) == 0) sh.some[threadIdx.x >> 6] = x;
  __syncthreads();
  x = sm_row_scan(sh.some[threadIdx.x & 15]);
  __syncthreads();
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 15);
}
// Inclusive sum over the block's threads; *all: over all of them.
__device__ __forceinline__ uint64_t sm_block_scan(SampleShared& sh, uint64_t x, uint64_t* all) {
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const uint64_t upto = sm_scan(x);
  if ((threadIdx.x & 63) == 63) sh.wave[wave] = upto;
  __syncthreads();
  const uint64_t waves = sm_row_scan(sh.wave[threadIdx.x & 15]);
  __syncthreads();
  *all = sm_lane(waves, 15);
  return upto + (wave != 0 ? sm_lane(waves, wave - 1) : 0);
}

// The bin, from the highest on, at which the running sum of the bins, `above` in front, is asked for (asked_of(sum of all bins)(running sum)); sh.above gets that
// of the bins above it.  Returns the sum of all bins.
template <typename A>
__device__ __forceinline__ uint64_t sm_find(SampleShared& sh, uint64_t above, A&& asked_of) {
  constexpr uint32_t PER = SM_BINS / SM_THREADS;
  const uint32_t first = SM_BINS - 1 - PER * threadIdx.x;      // the highest one of this thread's
  uint64_t x[PER], mine = 0, all;
#pragma unroll
  for (uint32_t e = 0; e < PER; ++e) mine += x[e] = sh.bins[first - e];
  if (threadIdx.x == 0) sh.bin = 0;
  const uint64_t upto = sm_block_scan(sh, mine, &all);
  uint64_t at = above + upto - mine;
  auto asked = asked_of(all);
  if (!asked(at) && asked(above + upto)) {       // one thread, or none where all bins together do not reach it
    uint32_t e = 0;
#pragma unroll
    for (uint32_t z = 0; z + 1 < PER; ++z)
      if (e == z && !asked(at + x[z])) { at += x[z]; e = z + 1; }
    sh.bin = first - e;
    sh.above = at;
  }
  __syncthreads();
  return all;
}
__device__ __forceinline__ void sm_clear(SampleShared& sh) {
  for (uint32_t b = threadIdx.x; b < SM_BINS; b += SM_THREADS) sh.bins[b] = 0;
  __syncthreads();
}
__device__ __forceinline__ void sm_add(SampleShared& sh, uint32_t bin, uint64_t x) { atomicAdd((unsigned long long*)&sh.bins[bin], (unsigned long long)x); }

struct MinP { double mass; float logit; };

template <typename E>
struct Sampler {
  static constexpr uint32_t N = SampleRow<E>::N, STEP = SampleRow<E>::STEP;
  typedef typename SampleRow<E>::Vec Vec;
  const SampleArgs& a;
  SampleShared& sh;
  SampleRow<E> row;
  SampleScale sc;
  uint32_t i, wave, lane;
  float temperature, top_p, min_p, random, top;
  int32_t top_k;
  MinP least;                         // what min-p asks for

  template <typename F> __device__ __forceinline__ void each(F&& f) const { row.template walk<false>(f); }
  __device__ __forceinline__ void answer(uint32_t token, float l, uint64_t all, uint32_t kept) const {
    a.token[i] = (int32_t)token;
    const double largest = sc.table[0];
    if (a.logprob != nullptr) a.logprob[i] = (float)(((double)l - (double)top) / (double)temperature - log((double)all / largest));
    if (a.kept != nullptr) a.kept[i] = (int32_t)kept;
  }
  __device__ __forceinline__ double goal(uint64_t all) const {
    return (double)(random > 0.f ? std::min(random, 0.99999994f) : 0.f) * (double)all;
  }
  __device__ __forceinline__ double share(uint64_t all) const { return fmax((double)top_p * (double)all, 0.5); }      // what top-p asks for; at least one token

  // Min-p: what is left has at least this logit, which lies a little below the limit (what is clearly below it needs no exponential), and at least this mass.  A limit below those that
  // masses are told from nothing by is one of the logit alone.
  __device__ __forceinline__ MinP limit() const {
    if (!(min_p > 0.f)) return {0.0, -INFINITY};
    if (min_p >= 0x1p-60f) {
      const double below = (double)top + (double)temperature * (log((double)min_p) - 1e-6);
      return {(double)min_p * sc.table[0], (float)(below - fabs(below) * 1e-6)};
    }
    const double cut = (double)top + (double)temperature * log((double)min_p);
    const float f = (float)cut;
    return {0.0, (double)f < cut ? sm_value(sm_key(f) + 1) : f};
  }

  // The least logit (no -inf) whose bin is `bin` or above.  It lies next to the bin's lower end: 64 numbers there are looked at, and where it is not among them (large logits
  // and temperatures) all numbers, 64 at a time.
  __device__ __forceinline__ float least_of(const SampleSteps& steps, uint32_t bin) const {
    auto reaches = [&](uint32_t key) { return SampleSteps::bin(steps.of(sm_value(key)).n) >= bin; };
    uint32_t lo = kKeyNone, hi = sm_key(top);      // hi's bin is the highest one, lo's (if any) is not asked for
    const float end = (float)(steps.top + ((double)((int)(bin - (SM_BINS - 1)) * 16) - 0.5) / steps.per);
    const uint32_t near_end = sm_key(fminf(fmaxf(end, -3.4028235e38f), top));
    if (near_end > lo + 64 && near_end < hi - 64) {
      const uint64_t f = __ballot(reaches(near_end - 32 + lane));
      if ((f & 1) == 0 && f != 0) return sm_value(near_end - 32 + (uint32_t)__ffsll((unsigned long long)f) - 1);
    }
    while (hi - lo > 1) {
      const uint64_t step = ((uint64_t)(hi - lo) + 63) / 64, size = hi - lo;
      const uint32_t at = lo + (uint32_t)std::min(step * (lane + 1), size);
      const int f = __ffsll((unsigned long long)__ballot(reaches(at))) - 1;
      hi = lo + (uint32_t)std::min(step * (uint64_t)(f + 1), size);
      lo += (uint32_t)(step * (uint64_t)f);
    }
    return sm_value(hi);
  }

  // Adds a vector's tokens with logits from `low` on, and of those what min-p leaves: a lane's sum, a wavefront's number.
  struct Sums { uint64_t sum = 0; uint32_t left = 0; };
  __device__ __forceinline__ void weigh(const Vec& v, float low, Sums& to) const {
    uint64_t in[N], some = 0;
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) some |= in[e] = __ballot(v.x[e] >= low);
    if (some == 0) return;
    double y[N];                                   // (all of them at once: one by one each would wait for its table entry)
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) y[e] = sc.scaled(sc.steps.of(v.x[e] >= low ? v.x[e] : -INFINITY));
    if (least.mass > 0.0) {
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        in[e] &= __ballot(!(y[e] < least.mass));
        y[e] = y[e] < least.mass ? 0.0 : y[e];
      }
    }
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) {
      to.sum += SampleScale::raw(y[e]);
      to.left += (uint32_t)__popcll(in[e]);
    }
    to.sum -= N * SampleScale::kRaw;
  }

  // Lists the tokens with logits from `low` up to below `high`, in no order, and ranks them.  Returns how many there are, more than SM_LIST if they do not fit.  WEIGH: and adds up
  // those from `high` on, by parts of the row.
  template <bool WEIGH> __device__ __forceinline__ uint32_t list(float low, float high) {
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    Sums above;
    uint32_t listed = 0;                           // by this wavefront, which comes to them in the order of their numbers
    each([&](uint32_t first, const Vec& v) {
      if (!__any(row.largest(v) >= low)) return;   // (of most vectors; NaN is not the largest of numbers)
      if constexpr (WEIGH) weigh(v, fmaxf(high, least.logit), above);
      uint32_t mine = 0;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) mine |= v.x[e] >= low && v.x[e] < high ? 1u << e : 0u;
      const uint32_t upto = sm_scan((uint32_t)__popc(mine)), n = sm_last(upto), before = upto - (uint32_t)__popc(mine);
      if (n == 0) return;
      uint32_t to = 0;                             // the wavefront's places, one request for all of them
      if (lane == 0) to = atomicAdd(&sh.listed, n);
      to = (uint32_t)__builtin_amdgcn_readfirstlane((int)to) + before;
      uint32_t turn = listed + before;
      for (; mine != 0; mine &= mine - 1, ++to, ++turn) {
        const uint32_t e = (uint32_t)__ffs((int)mine) - 1;
        float x = v.x[0];
#pragma unroll
        for (uint32_t z = 1; z < N; ++z) x = e == z ? v.x[z] : x;
        if (to < SM_LIST) {
          sh.order[to] = (uint64_t)(~sm_key(x)) << 32 | (first + e);
          sh.turn[to] = turn;
        }
      }
      listed += n;
    });
    if constexpr (WEIGH) {
      const uint64_t sum = sm_scan(above.sum);
      if (lane == 63) {
        sh.part_sum[wave] = sum;
        sh.part_left[wave] = above.left;
        sh.part_ties[wave] = 0;
      }
    }
    if (lane == 0) sh.some[wave] = listed;
    __syncthreads();
    const uint32_t m = sh.listed;
    if (m <= SM_LIST) rank(m);
    return m;
  }
  // Ranks the list, by falling logits and rising numbers.  Beside its logit an entry gets in the place of its number the place among the listed ones' numbers, which is of the same
  // order.  sorted[rank]: the entry; number[place].
  __device__ __forceinline__ void rank(uint32_t m) {
    const uint32_t t = threadIdx.x;
    uint64_t x = ~0ull;
    if (t < m) {
      const uint32_t at = (uint32_t)sh.order[t];
      uint32_t place = sh.turn[t];
#pragma unroll
      for (uint32_t w = 0; w + 1 < SM_WAVES; ++w) place += at >= (w + 1) * row.piece() ? sh.some[w] : 0;
      x = sh.order[t] >> 32 << 32 | place;
      sh.number[place] = at;
    }
    if (m <= SM_COUNTED) {
      // Every entry counts those in front of it, a share of the list for each of the threads that it gets.  (One row, top-k 200: 15.7 us so, 18.7 sorted; 256 rows, 300: 26.2 and 26.8, 400, some 500 listed: 29.1 and 27.0.)
      if (t < m) {
        sh.order[t] = x;
        sh.rank[t] = 0;
      }
      __syncthreads();
      uint32_t per = 1;                            // entries, as a power of two
      while (per < m) per <<= 1;
      const uint32_t mine = t & (per - 1), part = t / per, parts = SM_THREADS / per;
      if (mine < m) {
        const uint32_t size = (m + parts - 1) / parts, end = std::min(m, (part + 1) * size);
        x = sh.order[mine];
        uint32_t before = 0;
#pragma unroll 4
        for (uint32_t j = part * size; j < end; ++j) before += sh.order[j] < x ? 1u : 0u;
        if (before != 0) atomicAdd(&sh.rank[mine], before);
      }
      __syncthreads();
      if (t < m) sh.sorted[sh.rank[t]] = x;
    } else {
      x = sorted_one(x, m <= SM_LIST / 2 ? SM_LIST / 2 : SM_LIST);
      if (t < m) sh.sorted[t] = x;
    }
    __syncthreads();
  }
  // A bitonic sort of the first `all` threads' entries (a power of two): partners in other wavefronts exchange through LDS, others by shuffles, in the same sixteen by moves within them.
  __device__ __forceinline__ uint64_t sorted_one(uint64_t x, uint32_t all) {
    const uint32_t t = threadIdx.x;
#pragma unroll 1
    for (uint32_t size = 2; size <= all; size <<= 1) {
      auto take = [&](uint64_t y, uint32_t by) {
        const bool small = ((t & by) == 0) == ((t & size) == 0);
        x = (x < y) == small ? x : y;
      };
      auto far = [&](uint32_t by) { return (uint64_t)(uint32_t)__shfl_xor((uint32_t)(x >> 32), by, 64) << 32 | (uint32_t)__shfl_xor((uint32_t)x, by, 64); };
#pragma unroll 1
      for (uint32_t by = size >> 1; by >= 64; by >>= 1) {
        sh.weight[t] = x;
        __syncthreads();
        const uint64_t y = sh.weight[t ^ by];
        __syncthreads();
        take(y, by);
      }
      if (size >= 64) take(far(32), 32);
      if (size >= 32) take(far(16), 16);
      if (size >= 16) take(sm_dpp<0x128, 0xF>(x), 8);                        // sixteen turned by eight
      if (size >= 8) take(sm_dpp<0x1B, 0xF>(sm_dpp<0x141, 0xF>(x)), 4);      // 7 - i of eight, then 3 - i of four
      if (size >= 4) take(sm_dpp<0x4E, 0xF>(x), 2);                          // 2 3 0 1 of four
      take(sm_dpp<0xB1, 0xF>(x), 1);                                         // 1 0 3 2
    }
    return x;
  }
  __device__ __forceinline__ uint32_t ranked_key(uint32_t rank) const { return ~(uint32_t)(sh.sorted[rank] >> 32); }

  // The token, where the list holds all that a top-k leaves (and some that it does not).
  __device__ __forceinline__ void draw_from_list(uint32_t m) {
    const uint32_t r = threadIdx.x;
    const bool alone = m <= 64;                    // one wavefront has them all and waits for nobody (one row, top-k 50: 13.1 -> 11.9 us)
    if (alone && wave != 0) return;
    auto scan = [&](uint64_t x, uint64_t* all) {
      if (!alone) return sm_block_scan(sh, x, all);
      const uint64_t upto = sm_scan(x);
      *all = sm_lane(upto, 63);
      return upto;
    };
    const double y = r < m ? sc.scaled(sc.steps.of(sm_value(ranked_key(r)))) : 0.0;
    const uint64_t mass = SampleScale::whole(y);
    bool left = r < std::min(m, (uint32_t)top_k);
    if (top_p < 1.f) {
      uint64_t all;
      const uint64_t upto = scan(left ? mass : 0, &all);
      left = left && (double)(upto - mass) < share(all);
    }
    left = left && !(y < least.mass) && sm_value(ranked_key(r)) >= least.logit;
    if (r < m) {
      const uint32_t place = (uint32_t)sh.sorted[r];
      sh.weight[place] = left ? mass : 0;
      sh.rank[place] = r;
    }
    const uint32_t kept = alone ? sm_sum(left ? 1u : 0u) : sm_count(sh, left ? 1u : 0u);      // (its barriers stand behind the weights too)
    if (alone) sm_wait();
    const uint64_t mine = r < m ? sh.weight[r] : 0;
    uint64_t all;
    const uint64_t upto = scan(mine, &all);
    const double target = goal(all);
    if (!((double)(upto - mine) > target) && (double)upto > target) answer(sh.number[r], sm_value(ranked_key(sh.rank[r])), all, kept);
  }

  // The least key that is left and how many of those equal to it, from the keys' bits: for top-k, or by MASS for top-p of what `least` and `equal` leave so far.
  template <bool MASS>
  __device__ __forceinline__ void by_bits(uint32_t& least, uint32_t& equal) {
    uint32_t known = 0, mask = 0;
    uint64_t above = 0;
    double target = 0.0;
#pragma unroll 1
    for (int level = 0; level < 3; ++level) {
      const int low = level == 0 ? 21 : level == 1 ? 10 : 0;
      const uint32_t bits = level == 2 ? 1023u : 2047u;
      sm_clear(sh);
      each([&](uint32_t, const Vec& v) {
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) {
          const uint32_t key = sm_key(v.x[e]);
          if (key > least && (key & mask) == known) sm_add(sh, key >> low & bits, MASS ? sc.mass(v.x[e]) : 1ull);
        }
      });
      if (MASS && threadIdx.x == 0 && equal != 0 && (least & mask) == known) sm_add(sh, least >> low & bits, equal * sc.mass(sm_value(least)));
      __syncthreads();
      const int at_level = level;
      sm_find(sh, above, [&](uint64_t all) {
        if (at_level == 0) target = MASS ? share(all) : (double)top_k;
        return [&](uint64_t sum) { return (double)sum >= target; };
      });
      above = sh.above;
      known |= sh.bin << low;
      mask |= bits << low;
      __syncthreads();
    }
    if constexpr (!MASS) {
      least = known;
      equal = (uint32_t)top_k - (uint32_t)above;
    } else {
      // of those equal to `known` as many as it takes
      const uint64_t w = sc.mass(sm_value(known));
      uint64_t need = 1;
      if (w != 0) {
        need = (uint64_t)fmax((target - (double)above) / (double)w, 1.0);
        while (need > 1 && (double)(above + (need - 1) * w) >= target) --need;
        while ((double)(above + need * w) < target) ++need;
      }
      equal = (uint32_t)std::min<uint64_t>(need, known == least ? equal : row.vocab);
      least = known;
    }
  }

  // The token, by walking the row: logits above that of `key` are left, and the first `equal` of those that are equal to it.  The sums of sixteen pieces say on which one the
  // random number falls, this one's sixteen pieces go on, down to a vector for a lane.  The equal ones weigh all the same, so pieces only count them.  GIVEN: the first sums are there, the equal ones in them.
  template <bool GIVEN> __device__ __forceinline__ void draw_from_row(uint32_t key, uint32_t equal) {
    const float bound = sm_value(key);
    const double tie = sc.scaled(sc.steps.of(bound));
    if (tie < least.mass || bound < least.logit) equal = 0;
    const uint64_t tie_mass = SampleScale::whole(tie);
    const float low = fmaxf(sm_value(key + 1), least.logit);
    uint32_t lo = 0, hi = row.vocab, ties_before = 0, kept = 0, piece = 0;
    uint64_t before = 0, all = 0;
    double target = 0.0;
    for (bool whole = true;; whole = false) {
      const uint32_t per = ((hi - lo + SM_WAVES - 1) / SM_WAVES + STEP - 1) / STEP * STEP, first = lo + wave * per, end = std::min(first + per, hi);
      const bool mine = lane < SM_WAVES, given = GIVEN && whole;      // a piece to a lane
      uint32_t equals = 0, more = 0, seen;
      uint64_t here = 0;
      if (given) {
        if (mine) {
          here = sh.part_sum[lane];
          equals = sh.part_ties[lane];
          more = sh.part_left[lane];
        }
        seen = sm_scan(equals) - equals;
      } else {
        Sums sums;
        uint32_t ties = 0;
        auto add = [&](uint32_t, const Vec& v) {
          if (equal != 0) {
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) ties += (uint32_t)__popcll(__ballot(v.x[e] == bound));
          }
          weigh(v, low, sums);
        };
        if (!GIVEN && whole) each(add); else row.again(first, end, piece, add);
        const uint64_t sum = sm_scan(sums.sum);
        if (lane == 63) {
          sh.wave[wave] = sum;
          sh.some[wave] = ties;
          sh.more[wave] = sums.left;
        }
        __syncthreads();
        if (mine) {
          equals = sh.some[lane];
          more = sh.more[lane];
        }
        seen = ties_before + sm_scan(equals) - equals;
        const uint32_t left = std::min(equals, equal - std::min(equal, seen));
        if (mine) here = sh.wave[lane] + tie_mass * left;
        more += left;
      }
      const uint64_t upto = before + sm_scan(here);
      if (whole) {
        all = sm_lane(upto, 63);
        kept = sm_sum(more);
        target = goal(all);
      }
      const uint64_t beyond = __ballot(mine && (double)upto > target);      // the first piece at whose end the sum exceeds the target
      const uint32_t won = beyond != 0 ? (uint32_t)__ffsll((unsigned long long)beyond) - 1 : SM_WAVES - 1;
      before = sm_lane(upto - here, won);
      ties_before = (uint32_t)__builtin_amdgcn_readlane((int)seen, (int)won);
      if (whole) piece = won;
      lo += won * per;
      hi = std::min(lo + per, hi);
      if (per == STEP) break;
      if (!given) __syncthreads();                 // nobody reads this turn's sums any more
    }
    if (wave != 0) return;
    row.again(lo, hi, piece, [&](uint32_t i, const Vec& v) {
      uint64_t x[N], sum = 0;
      uint32_t mine = 0;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) mine += v.x[e] == bound ? 1u : 0u;
      uint32_t rank = ties_before + sm_scan(mine) - mine;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        const double y = sc.scaled(sc.steps.of(v.x[e]));
        x[e] = v.x[e] >= low && !(y < least.mass) ? SampleScale::whole(y) : 0;
        if (v.x[e] == bound && rank++ < equal) x[e] = tie_mass;
        sum += x[e];
      }
      uint64_t at = before + sm_scan(sum);
      const uint64_t hits = __ballot((double)at > target);
      if (lane != (uint32_t)__ffsll((unsigned long long)hits) - 1) return;
      uint32_t e = N - 1;
      float l = v.x[N - 1];
#pragma unroll
      for (uint32_t z = N; z-- > 0;) {              // the first at which the sum exceeds it, looked at from the last on
        if ((double)at > target) { e = z; l = v.x[z]; }
        at -= x[z];
      }
      answer(i + e, l, all, kept);
    });
  }

  __device__ __forceinline__ void run() {
    sh.table[threadIdx.x] = ldexp(sm_exp2((double)threadIdx.x * (1.0 / 1024.0)), (int)a.shift);
    for (uint32_t b = threadIdx.x; b < SM_BINS; b += SM_THREADS) sh.bins[b] = 0;      // (for the first histogram; a barrier comes with the largest logit)
    // (what the temperature gives, while the row is on its way)
    sc.table = sh.table;
    sc.steps.per = 1.44269504088896340736 * 1024.0 / (double)temperature;
    const double near_per = 65504.0 / (double)fmaxf(40.f * temperature, 64.f);
    // the largest logit, and where the first vector with it lies; and this thread's largest
    float mine = -INFINITY;
    uint32_t at = 0xFFFFFFFFu;
    row.template walk<true>([&](uint32_t first, const Vec& v) {
      const float x = row.largest(v);
      if (x > mine) { mine = x; at = first; }
    });
    top = sm_max(mine);
    if (lane == 0) sh.best[wave] = top;
    __syncthreads();
    top = sm_max(sh.best[lane & 15]);
    if (top == -INFINITY || !(temperature > 0.f)) {
      at = mine == top && top > -INFINITY ? at : 0xFFFFFFFFu;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) at = std::min(at, (uint32_t)__shfl_xor(at, o, 64));
      if (lane == 0) sh.some[wave] = at;
      __syncthreads();
      if (threadIdx.x != 0) return;
      for (uint32_t w = 0; w < SM_WAVES; ++w) at = std::min(at, sh.some[w]);
      const bool none = at == 0xFFFFFFFFu;
      if (!none) {
        const Vec v = row.values(row.raw(at, row.vocab));
        uint32_t e = N - 1;
#pragma unroll
        for (uint32_t z = N - 1; z-- > 0;) e = v.x[z] == top ? z : e;
        at += e;
      }
      a.token[i] = none ? -1 : (int32_t)at;
      if (a.logprob != nullptr) a.logprob[i] = none ? -INFINITY : 0.f;
      if (a.kept != nullptr) a.kept[i] = none ? 0 : 1;
      return;
    }
    if (top == INFINITY) {
      row.infinite = true;
      mine = mine == INFINITY ? 0.f : -INFINITY;
      top = 0.f;
    }
    sc.steps.top = (double)top;
    least = limit();
    // For counts, logits are divided into steps near the largest one, whatever the temperature.
    const SampleSteps near = {(double)top, near_per};
    uint32_t key = kKeyNone, equal = 0;          // the least logit that is left, and how many of those that equal it
    bool by_k = top_k > 0 && (uint32_t)top_k < row.vocab;
    if (by_k) {
      if ((uint32_t)top_k <= SM_FEW) {
        // at least top_k tokens reach the top_k-th of the threads' own largest (or there are fewer threads with tokens: the lowest bin, all tokens)
        if (mine > -INFINITY) sm_add(sh, SampleSteps::bin(near.of(mine).n), 1);
        __syncthreads();
        sm_find(sh, 0, [&](uint64_t) { return [&](uint64_t sum) { return sum >= (uint64_t)top_k; }; });
        // (the bin's lower end, a little below where it is; the first one also holds all that is further away)
        const double end = (double)top + ((double)((int)sh.bin - (int)(SM_BINS - 1)) * 16.0 - 1.0) / near.per;
        const uint32_t m = list<false>(sh.bin > 1 ? fmaxf((float)(end - fabs(end) * 1e-6), -3.4028235e38f) : -3.4028235e38f, INFINITY);
        if (m <= SM_LIST) return draw_from_list(m);
      }
      if ((uint32_t)top_k <= SM_FEW) {
        __syncthreads();
        sm_clear(sh);
      }
      each([&](uint32_t, const Vec& v) {
#pragma unroll
        for (uint32_t e = 0; e < N; ++e)
          if (v.x[e] > -INFINITY) sm_add(sh, SampleSteps::bin(near.of(v.x[e]).n), 1);
      });
      __syncthreads();
      const uint64_t some = sm_find(sh, 0, [&](uint64_t) { return [&](uint64_t sum) { return sum >= (uint64_t)top_k; }; });
      by_k = some > (uint64_t)(uint32_t)top_k;
      if (by_k) {
        const uint32_t bin = sh.bin, above = (uint32_t)sh.above, here = (uint32_t)sh.bins[bin];
        const bool whole = above + here <= SM_LIST;
        uint32_t m = SM_LIST + 1;
        if (whole || here <= SM_LIST) m = list<false>(least_of(near, bin), whole || bin + 1 == SM_BINS ? INFINITY : least_of(near, bin + 1));
        if (m <= SM_LIST && whole) return draw_from_list(m);
        if (m <= SM_LIST) {
          const uint32_t need = (uint32_t)top_k - above;                     // of the listed ones, in their order
          key = ranked_key(need - 1);
          equal = sm_count(sh, threadIdx.x < need && ranked_key(threadIdx.x) == key ? 1u : 0u);
        } else {
          by_bits<false>(key, equal);
        }
        if (top_p < 1.f) by_bits<true>(key, equal);
      }
    }
    if (!by_k && top_p < 1.f) {
      if (top_k > 0 && (uint32_t)top_k < row.vocab) {      // (a histogram was there before)
        __syncthreads();
        sm_clear(sh);
      }
      // Below this logit a probability is nothing as a whole number of 2^-s.
      const double nothing = (double)top - (double)temperature * (0.693147180559945309417 * (a.shift + 1));
      const float weightless = (float)(nothing - fabs(nothing) * 1e-6 - (double)temperature * 1e-6);
      // Those of nothing, no tokens or far away, add it to a bin for each lane: additions to one bin wait for each other.  (One row of which 99 in 100 are none 65 -> 36 us; at a temperature of 0.1 57 -> 16.5,
      // since most vectors are passed over; rows without such 0.5 to 1 us more.)
      const double last = -65504.0 + 16.0 * lane;
      each([&](uint32_t, const Vec& v) {
        if (!__any(row.largest(v) >= weightless)) return;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) {
          const SampleStep x = sc.steps.of(v.x[e], last);
          sm_add(sh, SampleSteps::bin(x.n), SampleScale::whole(sc.scaled(x)));
        }
      });
      __syncthreads();
      double target = 0.0;
      sm_find(sh, 0, [&](uint64_t sum) {
        target = share(sum);
        return [&](uint64_t x) { return (double)x >= target; };
      });
      const uint32_t bin = sh.bin;
      const uint64_t above = sh.above;
      const float low = least_of(sc.steps, bin);
      const uint32_t m = list<true>(low, bin + 1 == SM_BINS ? INFINITY : least_of(sc.steps, bin + 1));
      if (m <= SM_LIST) {
        const uint32_t r = threadIdx.x, k = r < m ? ranked_key(r) : kKeyNone, at = r < m ? sh.number[(uint32_t)sh.sorted[r]] : 0;
        const double y = r < m ? sc.scaled(sc.steps.of(sm_value(k))) : 0.0;
        const uint64_t mass = SampleScale::whole(y);
        uint64_t sum;
        const uint64_t upto = above + sm_block_scan(sh, mass, &sum);
        const bool left = r < m && (double)(upto - mass) < target;
        const uint32_t need = sm_count(sh, left ? 1u : 0u);
        key = ranked_key(need - 1);
        equal = sm_count(sh, left && k == key ? 1u : 0u);
        if (left && !(y < least.mass) && sm_value(k) >= least.logit) {
          atomicAdd((unsigned long long*)&sh.part_sum[at / row.piece()], (unsigned long long)mass);
          atomicAdd(&sh.part_left[at / row.piece()], 1u);
        }
        if (r < m && k == key) atomicAdd(&sh.part_ties[at / row.piece()], 1u);
        __syncthreads();
        return draw_from_row<true>(key, equal);
      }
      by_bits<true>(key, equal);
    }
    draw_from_row<false>(key, equal);
  }
};

template <typename E>
__global__ __launch_bounds__(SM_THREADS) void sample_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  const uint32_t i = blockIdx.x;
  Sampler<E> s = {a, sh, {(const E*)a.logits + (size_t)i * a.ld, sh.held, a.vocab, false}, {}, i, threadIdx.x >> 6, threadIdx.x & 63,
                  a.temperature_list != nullptr ? a.temperature_list[i] : a.temperature, a.top_p_list != nullptr ? a.top_p_list[i] : a.top_p,
                  std::min(a.min_p_list != nullptr ? a.min_p_list[i] : a.min_p, 1.f), a.random != nullptr ? a.random[i] : 0.f, 0.f, a.top_k_list != nullptr ? a.top_k_list[i] : a.top_k};
  s.run();
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
  while (1ull << (62 - x.shift) < a->vocab) --x.shift;
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
