// Rotations by position: a sif_rope as the kernels see it (checked), and the sines and cosines of its angles.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include "common.h"
#include "launch.h"

namespace sif {

// A kernel argument: the table is read from the argument itself, so a launch needs no memory of its own.
struct RopeView {
  uint32_t interleaved, half;        // half: pairs
  double magnitude;
  double turns[128];
};

// Checks a rotation for heads of d_head and fills in the view; `who` begins the error's text.
sif_status rope_check(const char* who, const sif_rope* r, uint32_t d_head, RopeView* out);

// m cos a and m sin a, a = 2 pi times the fraction of pos * turns.  In fp32 a far position's angle would be off by whole turns' 2^-24th (at
// 10^6 by a tenth of a radian), so turns are reduced in 64 bits, to an eighth of a turn; on +-pi/4 the Taylor series to x^9 and x^10 (fp32: the next terms are
// below 2e-9) and to x^17 and x^18 (64 bits: below 1e-19).
template <typename T> struct CosSin { T c, s; };
template <typename T>
__device__ __forceinline__ CosSin<T> rope_cos_sin(const RopeView& r, double pos, uint32_t pair) {
  double t = pos * r.turns[pair];
  t -= rint(t);
  const double q = rint(4.0 * t);
  const T x = (T)(6.283185307179586476925 * fma(q, -0.25, t)), y = x * x;
  T s, c;
  if constexpr (sizeof(T) == 4) {
    s = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f) * x;
    c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  } else {
    s = 1.0 / 355687428096000.0;
    s = fma(y, s, -1.0 / 1307674368000.0);
    s = fma(y, s, 1.0 / 6227020800.0);
    s = fma(y, s, -1.0 / 39916800.0);
    s = fma(y, s, 1.0 / 362880.0);
    s = fma(y, s, -1.0 / 5040.0);
    s = fma(y, s, 1.0 / 120.0);
    s = fma(y, s, -1.0 / 6.0);
    s = fma(y, s, 1.0) * x;
    c = -1.0 / 6402373705728000.0;
    c = fma(y, c, 1.0 / 20922789888000.0);
    c = fma(y, c, -1.0 / 87178291200.0);
    c = fma(y, c, 1.0 / 479001600.0);
    c = fma(y, c, -1.0 / 3628800.0);
    c = fma(y, c, 1.0 / 40320.0);
    c = fma(y, c, -1.0 / 720.0);
    c = fma(y, c, 1.0 / 24.0);
    c = fma(y, c, -0.5);
    c = fma(y, c, 1.0);
  }
  const T m = (T)r.magnitude;
  s *= m;
  c *= m;
  const int n = (int)q & 3;
  const T a = n & 1 ? s : c, b = n & 1 ? c : s;
  return {n == 1 || n == 2 ? -a : a, n & 2 ? -b : b};
}

__device__ __forceinline__ uint32_t rope_pair(uint32_t w, const CosSin<float>& cs, float back) {      // one pair in one word
  const float x = bflo(w), y = bfhi(w), s = cs.s * back;
  return pack_bf2(fmaf(x, cs.c, -(y * s)), fmaf(y, cs.c, x * s));
}
__device__ __forceinline__ void rope_two(uint32_t& u, uint32_t& v, const CosSin<float>& p, const CosSin<float>& q, float back) {      // two pairs, firsts in u, seconds in v
  const float x0 = bflo(u), x1 = bfhi(u), y0 = bflo(v), y1 = bfhi(v), s0 = p.s * back, s1 = q.s * back;
  u = pack_bf2(fmaf(x0, p.c, -(y0 * s0)), fmaf(x1, q.c, -(y1 * s1)));
  v = pack_bf2(fmaf(y0, p.c, x0 * s0), fmaf(y1, q.c, x1 * s1));
}
// Eight pairs of a row of a head: elements a .. a + 7 and b .. b + 7 of it, in halves the pairs' first and second elements, interleaved
// sixteen elements in a row.  cs: the pairs' cosines and sines; back = -1 turns back.
__device__ __forceinline__ void rope_turn8(bool interleaved, const CosSin<float>* cs, float back, uint4& a, uint4& b) {
  if (interleaved) {
    a.x = rope_pair(a.x, cs[0], back); a.y = rope_pair(a.y, cs[1], back); a.z = rope_pair(a.z, cs[2], back); a.w = rope_pair(a.w, cs[3], back);
    b.x = rope_pair(b.x, cs[4], back); b.y = rope_pair(b.y, cs[5], back); b.z = rope_pair(b.z, cs[6], back); b.w = rope_pair(b.w, cs[7], back);
  } else {
    rope_two(a.x, b.x, cs[0], cs[1], back);
    rope_two(a.y, b.y, cs[2], cs[3], back);
    rope_two(a.z, b.z, cs[4], cs[5], back);
    rope_two(a.w, b.w, cs[6], cs[7], back);
  }
}

}  // namespace sif
