// Attention with a sliding window of recent keys and a few first keys (sinks) that stay visible, forward and backward, with fewer key
// heads than query heads if wanted.  Single launches: no registered model contains them, so they carry no monitor record.
//
//   key j is visible to the query at position p  iff  j <= p  and  (window = 0  or  p - j < window  or  j < sinks)
//   forward    o = softmax(scale q k^T | visible) v,  lse = log sum exp
//   backward   delta = rowsum(do .* o),  P = exp(scale q k^T - lse),  dS = scale P .* (do v^T - delta)
//              dq = dS k (a block per query rows),  dk = dS^T q,  dv = P^T do (a block per key rows, summed over the query heads of
//              the key head in registers); P is recomputed in both, no atomics
//
// Products, operands and LDS tiles are those of attention.hip.  A block meets only the tiles that one of its rows sees: the sinks', then
// from the first key of its first row's window to its last row.  Those ranges begin and end exactly there and are not rounded to
// tiles, and what a fetch would read past the end is the last row again, so that a key or query that nobody sees is never read.
// Bound by the matrix and the vector units together: forward with heads of 128 the first are busy 43 % of a SIMD's cycles,
// the second 50 %, backward 42 and 42 (dq), 38 and 30 (dk, dv), and there is little
// overlap between the two wavefronts of a SIMD.  8192 rows, 16 query and 4 key heads of 128, window 1024: 84, 114, 150 us, that is 770,
// 850 and 860 TFLOP/s of the products that each kernel needs (a large matrix product reaches 1390 on this card); the sinks' two launches 22.
// (So once passes have followed one another for a while; the first dozen run at a lower clock and take 99, 134 and 189 us.  What is compared
// below, one form of a kernel with another, was measured in such short runs, both sides alike.)
#include <math.h>
#include <algorithm>

#include "attn_tiles.h"
#include "common.h"
#include "launch.h"

namespace sif {

constexpr int kSchedMfma = 0x8, kSchedLds = 0x100;      // instruction classes of the scheduling groups (LDS: reads)
constexpr float kLog2e = 1.44269504088896f, kLn2 = 0.693147180559945f;

// --- LDS tiles of this file ---
// A fetch instruction writes 1 KB of consecutive LDS: 4 rows of 128 or 8 rows of 64.  Each such group is followed by 16 bytes of nothing,
// and within it the 16-byte chunks of a row are exchanged (by XOR) by the row's place in the group, so that neither read meets a bank
// twice: a 16-byte read serves the lanes 0-3, 12-15, 20-27 of 32 in one cycle and the others in the next, sixteen rows that differ
// modulo 16; the transposing read takes 64 bytes of four rows in its first 32 lanes.  Because the exchange is the same in every group, a
// lane's addresses are few (rows 8, 16, 32 further are immediate offsets) and stay in registers.  (dk and dv of 8192 rows, 16 query and 4
// key heads of 128, window 1024: 330 us with attn_tiles.h's layout, which is free of conflicts for rows of 64 only, 477 with an exchange by
// sixteen different keys, whose addresses do not fit the registers, 185 so.)
constexpr uint32_t kWtGroup = 512 + 8;                     // elements of a group and its gap
template <int DH, int ROWS> constexpr int kWtTile = ROWS * DH / 512 * kWtGroup;
template <int DH> __device__ __forceinline__ uint32_t wt_row(uint32_t row) { return DH == 128 ? (row >> 2) * kWtGroup + (row & 3u) * 128 : (row >> 3) * kWtGroup + (row & 7u) * 64; }
template <int DH> __device__ __forceinline__ uint32_t wt_key(uint32_t row) { return DH == 128 ? (row & 3u) << 2 : (row & 2u) << 1 | ((row >> 2) & 1u) << 1; }

// ROWS rows from row0 on by WAVES wavefronts (this one is number `wave` of them); rows >= limit are row limit - 1 again.  Where none is, a
// lane's offset is the same in every tile and all else is scalar: the vector units have no address to work out.
template <int DH, int ROWS, int WAVES>
__device__ __forceinline__ void wt_fetch(bf16_t* dst, const bf16_t* src, uint32_t ld, uint32_t row0, uint32_t limit, uint32_t wave) {
  typedef __attribute__((address_space(3))) void* lds_void_ptr;
  typedef __attribute__((address_space(1))) const void* global_void_ptr;
  constexpr int CH = DH / 8, RPI = 64 / CH;
  const uint32_t lane = threadIdx.x & 63, in_group = lane / CH, c = (lane % CH) ^ wt_key<DH>(in_group);
  if (row0 + ROWS <= limit) {
    const uint32_t mine = (in_group * ld + c * 8) * 2;                 // bytes; ld < 2^27
#pragma unroll
    for (int i = 0; i < ROWS / (RPI * WAVES); ++i) {
      const uint32_t group = i * WAVES + wave;
      const char* base = reinterpret_cast<const char*>(src + (size_t)(row0 + group * RPI) * ld);
      __builtin_amdgcn_global_load_lds((global_void_ptr)(base + mine), (lds_void_ptr)(dst + group * kWtGroup), 16, 0, 0);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < ROWS / (RPI * WAVES); ++i) {
    const uint32_t group = i * WAVES + wave, row = row0 + group * RPI + in_group, r = row < limit ? row : limit - 1;
    __builtin_amdgcn_global_load_lds((global_void_ptr)(src + (size_t)r * ld + c * 8), (lds_void_ptr)(dst + group * kWtGroup), 16, 0, 0);
  }
}
// A lane's places in a tile, in elements: for operands with row = lane % 32 (+ a multiple of 32) and 8 consecutive d, and for operands
// with row d = lane % 32 whose k elements are tile rows.
template <int DH> struct WtLane {
  uint32_t row[4], col[DH / 32];
  __device__ __forceinline__ WtLane() {
    const uint32_t lane = threadIdx.x & 63, ki = lane & 31, h = lane >> 5, s = lane & 15;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) row[j] = wt_row<DH>(ki) + (((DH == 128 ? j * 4 : j * 2) + h) ^ wt_key<DH>(ki)) * 8;
    const uint32_t r = 4 * h + (s >> 2), d = ((lane >> 4) & 1u) * 16 + 4 * (s & 3u);
#pragma unroll
    for (uint32_t t = 0; t < DH / 32; ++t) col[t] = wt_row<DH>(r) + (((t * 4 + (d >> 3)) ^ wt_key<DH>(r)) * 8) + (d & 7u);
  }
};
// A or B operand: rows base + lane % 32 (base a multiple of 32), d = 16 ks + 8 h ..
template <int DH>
__device__ __forceinline__ bf16x8 wt_frag(const bf16_t* tile, const WtLane<DH>& l, uint32_t base, int ks) {
  const bf16_t* p = tile + wt_row<DH>(base);
  return *reinterpret_cast<const bf16x8*>(DH == 128 ? p + l.row[ks >> 1] + (ks & 1) * 16 : p + l.row[ks]);
}
// A operand of a product that contracts over tile rows: operand row d = 32 t + lane % 32, k elements 0..3 the tile rows kb + 4 h .., 4..7
// the rows kb + 8 + 4 h .. (kb a multiple of 16)
template <int DH>
__device__ __forceinline__ bf16x8 wt_frag_tr(const bf16_t* tile, const WtLane<DH>& l, int t, uint32_t kb) {
  typedef short short4_lds __attribute__((ext_vector_type(4)));
  typedef short short8_v __attribute__((ext_vector_type(8)));
  typedef __attribute__((address_space(3))) short4_lds* lds_ptr;
  const bf16_t* p = tile + wt_row<DH>(kb) + l.col[t];
  const short4_lds lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
  const short4_lds hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + wt_row<DH>(8)));
  const short8_v v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, v);
}

struct WinArgs {
  const bf16_t* q; const bf16_t* k; const bf16_t* v;
  bf16_t* o;
  float* lse;
  const int32_t* starts;
  const bf16_t* d_o;
  bf16_t* dq; bf16_t* dk; bf16_t* dv;
  float* delta;                      // [heads][query rows]
  float* lse2;                       // [heads][query rows], minus the log sum exp in base-2 units
  float* part;                       // sums of the sinks' dk and dv by pieces (null: none), see win_sink_kernel
  uint32_t pieces;
  uint32_t heads, kv_heads, group, hb;      // hb: query heads of one key head that a block works on
  uint32_t batch, sq, sk, window, sinks, rows, rows_q;
  uint32_t ld_q, ld_k, ld_v, ld_o, ld_do, ld_dq, ld_dk, ld_dv;
  float scale;
};

// Where a sequence's rows are.
struct WinSeq { uint32_t q0, k0, nq, nk; };
__device__ __forceinline__ WinSeq win_seq(const WinArgs& a, uint32_t b) {
  if (a.starts == nullptr) return {b * a.sq, b * a.sk, a.sq, a.sk};
  const int32_t top = (int32_t)a.rows, s0 = min(max(a.starts[b], 0), top), s1 = min(max(a.starts[b + 1], s0), top);
  const uint32_t n = min((uint32_t)(s1 - s0), a.sq);
  return {(uint32_t)s0, (uint32_t)s0, n, n};
}

// The keys that rows at positions p0 .. p1 see at all: the first `sinks` (as far as they lie below lo), and lo .. hi - 1.
struct WinSpan { uint32_t lo, hi, sinks; };
__device__ __forceinline__ WinSpan win_span(const WinArgs& a, int32_t p0, int32_t p1, uint32_t nk) {
  WinSpan s;
  s.hi = p1 < 0 ? 0u : min((uint32_t)p1 + 1u, nk);
  s.lo = a.window != 0 && p0 >= 0 && (uint32_t)p0 >= a.window ? (uint32_t)p0 - a.window + 1u : 0u;
  s.sinks = min(a.sinks, s.lo);
  return s;
}

__device__ __forceinline__ float max_over_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// What a wavefront's 32 rows (positions pw .. pw + 31) have to do with keys first .. first + n - 1, of which those below `end` exist.
__device__ __forceinline__ bool win_none(const WinArgs& a, int32_t pw, uint32_t first, uint32_t n, uint32_t end) {
  if (pw + 31 < 0 || first >= end || (int32_t)first > pw + 31) return true;
  return a.window != 0 && (int32_t)(first + n - 1) <= pw - (int32_t)a.window && first >= a.sinks;
}
__device__ __forceinline__ bool win_all(const WinArgs& a, int32_t pw, uint32_t first, uint32_t n, uint32_t end) {
  if (first + n > end || (int32_t)(first + n - 1) > pw) return false;
  return a.window == 0 || (int32_t)first > pw + 31 - (int32_t)a.window || first + n <= a.sinks;
}
__device__ __forceinline__ bool win_sees(const WinArgs& a, int32_t p, uint32_t j, uint32_t end) {
  return j < end && (int32_t)j <= p && (a.window == 0 || (int32_t)j > p - (int32_t)a.window || j < a.sinks);
}

template <int DH> constexpr int kWinKv = DH == 64 ? 128 : 64;        // keys of a tile: two buffers of K and V are 64 KB

// Forward.  Four wavefronts of 32 rows: hb query heads of a key head (1, 2 or 4), 128 / hb rows each, so that the wavefronts of a
// block have nearly the same keys and share them.  (Timing variants at 8192 rows as above, where the whole took 93 us: without the
// exponentials 84, without the fetches after the first 82, without both 71.)
template <int DH>
__global__ __launch_bounds__(AT_THREADS, 2) void win_fwd_kernel(WinArgs a) {
  constexpr int KS = DH / 16, DT = DH / 32, KV = kWinKv<DH>, NT = KV / 32;
  constexpr uint32_t TILE = kWtTile<DH, KV>;
  // (four objects, so that the compiler can tell the buffer that is being filled from the one that is being read: of one, its transposing
  // reads would wait for the fetches under way)
  __shared__ __align__(1024) bf16_t sK0[TILE];
  __shared__ __align__(1024) bf16_t sV0[TILE];
  __shared__ __align__(1024) bf16_t sK1[TILE];
  __shared__ __align__(1024) bf16_t sV1[TILE];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qi = lane & 31, h = lane >> 5;
  const uint32_t units = a.heads / a.hb, b = blockIdx.x / units, head0 = blockIdx.x % units * a.hb, head = head0 + wave % a.hb, kvh = head0 / a.group;
  const WinSeq sq = win_seq(a, b);
  // (the last rows see the most keys where there is no window: their blocks start first)
  const uint32_t per = AT_Q / a.hb, q_blk = (gridDim.y - 1 - blockIdx.y) * per;
  if (q_blk >= sq.nq) return;
  const uint32_t qw = q_blk + wave / a.hb * 32, q = qw + qi;
  const int32_t off = (int32_t)sq.nk - (int32_t)sq.nq, pw = (int32_t)qw + off, p = pw + (int32_t)qi;
  const uint32_t q_end = min(q_blk + per, sq.nq);
  const WinSpan sp = win_span(a, (int32_t)q_blk + off, (int32_t)q_end - 1 + off, sq.nk);
  const bf16_t* kbase = a.k + (size_t)sq.k0 * a.ld_k + kvh * DH;
  const bf16_t* vbase = a.v + (size_t)sq.k0 * a.ld_v + kvh * DH;
  const float c2 = a.scale * kLog2e;
  const WtLane<DH> at;
  const uint32_t sink_tiles = (sp.sinks + KV - 1) / KV, tiles = sink_tiles + (sp.hi > sp.lo ? (sp.hi - sp.lo + KV - 1) / KV : 0u);

  bf16x8 fq[KS];
  {
    const bf16_t* qp = a.q + (size_t)(sq.q0 + (q < sq.nq ? q : sq.nq - 1)) * a.ld_q + head * DH;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) fq[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16 + h * 8);
  }
  floatx16 oacc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[d][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;            // l: of this lane's keys only

  auto first_of = [&](uint32_t t) { return t < sink_tiles ? t * KV : sp.lo + (t - sink_tiles) * KV; };
  auto end_of = [&](uint32_t t) { return t < sink_tiles ? sp.sinks : sp.hi; };
  auto fetch = [&](bf16_t* sK, bf16_t* sV, uint32_t t) {
    wt_fetch<DH, KV, 4>(sK, kbase, a.ld_k, first_of(t), end_of(t), wave);
    wt_fetch<DH, KV, 4>(sV, vbase, a.ld_v, first_of(t), end_of(t), wave);
  };
  // (one body for tiles with and without a mask: of two, each copied all sums on its way in)
  auto turn = [&](const bf16_t* sK, const bf16_t* sV, bf16_t* next_k, bf16_t* next_v, uint32_t t) {
    wait_fetches();
    __syncthreads();                                       // tile t has landed, nobody reads the other buffer any more
    const uint32_t kv0 = first_of(t), end = end_of(t);
    if (t + 1 < tiles) fetch(next_k, next_v, t + 1);
    if (win_none(a, pw, kv0, KV, end)) return;
    floatx16 sacc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (NT > 2 && win_none(a, pw, kv0 + n * 32, 32, end)) {          // (short windows meet such parts often)
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[n][r] = -INFINITY;
        continue;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[n][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sacc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wt_frag<DH>(sK, at, n * 32, ks), fq[ks], sacc[n], 0, 0, 0);
    }
    if constexpr (NT == 2) {                               // the order of this part: operands are read eight products ahead
      __builtin_amdgcn_sched_group_barrier(kSchedLds, KS, 0);
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kSchedLds, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(kSchedMfma, KS, 0);
    }
    if (!win_all(a, pw, kv0, KV, end)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[n][r] = win_sees(a, p, kv0 + n * 32 + (r >> 2) * 8 + h * 4 + (r & 3), end) ? sacc[n][r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[n][r]);
    mx = max_over_halves(mx) * c2;                         // c2 > 0
    // The running maximum follows only where scores pass it by more than 2^8 (or there was none): sums and accumulators are fp32 and
    // the probabilities' rounding is relative, so a maximum that is a little low costs nothing, and the accumulators are seldom scaled.
    if (__any(mx > m_run + 8.0f)) {
      const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d) oacc[d] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (NT > 2 && win_none(a, pw, kv0 + n * 32, 32, end)) continue;
      float pt[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) { pt[r] = __builtin_amdgcn_exp2f(fmaf(sacc[n][r], c2, -m_use)); l_run += pt[r]; }
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const bf16x8 fp = at_pack8(pt, 8 * s2);
#pragma unroll
        for (int d = 0; d < DT; ++d) oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wt_frag_tr<DH>(sV, at, d, n * 32 + 16 * s2), fp, oacc[d], 0, 0, 0);
      }
    }
  };
  if (tiles > 0) fetch(sK0, sV0, 0);
  for (uint32_t t = 0; t < tiles; t += 2) {
    turn(sK0, sV0, sK1, sV1, t);
    if (t + 1 == tiles) break;
    turn(sK1, sV1, sK0, sV0, t + 1);
  }
  l_run += __shfl_xor(l_run, 32, 64);
  __syncthreads();                                         // nobody reads the last tiles any more: K's buffers stage the output
  const uint32_t rows = qw < q_end ? q_end - qw : 0u;
  bf16_t* stage = KV == AT_KV ? sK0 + wave * (32 * DH) : (wave < 2 ? sK0 : sK1) + (wave & 1) * (32 * DH);
  at_store_tile<DH>(stage, oacc, l_run > 0.f ? 1.0f / l_run : 0.f, a.o + (size_t)(sq.q0 + qw) * a.ld_o + head * DH, a.ld_o, rows);
  if (qi < rows && h == 0 && a.lse != nullptr) a.lse[(size_t)head * a.rows_q + sq.q0 + q] = (m_run + __log2f(l_run)) * kLn2;
}

// Backward, dq.  Rows and wavefronts as in the forward kernel.  Also writes delta.
// delta = rowsum(do .* o) is taken from o as it is stored, whose two roundings to bf16 (of the probabilities and of o itself) it inherits.
// Beside the sums of many keys that is little (dq 2.5e-3 off in the norm for windows of 256 and more, where the roundings of dS and dq
// alone make 2.35e-3), but where a row sees some tens, o is as large as v: 2.6e-3 (100 keys), 2.7e-3 (16), 3.0e-3 (sequences of 16).  There it is
// taken as the sum of P dP, which is the same in exact arithmetic, in a sweep of its own over the tiles: 2.35e-3, for 26 us instead of 17 (nine
// sequences of 1 to 611 rows, 12 heads of 64, window 100).  Each block decides by what its own rows see at most (256 keys): how near a sequence's
// gradients are does not depend on the others in the call.
template <int DH>
__global__ __launch_bounds__(AT_THREADS, 2) void win_dq_kernel(WinArgs a) {
  constexpr int KS = DH / 16, DT = DH / 32, KV = kWinKv<DH>;
  constexpr uint32_t TILE = kWtTile<DH, KV>;
  // (four objects, so that the compiler can tell the buffer that is being filled from the one that is being read: of one, its transposing
  // reads would wait for the fetches under way)
  __shared__ __align__(1024) bf16_t sK0[TILE];
  __shared__ __align__(1024) bf16_t sV0[TILE];
  __shared__ __align__(1024) bf16_t sK1[TILE];
  __shared__ __align__(1024) bf16_t sV1[TILE];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qi = lane & 31, h = lane >> 5;
  const uint32_t units = a.heads / a.hb, b = blockIdx.x / units, head0 = blockIdx.x % units * a.hb, head = head0 + wave % a.hb, kvh = head0 / a.group;
  const WinSeq sq = win_seq(a, b);
  // (the last rows see the most keys where there is no window: their blocks start first)
  const uint32_t per = AT_Q / a.hb, q_blk = (gridDim.y - 1 - blockIdx.y) * per;
  if (q_blk >= sq.nq) return;
  const uint32_t qw = q_blk + wave / a.hb * 32, q = qw + qi;
  const int32_t off = (int32_t)sq.nk - (int32_t)sq.nq, pw = (int32_t)qw + off, p = pw + (int32_t)qi;
  const uint32_t q_end = min(q_blk + per, sq.nq);
  const WinSpan sp = win_span(a, (int32_t)q_blk + off, (int32_t)q_end - 1 + off, sq.nk);
  const bf16_t* kbase = a.k + (size_t)sq.k0 * a.ld_k + kvh * DH;
  const bf16_t* vbase = a.v + (size_t)sq.k0 * a.ld_v + kvh * DH;
  const float c2 = a.scale * kLog2e;
  const WtLane<DH> at;
  const uint32_t sink_tiles = (sp.sinks + KV - 1) / KV, tiles = sink_tiles + (sp.hi > sp.lo ? (sp.hi - sp.lo + KV - 1) / KV : 0u);

  bf16x8 fq[KS], fdo[KS];
  float dsum = 0.f;
  const uint32_t row = sq.q0 + (q < sq.nq ? q : sq.nq - 1);
  {
    const bf16_t* qp = a.q + (size_t)row * a.ld_q + head * DH;
    const bf16_t* dop = a.d_o + (size_t)row * a.ld_do + head * DH;
    const bf16_t* op = a.o + (size_t)row * a.ld_o + head * DH;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      fq[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16 + h * 8);
      const uint4 vd = *reinterpret_cast<const uint4*>(dop + ks * 16 + h * 8), vo = *reinterpret_cast<const uint4*>(op + ks * 16 + h * 8);
      fdo[ks] = *reinterpret_cast<const bf16x8*>(&vd);
      dsum += bflo(vd.x) * bflo(vo.x) + bfhi(vd.x) * bfhi(vo.x) + bflo(vd.y) * bflo(vo.y) + bfhi(vd.y) * bfhi(vo.y) +
              bflo(vd.z) * bflo(vo.z) + bfhi(vd.z) * bfhi(vo.z) + bflo(vd.w) * bflo(vo.w) + bfhi(vd.w) * bfhi(vo.w);
    }
  }
  dsum += __shfl_xor(dsum, 32, 64);
  const float lq2 = a.lse[(size_t)head * a.rows_q + row] * kLog2e;

  auto first_of = [&](uint32_t t) { return t < sink_tiles ? t * KV : sp.lo + (t - sink_tiles) * KV; };
  auto end_of = [&](uint32_t t) { return t < sink_tiles ? sp.sinks : sp.hi; };
  auto fetch = [&](bf16_t* sK, bf16_t* sV, uint32_t t) {
    wt_fetch<DH, KV, 4>(sK, kbase, a.ld_k, first_of(t), end_of(t), wave);
    wt_fetch<DH, KV, 4>(sV, vbase, a.ld_v, first_of(t), end_of(t), wave);
  };
  // scores and products with the values of 32 keys: S^T, dP^T
  auto products = [&](const bf16_t* sK, const bf16_t* sV, int n, floatx16& sacc, floatx16& pacc) {
#pragma unroll
    for (int r = 0; r < 16; ++r) { sacc[r] = 0.f; pacc[r] = 0.f; }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wt_frag<DH>(sK, at, n * 32, ks), fq[ks], sacc, 0, 0, 0);
      pacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wt_frag<DH>(sV, at, n * 32, ks), fdo[ks], pacc, 0, 0, 0);
    }
  };
  // all tiles in turn, each with the next one's fetch under way
  auto sweep = [&](auto use) {
    auto turn = [&](const bf16_t* sK, const bf16_t* sV, bf16_t* next_k, bf16_t* next_v, uint32_t t) {
      wait_fetches();
      __syncthreads();                                     // tile t has landed, nobody reads the other buffer any more
      const uint32_t kv0 = first_of(t), end = end_of(t);
      if (t + 1 < tiles) fetch(next_k, next_v, t + 1);
#pragma unroll
      for (int n = 0; n < KV / 32; ++n)
        if (!win_none(a, pw, kv0 + n * 32, 32, end)) use(sK, sV, n, kv0 + n * 32, end);
    };
    if (tiles > 0) fetch(sK0, sV0, 0);
    for (uint32_t t = 0; t < tiles; t += 2) {
      turn(sK0, sV0, sK1, sV1, t);
      if (t + 1 == tiles) break;
      turn(sK1, sV1, sK0, sV0, t + 1);
    }
  };
  const bool exact = (a.window != 0 ? min(sp.hi, a.window + a.sinks) : sp.hi) <= 256;
  if (exact) {
    dsum = 0.f;
    sweep([&](const bf16_t* sK, const bf16_t* sV, int n, uint32_t first, uint32_t end) {
      floatx16 sacc, pacc;
      products(sK, sV, n, sacc, pacc);
      float x[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f(fmaf(sacc[r], c2, -lq2)) * pacc[r];
      if (!win_all(a, pw, first, 32, end)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = win_sees(a, p, first + (r >> 2) * 8 + h * 4 + (r & 3), end) ? x[r] : 0.f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) dsum += x[r];
    });
    dsum += __shfl_xor(dsum, 32, 64);
    __syncthreads();                                       // nobody reads the last tiles any more
  }
  if (q < q_end && h == 0) {
    a.delta[(size_t)head * a.rows_q + row] = dsum;
    a.lse2[(size_t)head * a.rows_q + row] = -lq2;
  }
  floatx16 dqacc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) dqacc[d][r] = 0.f;
  sweep([&](const bf16_t* sK, const bf16_t* sV, int n, uint32_t first, uint32_t end) {
    floatx16 sacc, pacc;
    products(sK, sV, n, sacc, pacc);
    float ds[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) ds[r] = __builtin_amdgcn_exp2f(fmaf(sacc[r], c2, -lq2)) * (pacc[r] - dsum);      // (the scale is left for the end)
    if (!win_all(a, pw, first, 32, end)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) ds[r] = win_sees(a, p, first + (r >> 2) * 8 + h * 4 + (r & 3), end) ? ds[r] : 0.f;
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      const bf16x8 fds = at_pack8(ds, 8 * s2);
#pragma unroll
      for (int d = 0; d < DT; ++d) dqacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wt_frag_tr<DH>(sK, at, d, n * 32 + 16 * s2), fds, dqacc[d], 0, 0, 0);
    }
  });
  __syncthreads();
  const uint32_t rows = qw < q_end ? q_end - qw : 0u;
  bf16_t* stage = KV == AT_KV ? sK0 + wave * (32 * DH) : (wave < 2 ? sK0 : sK1) + (wave & 1) * (32 * DH);
  at_store_tile<DH>(stage, dqacc, a.scale, a.dq + (size_t)(sq.q0 + qw) * a.ld_dq + head * DH, a.ld_dq, rows);
}

// The part of dk and dv that sink keys get from rows far behind them.  A sequence's first 128 keys are one block of win_dkv_kernel, which
// goes as far as their windows; the rows from there on see nothing of them but the sinks, all of these, and there are as many as the
// sequence is long.  They are cut into pieces (a wavefront takes every fourth 32 rows of a piece, with 16 sinks in its registers:
// mostly there are no more than a few), whose sums are added up afterwards in a fixed order, together with that block's.  Without this
// the first block of 8192 rows with a window of 1024 had eight times the work of any other: dk and dv of 16 query and 4 key heads
// took 2216 us.
typedef float floatx4 __attribute__((ext_vector_type(4)));
template <int DH>
__device__ __forceinline__ float* win_part(const WinArgs& a, uint32_t unit, uint32_t sub, uint32_t piece) {      // [dk, dv][16 keys][DH]
  const uint32_t subs = (a.sinks + 15) / 16;
  return a.part + (((size_t)unit * subs + sub) * (a.pieces + 1) + piece) * (2 * 16 * DH);
}
struct WinFar { uint32_t first, steps, per, used; };       // rows from `first` on, 32 at a time (for all query heads), steps of a piece, pieces used
__device__ __forceinline__ WinFar win_far(const WinArgs& a, const WinSeq& sq) {
  WinFar f;
  const int64_t near_end = (int64_t)min(127u, sq.nk - 1) + a.window - ((int64_t)sq.nk - (int64_t)sq.nq);
  f.first = sq.nk == 0 || near_end >= (int64_t)sq.nq ? sq.nq : (uint32_t)max(near_end, (int64_t)0);
  f.steps = (sq.nq - f.first + 31) / 32;
  const uint32_t all = f.steps * a.group;
  f.per = (all + a.pieces - 1) / a.pieces;
  f.used = all > 0 ? (all + f.per - 1) / f.per : 0u;
  return f;
}
// The same for 16x16x32 products: rows 16 n + lane % 16 with d = 32 ks + 8 g .. (g = lane / 16); and operand row d = 16 t + lane % 16, k
// elements 0..3 the tile rows 4 g .., 4..7 the rows 16 + 4 g ..
template <int DH>
__device__ __forceinline__ bf16x8 win_frag16(const bf16_t* tile, int n, int ks) {
  const uint32_t lane = threadIdx.x & 63, row = n * 16 + (lane & 15);
  return *reinterpret_cast<const bf16x8*>(tile + wt_row<DH>(row) + (((uint32_t)ks * 4 + (lane >> 4)) ^ wt_key<DH>(row)) * 8);
}
template <int DH>
__device__ __forceinline__ bf16x8 win_frag_tr16(const bf16_t* tile, int t) {
  typedef short short4_lds __attribute__((ext_vector_type(4)));
  typedef short short8_v __attribute__((ext_vector_type(8)));
  typedef __attribute__((address_space(3))) short4_lds* lds_ptr;
  const uint32_t lane = threadIdx.x & 63, s = lane & 15, row = (lane >> 4) * 4 + (s >> 2), d = t * 16 + 4 * (s & 3u);
  const bf16_t* p = tile + wt_row<DH>(row) + (((d >> 3) ^ wt_key<DH>(row)) * 8) + (d & 7u);
  const short4_lds lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
  const short4_lds hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + wt_row<DH>(16)));
  const short8_v v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, v);
}

template <int DH>
__global__ __launch_bounds__(AT_THREADS, 2) void win_sink_kernel(WinArgs a) {
  constexpr int KS = DH / 32, DT = DH / 16;
  __shared__ __align__(1024) bf16_t sQ[4][kWtTile<DH, 32>];
  __shared__ __align__(1024) bf16_t sDo[4][kWtTile<DH, 32>];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
  const uint32_t b = blockIdx.x / a.kv_heads, kvh = blockIdx.x % a.kv_heads, kv = blockIdx.y * 16 + col, piece = blockIdx.z;
  const WinSeq sq = win_seq(a, b);
  const WinFar far = win_far(a, sq);
  if (piece >= far.used) return;
  const uint32_t begin = piece * far.per, end = min(begin + far.per, far.steps * a.group);
  const float c2 = a.scale * kLog2e;
  const bool kv_ok = kv < a.sinks;
  bf16x8 fk[KS], fv[KS];
  {
    const uint32_t r = sq.k0 + min(kv, sq.nk - 1);
    const bf16_t* kp = a.k + (size_t)r * a.ld_k + kvh * DH;
    const bf16_t* vp = a.v + (size_t)r * a.ld_v + kvh * DH;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      fk[ks] = *reinterpret_cast<const bf16x8*>(kp + ks * 32 + g * 8);
      fv[ks] = *reinterpret_cast<const bf16x8*>(vp + ks * 32 + g * 8);
    }
  }
  floatx4 dkacc[DT], dvacc[DT];                    // [d][key]: element e is d = 16 t + 4 g + e of key col
#pragma unroll
  for (int d = 0; d < DT; ++d) dkacc[d] = dvacc[d] = floatx4{0.f, 0.f, 0.f, 0.f};
  const bf16_t* q = sQ[wave];
  const bf16_t* d_o = sDo[wave];
  for (uint32_t t = begin + wave; t < end; t += 4) {
    const uint32_t head = kvh * a.group + t / far.steps, q0 = far.first + t % far.steps * 32;
    wt_fetch<DH, 32, 1>(sQ[wave], a.q + (size_t)sq.q0 * a.ld_q + head * DH, a.ld_q, q0, sq.nq, 0);
    wt_fetch<DH, 32, 1>(sDo[wave], a.d_o + (size_t)sq.q0 * a.ld_do + head * DH, a.ld_do, q0, sq.nq, 0);
    float lv[2][4], dl[2][4];                      // of rows 16 n + 4 g + e
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const size_t at = (size_t)head * a.rows_q + sq.q0 + min(q0 + n * 16 + g * 4 + e, sq.nq - 1);
        lv[n][e] = a.lse2[at];
        dl[n][e] = a.delta[at];
      }
    wait_fetches();                                // this wavefront's own rows
    uint32_t fp[4], fds[4];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      floatx4 s = floatx4{0.f, 0.f, 0.f, 0.f}, p = s;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(win_frag16<DH>(q, n, ks), fk[ks], s, 0, 0, 0);
        p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(win_frag16<DH>(d_o, n, ks), fv[ks], p, 0, 0, 0);
      }
      float pr[4], ds[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool ok = kv_ok && q0 + n * 16 + g * 4 + e < sq.nq;
        const float x = __builtin_amdgcn_exp2f(fmaf(s[e], c2, lv[n][e]));
        pr[e] = ok ? x : 0.f;
        ds[e] = ok ? x * (p[e] - dl[n][e]) : 0.f;
      }
      fp[2 * n] = pack_bf2(pr[0], pr[1]);
      fp[2 * n + 1] = pack_bf2(pr[2], pr[3]);
      fds[2 * n] = pack_bf2(ds[0], ds[1]);
      fds[2 * n + 1] = pack_bf2(ds[2], ds[3]);
    }
    const uint4 vp = make_uint4(fp[0], fp[1], fp[2], fp[3]), vs = make_uint4(fds[0], fds[1], fds[2], fds[3]);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      dvacc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(win_frag_tr16<DH>(d_o, d), *reinterpret_cast<const bf16x8*>(&vp), dvacc[d], 0, 0, 0);
      dkacc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(win_frag_tr16<DH>(q, d), *reinterpret_cast<const bf16x8*>(&vs), dkacc[d], 0, 0, 0);
    }
  }
  // the four wavefronts' sums through LDS: [wavefront][dk, dv][16 keys][DH]
  __syncthreads();
  float* sum = reinterpret_cast<float*>(&sQ[0][0]);
  static_assert(sizeof(sQ) >= 4 * 16 * DH * sizeof(float) && sizeof(sDo) >= 4 * 16 * DH * sizeof(float), "room for four wavefronts' sums of one result");
  float* sum_v = reinterpret_cast<float*>(&sDo[0][0]);
#pragma unroll
  for (int d = 0; d < DT; ++d) {
    *reinterpret_cast<floatx4*>(sum + (wave * 16 + col) * DH + d * 16 + g * 4) = dkacc[d];
    *reinterpret_cast<floatx4*>(sum_v + (wave * 16 + col) * DH + d * 16 + g * 4) = dvacc[d];
  }
  __syncthreads();
  float* out = win_part<DH>(a, blockIdx.x, blockIdx.y, piece);
  for (uint32_t i = threadIdx.x * 4; i < 2 * 16 * DH; i += AT_THREADS * 4) {
    const float* from = (i < 16 * DH ? sum : sum_v - 16 * DH) + i;
    floatx4 s = *reinterpret_cast<const floatx4*>(from);
#pragma unroll
    for (int w = 1; w < 4; ++w) s += *reinterpret_cast<const floatx4*>(from + w * (16 * DH));
    *reinterpret_cast<floatx4*>(out + i) = s;
  }
}

// Adds the pieces up: a block takes 64 vectors of a unit's 16 sinks (dk, then dv), each wavefront every fourth piece.
template <int DH>
__global__ __launch_bounds__(256) void win_sink_join_kernel(WinArgs a) {
  __shared__ __align__(16) floatx4 s_sum[4][64];
  const uint32_t b = blockIdx.x / a.kv_heads, kvh = blockIdx.x % a.kv_heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const WinSeq sq = win_seq(a, b);
  const WinFar far = win_far(a, sq);
  const uint32_t i = (blockIdx.z * 64 + lane) * 4, which = i / (16 * DH), key = blockIdx.y * 16 + i / DH % 16;
  const float* at = win_part<DH>(a, blockIdx.x, blockIdx.y, 0) + i;
  floatx4 s = floatx4{0.f, 0.f, 0.f, 0.f};
  if (blockIdx.y * 16 < sq.nk) {
    if (wave == 0) s = *reinterpret_cast<const floatx4*>(at + (size_t)a.pieces * (2 * 16 * DH));      // the first block's own
#pragma unroll 8
    for (uint32_t p = wave; p < far.used; p += 4) s += *reinterpret_cast<const floatx4*>(at + (size_t)p * (2 * 16 * DH));
  }
  s_sum[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || key >= sq.nk) return;
  s = (s_sum[0][lane] + s_sum[1][lane] + s_sum[2][lane] + s_sum[3][lane]) * (which ? 1.0f : a.scale);
  bf16_t* out = which ? a.dv : a.dk;
  *reinterpret_cast<uint2*>(out + (size_t)(sq.k0 + key) * (which ? a.ld_dv : a.ld_dk) + kvh * DH + i % DH) = make_uint2(pack_bf2(s[0], s[1]), pack_bf2(s[2], s[3]));
}

// Backward, dk and dv.  A block is 128 keys of a key head; the rows that see them are streamed 64 at a time, query head after query head.
// Eight wavefronts: 32 keys and 32 of the 64 rows each, the two with the same keys add their sums up at the end.  K and V stay in LDS as
// well, since with them in registers (64 of heads of 128, beside 128 of sums and 32 of scores) there is room for one wavefront
// per SIMD only, whose exponentials then hold up its products (8192 rows as above: 290 us, so 177).
constexpr int WIN_DKV_THREADS = 512;
template <int DH>
__global__ __launch_bounds__(WIN_DKV_THREADS, 2) void win_dkv_kernel(WinArgs a) {
  constexpr int KS = DH / 16, DT = DH / 32;
  constexpr uint32_t TILE = kWtTile<DH, AT_QB>;
  __shared__ __align__(1024) bf16_t sQ0[TILE];
  __shared__ __align__(1024) bf16_t sDo0[TILE];
  __shared__ __align__(1024) bf16_t sQ1[TILE];
  __shared__ __align__(1024) bf16_t sDo1[TILE];
  __shared__ __align__(16) float sL0[2 * AT_QB];                    // log sum exp, row term
  __shared__ __align__(16) float sL1[2 * AT_QB];
  __shared__ __align__(1024) bf16_t sK[kWtTile<DH, AT_KV>];
  __shared__ __align__(1024) bf16_t sV[kWtTile<DH, AT_KV>];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ki = lane & 31, h = lane >> 5;
  const uint32_t part = wave & 3, u = wave >> 2;           // keys 32 part .., rows 32 u .. of a step
  const uint32_t b = blockIdx.x / a.kv_heads, kvh = blockIdx.x % a.kv_heads;
  const WinSeq sq = win_seq(a, b);
  const uint32_t kv_blk = blockIdx.y * AT_KV, kw = kv_blk + part * 32, kv = kw + ki;
  if (kv_blk >= sq.nk) return;
  const int32_t off = (int32_t)sq.nk - (int32_t)sq.nq;
  const float c2 = a.scale * kLog2e;
  const WtLane<DH> at;
  // rows (of the sequence) that see one of the block's keys; of the sinks' only those that see its last key too, or might
  const uint32_t kv_last = min(kv_blk + AT_KV, sq.nk) - 1;
  const int32_t row_a = max((int32_t)kv_blk - off, 0);
  const int64_t row_z = a.window == 0 ? (int64_t)sq.nq : min((int64_t)kv_last + a.window - off, (int64_t)sq.nq);
  const uint32_t q_first = (uint32_t)row_a, q_end = row_z > row_a ? (uint32_t)row_z : q_first;
  const uint32_t steps = (q_end - q_first + AT_QB - 1) / AT_QB, total = steps * a.group;

  floatx16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) { dkacc[d][r] = 0.f; dvacc[d][r] = 0.f; }

  auto fetch = [&](bf16_t* sQ, bf16_t* sDo, float* sL, uint32_t t) {
    const uint32_t head = kvh * a.group + t / steps, q0 = q_first + t % steps * AT_QB;
    wt_fetch<DH, AT_QB, 8>(sQ, a.q + (size_t)sq.q0 * a.ld_q + head * DH, a.ld_q, q0, q_end, wave);
    wt_fetch<DH, AT_QB, 8>(sDo, a.d_o + (size_t)sq.q0 * a.ld_do + head * DH, a.ld_do, q0, q_end, wave);
    if (wave < 2) {                                        // log sum exp (wavefront 0) and row term (1) of the 64 rows
      typedef __attribute__((address_space(3))) void* lds_void_ptr;
      typedef __attribute__((address_space(1))) const void* global_void_ptr;
      const size_t row = (size_t)head * a.rows_q + sq.q0 + min(q0 + lane, q_end - 1);
      __builtin_amdgcn_global_load_lds((global_void_ptr)((wave == 0 ? a.lse2 : a.delta) + row), (lds_void_ptr)(sL + wave * AT_QB), 4, 0, 0);
    }
  };
  if (total > 0) {
    wt_fetch<DH, AT_KV, 8>(sK, a.k + (size_t)sq.k0 * a.ld_k + kvh * DH, a.ld_k, kv_blk, sq.nk, wave);
    wt_fetch<DH, AT_KV, 8>(sV, a.v + (size_t)sq.k0 * a.ld_v + kvh * DH, a.ld_v, kv_blk, sq.nk, wave);
    fetch(sQ0, sDo0, sL0, 0);
  }
  auto turn = [&](const bf16_t* sQ, const bf16_t* sDo, const float* sLd, bf16_t* next_q, bf16_t* next_do, float* next_l, uint32_t t) {
    wait_fetches();
    __syncthreads();                                       // step t has landed, nobody reads the other buffer any more
    const uint32_t qu = q_first + t % steps * AT_QB + u * 32;
    if (t + 1 < total) fetch(next_q, next_do, next_l, t + 1);
    const int32_t pw = (int32_t)qu + off;
    if (qu >= q_end || win_none(a, pw, kw, 32, sq.nk)) return;
    const float* sL = sLd + u * 32 + h * 4;
    floatx16 sacc, pacc;
#pragma unroll
    for (int r = 0; r < 16; ++r) { sacc[r] = 0.f; pacc[r] = 0.f; }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wt_frag<DH>(sQ, at, u * 32, ks), wt_frag<DH>(sK, at, part * 32, ks), sacc, 0, 0, 0);      // S  [q][kv]
      pacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wt_frag<DH>(sDo, at, u * 32, ks), wt_frag<DH>(sV, at, part * 32, ks), pacc, 0, 0, 0);     // dP [q][kv]
    }
    float pr[16], ds[16];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 l4 = *reinterpret_cast<const float4*>(sL + g * 8);
      const float4 d4 = *reinterpret_cast<const float4*>(sL + AT_QB + g * 8);
      const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = g * 4 + e;
        pr[r] = __builtin_amdgcn_exp2f(fmaf(sacc[r], c2, lv[e]));
        ds[r] = pr[r] * (pacc[r] - dv[e]);
      }
    }
    if (qu + 32 > q_end || !win_all(a, pw, kw, 32, sq.nk)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t row = qu + (r >> 2) * 8 + h * 4 + (r & 3);
        const bool ok = row < q_end && win_sees(a, (int32_t)row + off, kv, sq.nk);
        pr[r] = ok ? pr[r] : 0.f;
        ds[r] = ok ? ds[r] : 0.f;
      }
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      const bf16x8 fp = at_pack8(pr, 8 * s2), fds = at_pack8(ds, 8 * s2);
      const uint32_t qb = u * 32 + 16 * s2;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        dvacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wt_frag_tr<DH>(sDo, at, d, qb), fp, dvacc[d], 0, 0, 0);      // dV^T
        dkacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wt_frag_tr<DH>(sQ, at, d, qb), fds, dkacc[d], 0, 0, 0);      // dK^T
      }
    }
  };
  for (uint32_t t = 0; t < total; t += 2) {
    turn(sQ0, sDo0, sL0, sQ1, sDo1, sL1, t);
    if (t + 1 == total) break;
    turn(sQ1, sDo1, sL1, sQ0, sDo0, sL0, t + 1);
  }
  // the second four wavefronts' sums go to the first four through LDS (dk in K's and V's place, then dv), as they lie in the registers
  float4* pass = reinterpret_cast<float4*>(part < 2 ? sK : sV) + (part & 1) * (DT * 4 * 64);
  static_assert(sizeof(sK) >= 2 * DT * 4 * 64 * sizeof(float4), "room for two wavefronts' sums");
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
    if (u == 1) {
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const floatx16& x = which ? dvacc[d] : dkacc[d];
          pass[(d * 4 + g) * 64 + lane] = make_float4(x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]);
        }
    }
    __syncthreads();
    if (u == 0) {
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 v = pass[(d * 4 + g) * 64 + lane];
          floatx16& x = which ? dvacc[d] : dkacc[d];
          x[4 * g] += v.x; x[4 * g + 1] += v.y; x[4 * g + 2] += v.z; x[4 * g + 3] += v.w;
        }
    }
  }
  if (u == 1) return;
  const uint32_t rows = kw < sq.nk ? sq.nk - kw : 0u;
  if (a.part != nullptr && kw < a.sinks) {       // more is to be added to some of these rows: they go on as sums
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (kw + half * 16 >= a.sinks) break;
      float* part_at = win_part<DH>(a, blockIdx.x, kw / 16 + half, a.pieces) + (ki & 15) * DH + h * 4;
      if ((ki >> 4) == (uint32_t)half) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            *reinterpret_cast<float4*>(part_at + d * 32 + g * 8) = make_float4(dkacc[d][4 * g], dkacc[d][4 * g + 1], dkacc[d][4 * g + 2], dkacc[d][4 * g + 3]);
            *reinterpret_cast<float4*>(part_at + 16 * DH + d * 32 + g * 8) = make_float4(dvacc[d][4 * g], dvacc[d][4 * g + 1], dvacc[d][4 * g + 2], dvacc[d][4 * g + 3]);
          }
      }
    }
  }
  // (rows that the pieces are added to are written again by the launch that adds them up)
  bf16_t* stage = (part < 2 ? sQ0 : sDo0) + (part & 1) * (32 * DH);
  at_store_tile<DH>(stage, dkacc, a.scale, a.dk + (size_t)(sq.k0 + kw) * a.ld_dk + kvh * DH, a.ld_dk, rows);
  at_store_tile<DH>(stage, dvacc, 1.0f, a.dv + (size_t)(sq.k0 + kw) * a.ld_dv + kvh * DH, a.ld_dv, rows);
}

static bool al16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Extents of either pass, and what the kernels are told.
static sif_status win_plan(const char* who, const sif_window_attn_args* a, WinArgs* w) {
  if (!a) return fail(SIF_E_INVAL, "%s: null arguments", who);
  if (a->struct_size != sizeof(sif_window_attn_args)) return fail(SIF_E_INVAL, "%s: struct_size", who);
  if (!a->heads || !a->kv_heads || a->heads % a->kv_heads) return fail(SIF_E_INVAL, "%s: heads must be a multiple of kv_heads", who);
  if (a->d_head != 64 && a->d_head != 128) return fail(SIF_E_INVAL, "%s: d_head must be 64 or 128", who);
  if (!a->batch || !a->seq_q || !a->seq_k) return fail(SIF_E_INVAL, "%s: empty extent", who);
  if (a->heads > 1024) return fail(SIF_E_INVAL, "%s: at most 1024 heads", who);
  if (a->seq_q > (1u << 20) || a->seq_k > (1u << 20)) return fail(SIF_E_INVAL, "%s: sequences of at most 2^20 rows", who);
  if ((uint64_t)a->batch * a->heads >= 1ull << 23) return fail(SIF_E_INVAL, "%s: batch * heads below 2^23", who);       // threads of a grid stay below 2^32
  if ((uint64_t)a->batch * a->seq_q > 0x7FFFFFFFull || (uint64_t)a->batch * a->seq_k > 0x7FFFFFFFull) return fail(SIF_E_INVAL, "%s: rows beyond 31 bits", who);
  if (a->sinks > 128) return fail(SIF_E_INVAL, "%s: at most 128 sinks", who);
  if (a->window > (1u << 30)) return fail(SIF_E_INVAL, "%s: a window of at most 2^30 (0: no limit)", who);
  if (!(a->scale >= 0.f) || !std::isfinite(a->scale * kLog2e)) return fail(SIF_E_INVAL, "%s: scale must be finite (in base 2 too) and not negative", who);
  if (a->starts_dev && (a->seq_q != a->seq_k || a->rows == 0 || a->rows > 0x7FFFFFFFu)) return fail(SIF_E_INVAL, "%s: with starts, seq_q = seq_k and rows in 1 .. 2^31 - 1", who);
  if ((uintptr_t)a->starts_dev & 3) return fail(SIF_E_INVAL, "%s: misaligned starts", who);
  w->starts = a->starts_dev;
  w->heads = a->heads;
  w->kv_heads = a->kv_heads;
  w->group = a->heads / a->kv_heads;
  w->hb = w->group % 4 == 0 ? 4 : (w->group % 2 == 0 ? 2 : 1);
  w->batch = a->batch;
  w->sq = a->seq_q;
  w->sk = a->seq_k;
  w->window = a->window;
  w->sinks = a->window != 0 ? a->sinks : 0;
  w->rows = a->rows;
  w->rows_q = a->starts_dev ? a->rows : a->batch * a->seq_q;
  w->scale = a->scale != 0.f ? a->scale : 1.0f / sqrtf((float)a->d_head);
  w->q = (const bf16_t*)a->q_dev;
  w->k = (const bf16_t*)a->k_dev;
  w->v = (const bf16_t*)a->v_dev;
  w->o = (bf16_t*)a->o_dev;
  w->lse = a->lse_dev;
  w->d_o = (const bf16_t*)a->do_dev;
  w->dq = (bf16_t*)a->dq_dev;
  w->dk = (bf16_t*)a->dk_dev;
  w->dv = (bf16_t*)a->dv_dev;
  w->delta = w->lse2 = w->part = nullptr;
  w->pieces = 0;
  w->ld_q = a->ld_q; w->ld_k = a->ld_k; w->ld_v = a->ld_v; w->ld_o = a->ld_o;
  w->ld_do = a->ld_do; w->ld_dq = a->ld_dq; w->ld_dk = a->ld_dk; w->ld_dv = a->ld_dv;
  return SIF_OK;
}

static sif_status win_check(const char* who, const sif_window_attn_args* a) {
  const uint32_t wq = a->heads * a->d_head, wk = a->kv_heads * a->d_head;
  if (!a->q_dev || !a->k_dev || !a->v_dev || !a->o_dev) return fail(SIF_E_INVAL, "%s: null operand", who);
  if (a->ld_q < wq || a->ld_o < wq || a->ld_k < wk || a->ld_v < wk || ((a->ld_q | a->ld_o | a->ld_k | a->ld_v) & 7)) return fail(SIF_E_INVAL, "%s: bad leading dimensions", who);
  if ((a->ld_q | a->ld_k | a->ld_v | a->ld_do) >> 27) return fail(SIF_E_INVAL, "%s: leading dimensions below 2^27", who);
  if (!al16(a->q_dev) || !al16(a->k_dev) || !al16(a->v_dev) || !al16(a->o_dev)) return fail(SIF_E_INVAL, "%s: pointers must be 16-byte aligned", who);
  if ((uintptr_t)a->lse_dev & 3) return fail(SIF_E_INVAL, "%s: misaligned lse", who);
  return SIF_OK;
}

// Workspace of the backward pass: delta and log sum exp per row, and the sinks' pieces where some row is far enough from them; as many pieces as give the chip two
// blocks per CU, of at least 8 steps of 32 rows.
static uint64_t win_workspace(WinArgs& w, uint32_t d_head, void* at) {
  const uint64_t rows = (uint64_t)w.heads * w.rows_q, delta = (2 * rows * sizeof(float) + 255) / 256 * 256;
  w.delta = (float*)at;
  w.lse2 = w.delta + rows;
  w.part = nullptr;
  w.pieces = 0;
  if (w.sinks == 0 || (uint64_t)w.sk <= 127ull + w.window) return delta;
  const uint64_t units = (uint64_t)w.batch * w.kv_heads, subs = (w.sinks + 15) / 16;
  const uint64_t steps = (uint64_t)((std::min(w.sq, w.sk - 127 - w.window) + 31) / 32) * w.group;
  w.pieces = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(512 / (units * subs), (steps + 7) / 8));
  w.part = (float*)((unsigned char*)at + delta);
  return delta + units * subs * (w.pieces + 1) * (2 * 16 * (uint64_t)d_head * sizeof(float));
}

}  // namespace sif

using namespace sif;

extern "C" {

sif_status sif_k_window_attn_fwd(const sif_window_attn_args* a, void* stream) {
  WinArgs w;
  if (sif_status st = win_plan("window_attn_fwd", a, &w)) return st;
  if (sif_status st = win_check("window_attn_fwd", a)) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const uint32_t per = AT_Q / w.hb;
  const dim3 grid(w.batch * (w.heads / w.hb), (w.sq + per - 1) / per);
  if (a->d_head == 64) hipLaunchKernelGGL((win_fwd_kernel<64>), grid, dim3(AT_THREADS), 0, s, w);
  else hipLaunchKernelGGL((win_fwd_kernel<128>), grid, dim3(AT_THREADS), 0, s, w);
  return check_launch("window_attn_fwd");
}

uint64_t sif_window_attn_bwd_workspace_bytes(const sif_window_attn_args* a) {
  WinArgs w;
  return win_plan("window_attn_bwd_workspace_bytes", a, &w) == SIF_OK ? win_workspace(w, a->d_head, nullptr) : 0;
}

sif_status sif_k_window_attn_bwd(const sif_window_attn_args* a, void* stream) {
  WinArgs w;
  if (sif_status st = win_plan("window_attn_bwd", a, &w)) return st;
  if (sif_status st = win_check("window_attn_bwd", a)) return st;
  const uint32_t wq = a->heads * a->d_head, wk = a->kv_heads * a->d_head;
  if (!a->lse_dev || !a->do_dev || !a->dq_dev || !a->dk_dev || !a->dv_dev) return fail(SIF_E_INVAL, "window_attn_bwd: null operand");
  if (a->ld_do < wq || a->ld_dq < wq || a->ld_dk < wk || a->ld_dv < wk || ((a->ld_do | a->ld_dq | a->ld_dk | a->ld_dv) & 7))
    return fail(SIF_E_INVAL, "window_attn_bwd: bad leading dimensions");
  if (!al16(a->do_dev) || !al16(a->dq_dev) || !al16(a->dk_dev) || !al16(a->dv_dev)) return fail(SIF_E_INVAL, "window_attn_bwd: pointers must be 16-byte aligned");
  if (!a->workspace_dev || ((uintptr_t)a->workspace_dev & 255)) return fail(SIF_E_INVAL, "window_attn_bwd: the workspace must be 256-byte aligned");
  const uint64_t need = win_workspace(w, a->d_head, a->workspace_dev);
  if (a->workspace_bytes < need)
    return fail(SIF_E_NOMEM, "window_attn_bwd: the workspace holds %llu of %llu bytes", (unsigned long long)a->workspace_bytes, (unsigned long long)need);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const uint32_t per = AT_Q / w.hb;
  const dim3 gq(w.batch * (w.heads / w.hb), (w.sq + per - 1) / per), gk(w.batch * w.kv_heads, (w.sk + AT_KV - 1) / AT_KV);
  if (a->d_head == 64) hipLaunchKernelGGL((win_dq_kernel<64>), gq, dim3(AT_THREADS), 0, s, w);
  else hipLaunchKernelGGL((win_dq_kernel<128>), gq, dim3(AT_THREADS), 0, s, w);
  if (sif_status st = check_launch("window_attn_bwd: dq")) return st;
  if (a->d_head == 64) hipLaunchKernelGGL((win_dkv_kernel<64>), gk, dim3(WIN_DKV_THREADS), 0, s, w);
  else hipLaunchKernelGGL((win_dkv_kernel<128>), gk, dim3(WIN_DKV_THREADS), 0, s, w);
  if (sif_status st = check_launch("window_attn_bwd: dk and dv")) return st;
  if (w.part == nullptr) return SIF_OK;
  const dim3 gs(w.batch * w.kv_heads, (w.sinks + 15) / 16, w.pieces), gj(w.batch * w.kv_heads, (w.sinks + 15) / 16, a->d_head / 8);
  if (a->d_head == 64) hipLaunchKernelGGL((win_sink_kernel<64>), gs, dim3(AT_THREADS), 0, s, w);
  else hipLaunchKernelGGL((win_sink_kernel<128>), gs, dim3(AT_THREADS), 0, s, w);
  if (sif_status st = check_launch("window_attn_bwd: sinks")) return st;
  if (a->d_head == 64) hipLaunchKernelGGL((win_sink_join_kernel<64>), gj, dim3(AT_THREADS), 0, s, w);
  else hipLaunchKernelGGL((win_sink_join_kernel<128>), gj, dim3(AT_THREADS), 0, s, w);
  return check_launch("window_attn_bwd: sum of the sinks' pieces");
}

}  // extern "C"
