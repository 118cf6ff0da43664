// What the kernels of attention over a paged cache share, whatever the cache's format: the division of the work, the steps a sequence's tokens
// lie in, streaming loads, and what a block does with its wavefronts' results.
#pragma once
#include <math.h>
#include <algorithm>

#include "common.h"
#include "kv_cache.h"

namespace sif {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr uint32_t AD_WAVES = 4, AD_HEADS = 16, AD_BLOCKS = 256;      // AD_BLOCKS: a block for each CU, and the most splits
constexpr float kNoSplit = -1.0f;       // in the place of a split's sum

struct DecodeArgs {
  KvView c;
  const int32_t* seqs;
  const bf16_t* q;
  bf16_t* o;
  float* lse;
  float* part;                       // [sequence][query head][split][DH + 4]: m, l, -, -, O
  uint32_t layer, n, heads, group, head_tiles, window, sinks, splits, chunk, ld_q, ld_o;      // chunk: steps of a split
  float scale;
};

// The steps in which a sequence's visible tokens lie: `sink_steps` from the first token on, the others from token `from` (a multiple of
// a step's tokens) on.
struct DecodeSpan { uint32_t len, lo, sink_steps, from, steps; };
template <uint32_t TOK>
__device__ __forceinline__ DecodeSpan decode_span(uint32_t len, uint32_t window, uint32_t sinks) {
  DecodeSpan s;
  s.len = len;
  s.lo = window != 0 && len > window ? len - window : 0u;          // the first token of the window
  const uint32_t first = s.lo / TOK, end = (len + TOK - 1) / TOK;
  const uint32_t sink_end = (std::min(sinks, len) + TOK - 1) / TOK;
  s.sink_steps = s.lo == 0 ? 0u : std::min(sink_end, first);
  s.from = first * TOK;
  s.steps = s.sink_steps + end - first;
  return s;
}

// 16 bytes of lines that one fetch instruction takes whole and that this sequence does not read again: loads that claim no place in the
// caches.  (Sequences that share pages after a fork read them once each; that case has not been timed both ways.)  (1 GiB read by
// 256 to 1024 blocks in the ordinary way takes 167 to 222 us, 4.8 to 6.4 TB/s, in this way 148 to 206.)  That is V's case where a page is no
// longer than a step: 64 sequences of 4096 tokens 189 -> 171 us, of 1 to 8192 215 -> 201.  K's rows of more than 64 bytes take several
// instructions to a line, and so do V's in longer pages; with these loads the line came from memory again (one sequence of
// 262011 tokens, pages of 64: 186 -> 206 us; K too: 64 sequences of 1 to 8192 222).
__device__ __forceinline__ uint4 fetch16(const unsigned char* p) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ bf16x8 as_bf16(const uint4& v) { return *reinterpret_cast<const bf16x8*>(&v); }

// A block's end: every wavefront has a running maximum (base 2), its lane's part of the sum and, unnormalized, the results of sixteen query heads; they are joined and
// written, the answer itself or this split's part of it.  vs: the cache's scale of values.
template <int DH>
__device__ __forceinline__ void decode_finish(const DecodeArgs& a, uint32_t i, uint32_t kvh, uint32_t ht, uint32_t split, uint32_t parts, float m_run, float l_run,
                                              const floatx4 (&oacc)[DH / 16], float vs) {
  constexpr uint32_t DT = DH / 16;
  __shared__ __align__(16) float s_o[AD_WAVES][AD_HEADS][DH + 4];
  __shared__ float s_m[AD_WAVES][AD_HEADS], s_l[AD_WAVES][AD_HEADS];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);

  // the four wavefronts' results, joined through LDS: accumulator element e of tile d is column d*16 + 4 g + e of query head `col`
  if (g == 0) { s_m[wave][col] = m_run; s_l[wave][col] = l_run; }
#pragma unroll
  for (uint32_t d = 0; d < DT; ++d) *reinterpret_cast<float4*>(&s_o[wave][col][d * 16 + g * 4]) = make_float4(oacc[d][0], oacc[d][1], oacc[d][2], oacc[d][3]);
  __syncthreads();
  const uint32_t r = threadIdx.x >> 4, x = threadIdx.x & 15;           // a query head per sixteen threads
  const uint32_t rows = std::min(a.group - ht * AD_HEADS, AD_HEADS);
  if (r >= rows) return;
  float m = -INFINITY;
#pragma unroll
  for (uint32_t w = 0; w < AD_WAVES; ++w) m = fmaxf(m, s_m[w][r]);
  float f[AD_WAVES], l = 0.f;
#pragma unroll
  for (uint32_t w = 0; w < AD_WAVES; ++w) {
    f[w] = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][r] - m);
    l += f[w] * s_l[w][r];
  }
  const float inv = parts > 1 ? vs : (l > 0.f ? vs / l : 0.f);
  const uint32_t out_head = kvh * a.group + ht * AD_HEADS + r;
  float y[DH / 16];
#pragma unroll
  for (uint32_t e = 0; e < DH / 16; ++e) {
    const uint32_t d = x * (DH / 16) + e;
    float t = 0.f;
#pragma unroll
    for (uint32_t w = 0; w < AD_WAVES; ++w) t += f[w] * s_o[w][r][d];
    y[e] = t * inv;
  }
  if (parts == 1) {
    bf16_t* to = a.o + (size_t)i * a.ld_o + (size_t)out_head * DH + x * (DH / 16);
    if constexpr (DH == 128) *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3]), pack_bf2(y[4], y[5]), pack_bf2(y[6], y[7]));
    else *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3]));
    if (x == 0 && a.lse != nullptr) a.lse[(size_t)i * a.heads + out_head] = (m + __log2f(l)) * 0.693147180559945f;
  } else {
    float* to = a.part + (((size_t)i * a.heads + out_head) * a.splits + split) * (DH + 4);
#pragma unroll
    for (uint32_t e = 0; e < DH / 16; e += 4) *reinterpret_cast<float4*>(to + 4 + x * (DH / 16) + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
    if (x == 0) *reinterpret_cast<float2*>(to) = make_float2(m, l);
  }
}

// A launch over a cache in 4 bits (attn_decode4.hip).
void launch_attn_decode4(const DecodeArgs& d, uint32_t d_head, dim3 grid, bool stream_v, hipStream_t s);

}  // namespace sif
