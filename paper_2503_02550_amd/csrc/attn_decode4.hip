// Attention of one new token per sequence over a paged cache in 4 bits (the formulas and the division of the work: attn_decode.hip).
//
// A token of a kv head of 128 is 136 bytes, so that what the memory delivers in a given time is four times as many tokens as in bf16 and the vector units have to
// keep up: numbers are brought to bf16 two at a time by the conversion instruction, which takes the keys' powers of two along, and go into the matrix units as
// they are.  A wavefront's step is 64 tokens:
//
//   S^T = K Q^T    row 4a + b of tile t is token 16 a + 4 b + t.  A lane (row, g) has the d of its token that make one 16-byte fetch (8 of a head of 64): 32
//                  consecutive d, so one power; its four tiles' powers are one word.  Its results (column = query head, rows 4g ..) are 16 consecutive tokens
//   O^T = V^T P^T  byte (b, c) of a token holds d = 32 b + c and d + 16, so a lane's 16-byte fetch is the operand of two tiles of 16 d and 16 tokens.  The values'
//                  powers differ from token to token: they go into P, whose rounding to bf16 they do not touch, once for each 32 d.  Lane (c, g) has those of
//                  token 16 g + c, and hands them to the others of its sixteen as it multiplies.
#include <type_traits>
#include <utility>

#include "attn_decode.h"
#include "e2m1.h"

namespace sif {

// lane U of the sixteen to all of them
template <int U>
__device__ __forceinline__ float of_row(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x150 + U, 0xF, 0xF, true));
}
template <typename F, int... I>
__device__ __forceinline__ void for_each(std::integer_sequence<int, I...>, F&& f) { (f(std::integral_constant<int, I>{}), ...); }

template <int DH, bool STREAM>
__global__ __launch_bounds__(256, 2) void attn_decode4_kernel(DecodeArgs a) {
  constexpr uint32_t TOK = 64, NT = 4, NB = DH / 32, KW = DH / 32, DT = DH / 16;      // tiles of 16 tokens; powers of a token; words of a lane's d
  const KvView& c = a.c;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
  const uint32_t ht = blockIdx.x % a.head_tiles, kvh = blockIdx.x / a.head_tiles % c.kv_heads, i = blockIdx.x / a.head_tiles / c.kv_heads;
  const int32_t s = kv_listed(c, a.seqs, i);
  const DecodeSpan sp = decode_span<TOK>(s >= 0 ? kv_length(c, s) : 0u, a.window, a.sinks);
  const uint32_t parts = sp.steps == 0 ? 1u : std::min((sp.steps + a.chunk - 1) / a.chunk, a.splits), split = blockIdx.y;
  auto unused = [&](uint32_t which) {
    if (threadIdx.x < std::min(a.group - ht * AD_HEADS, AD_HEADS))
      a.part[(((size_t)i * a.heads + kvh * a.group + ht * AD_HEADS + threadIdx.x) * a.splits + which) * (DH + 4) + 1] = kNoSplit;
  };
  if (split >= parts) { unused(split); return; }
  if (parts == 1 && a.splits > 1) unused(0);
  const uint32_t per = (sp.steps + parts - 1) / parts, end = std::min(sp.steps, (split + 1) * per);
  const uint32_t in_group = ht * AD_HEADS + col, head = kvh * a.group + in_group;
  const bool head_ok = in_group < a.group;

  bf16x8 fq[KW];
  {
    const bf16_t* qp = a.q + (size_t)i * a.ld_q + (size_t)(head_ok ? head : kvh * a.group) * DH + g * (DH / 4);
#pragma unroll
    for (uint32_t j = 0; j < KW; ++j) {
      uint4 v = *reinterpret_cast<const uint4*>(qp + j * 8);
      if (!head_ok) v = make_uint4(0, 0, 0, 0);
      fq[j] = as_bf16(v);
    }
  }
  const float c2 = a.scale * 1.44269504088896f;
  const size_t head_off = (size_t)kvh * (c.page_bytes / c.kv_heads), layer_off = (size_t)a.layer * c.n_pages;
  const unsigned char* kbase = c.k + layer_off * c.page_bytes + head_off;
  const unsigned char* vbase = c.v + layer_off * c.page_bytes + head_off;
  const int32_t* row = c.table + (size_t)(s >= 0 ? s : 0) * c.table_ld;
  const uint32_t page_mask = (1u << c.page_lg) - 1u, pages = kv_pages_of(c, sp.len), powers = (DH / 2) << c.page_lg;      // where a page's powers begin

  floatx4 oacc[DT];
#pragma unroll
  for (uint32_t d = 0; d < DT; ++d) oacc[d] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;

  struct Tile { uint32_t k[NT][KW]; uint4 v[NB]; uint32_t kpow, vpow, base; bool there; };
  auto base_of = [&](uint32_t step) { return step < sp.sink_steps ? step * TOK : sp.from + (step - sp.sink_steps) * TOK; };
  auto page_at = [&](uint32_t token) { const uint32_t slot = token >> c.page_lg; return slot < pages ? row[slot] : -1; };
  auto fetch = [&](Tile& t, uint32_t step, int32_t kp, int32_t vp) {
    t.base = base_of(step);
    t.there = (uint32_t)vp < c.n_pages;
    const uint32_t koff = (t.base + (col >> 2) * 16 + (col & 3) * 4) & page_mask, voff = (t.base + g * 16) & page_mask;
    const unsigned char* kp8 = kbase + (size_t)((uint32_t)kp < c.n_pages ? kp : 0) * c.page_bytes;
    const unsigned char* vp8 = vbase + (size_t)(t.there ? vp : 0) * c.page_bytes;
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n) {
      const unsigned char* at = kp8 + (koff + n) * (DH / 2) + g * (DH / 8);
      if constexpr (KW == 4) *reinterpret_cast<uint4*>(t.k[n]) = *reinterpret_cast<const uint4*>(at);
      else *reinterpret_cast<uint2*>(t.k[n]) = *reinterpret_cast<const uint2*>(at);
    }
    t.kpow = *reinterpret_cast<const uint32_t*>(kp8 + powers + ((g * DH / 128) << c.page_lg) + koff);
#pragma unroll
    for (uint32_t b = 0; b < NB; ++b) {
      const unsigned char* at = vp8 + ((b * 16 + col) << c.page_lg) + voff;
      if constexpr (STREAM) t.v[b] = fetch16(at); else t.v[b] = *reinterpret_cast<const uint4*>(at);
    }
    const unsigned char* at = vp8 + powers + (voff + col) * NB;
    if constexpr (NB == 4) t.vpow = *reinterpret_cast<const uint32_t*>(at); else t.vpow = *reinterpret_cast<const uint16_t*>(at);
  };
  auto use = [&](Tile& t) {
    floatx4 sc[NT];                                        // element e of sc[n]: token 4 e + n of the lane's sixteen
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n) {
      const float power = e2m1_power(t.kpow >> (8 * n) & 255u);
      sc[n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (uint32_t j = 0; j < KW; ++j) {
        const uint32_t w = t.k[n][j];
        sc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(make_uint4(e2m1x2<0>(w, power), e2m1x2<1>(w, power), e2m1x2<2>(w, power), e2m1x2<3>(w, power))), fq[j], sc[n], 0, 0, 0);
      }
      sc[n] *= c2;
    }
    float vp[NB];
#pragma unroll
    for (uint32_t b = 0; b < NB; ++b) vp[b] = e2m1_power(t.vpow >> (8 * b) & 255u);
    // masks: what is held in tokens that are not visible may be anything, and their powers NaN: scores become -inf, powers zero
    const uint32_t first = t.base + g * 16;
    const bool whole = t.base + TOK <= sp.len && (t.base >= sp.lo || t.base + TOK <= a.sinks);
    if (!whole || !__all(t.there)) {
      uint32_t keep = 0;
#pragma unroll
      for (uint32_t e = 0; e < 16; ++e) {
        const uint32_t tok = first + e;
        keep |= (t.there && tok < sp.len && (tok >= sp.lo || tok < a.sinks)) ? 1u << e : 0u;
      }
#pragma unroll
      for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) sc[n][e] = (keep >> (e * 4 + n)) & 1u ? sc[n][e] : -INFINITY;
#pragma unroll
      for (uint32_t b = 0; b < NB; ++b) vp[b] = (keep >> col) & 1u ? vp[b] : 0.f;
    }
    float mx = -INFINITY;
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) mx = fmaxf(mx, sc[n][e]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
    if (__any(m_new > m_run)) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
      l_run *= alpha;
#pragma unroll
      for (uint32_t d = 0; d < DT; ++d) oacc[d] *= alpha;
    }
    m_run = m_new;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e)
#pragma unroll
      for (uint32_t n = 0; n < NT; ++n) { sc[n][e] = __builtin_amdgcn_exp2f(sc[n][e] - m_use); l_run += sc[n][e]; }
#pragma unroll
    for (uint32_t b = 0; b < NB; ++b) {
      uint32_t pk[8];                                      // words 2 e and 2 e + 1: tokens 4 e .. 4 e + 3
      for_each(std::make_integer_sequence<int, 4>{}, [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        pk[2 * e] = pack_bf2(sc[0][e] * of_row<4 * e>(vp[b]), sc[1][e] * of_row<4 * e + 1>(vp[b]));
        pk[2 * e + 1] = pack_bf2(sc[2][e] * of_row<4 * e + 2>(vp[b]), sc[3][e] * of_row<4 * e + 3>(vp[b]));
      });
      const uint32_t w[4] = {t.v[b].x, t.v[b].y, t.v[b].z, t.v[b].w};
#pragma unroll
      for (uint32_t h = 0; h < 2; ++h) {
        uint32_t x[4];                                     // of four tokens' bytes one half each, two to a byte: bytes 0 and 2
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
          x[e] = (h == 0 ? w[e] : w[e] >> 4) & 0x0F0F0F0Fu;
          x[e] |= x[e] >> 4;
        }
#pragma unroll
        for (uint32_t o = 0; o < 2; ++o)
          oacc[2 * b + h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              as_bf16(make_uint4(e2m1x2<0>(x[2 * o], 1.f), e2m1x2<2>(x[2 * o], 1.f), e2m1x2<0>(x[2 * o + 1], 1.f), e2m1x2<2>(x[2 * o + 1], 1.f))),
              as_bf16(make_uint4(pk[4 * o], pk[4 * o + 1], pk[4 * o + 2], pk[4 * o + 3])), oacc[2 * b + h], 0, 0, 0);
      }
    }
  };
  // (every fourth of the split's steps, the next one's contents on the way, in front of them the page numbers of the one after that)
  auto kpage_of = [&](uint32_t step) { return step < end ? page_at(base_of(step) + (col >> 2) * 16) : -1; };
  auto vpage_of = [&](uint32_t step) { return step < end ? page_at(base_of(step) + g * 16) : -1; };
  uint32_t step = split * per + wave;
  if (step < end) {
    Tile t0, t1;
    int32_t kp = kpage_of(step), vp = vpage_of(step), kn = kpage_of(step + AD_WAVES), vn = vpage_of(step + AD_WAVES);
    fetch(t0, step, kp, vp);
    for (;;) {
      kp = kpage_of(step + 2 * AD_WAVES);
      vp = vpage_of(step + 2 * AD_WAVES);
      const bool more = step + AD_WAVES < end;
      if (more) fetch(t1, step + AD_WAVES, kn, vn);
      use(t0);
      if (!more) break;
      step += AD_WAVES;
      kn = kpage_of(step + 2 * AD_WAVES);
      vn = vpage_of(step + 2 * AD_WAVES);
      const bool more2 = step + AD_WAVES < end;
      if (more2) fetch(t0, step + AD_WAVES, kp, vp);
      use(t1);
      if (!more2) break;
      step += AD_WAVES;
    }
  }
  decode_finish<DH>(a, i, kvh, ht, split, parts, m_run, l_run, oacc, 1.f);
}

void launch_attn_decode4(const DecodeArgs& d, uint32_t d_head, dim3 grid, bool stream_v, hipStream_t s) {
#define AD4_LAUNCH(DH) \
  if (stream_v) hipLaunchKernelGGL((attn_decode4_kernel<DH, true>), grid, dim3(64 * AD_WAVES), 0, s, d); \
  else hipLaunchKernelGGL((attn_decode4_kernel<DH, false>), grid, dim3(64 * AD_WAVES), 0, s, d)
  if (d_head == 64) { AD4_LAUNCH(64); } else { AD4_LAUNCH(128); }
#undef AD4_LAUNCH
}

}  // namespace sif
