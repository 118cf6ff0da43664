// Attention of one new token per sequence over a paged cache in 4 bits (the formulas and the division of the work: attn_decode.hip).
//
// A token of a kv head of 128 is 136 bytes, so that what the memory delivers in a given time is four times as many tokens as in bf16 and the vector units have to
// keep up.  A wavefront's step is 64 tokens:
//
//   S^T = K Q^T    K is brought to bf16 by the conversion instruction, which takes the powers along; a lane (row, g) has a quarter of its token's d, which one power goes with.  Row 4a + b of
//                  tile t is token 16 a + 4 t + b, and its powers are byte b of word t of a 16-byte fetch.
//   O^T = V^T P^T  byte (b, c) of a token holds d = 32 b + c and d + 16.  The conversion makes a pair of it, times the token's power, and a pair is two elements of a product's k
//                  as well as any: P stands in one and zero in the other, first for the tile of d, then for that of d + 16.  That is twice the products for no shuffles at all;
//                  the matrix units have the time.  Lane (c, g) has the powers of token 16 g + c and hands them to the others of its sixteen.
//
// Measured (64 sequences of 1 to 8192 tokens, 8 kv heads of 128, 286 MB): 75 us with the join's 5, 4.1 TB/s without it; loads alone, with nothing done to what they bring, 65.  With
// V's halves brought together by masks and shifts and its powers multiplied into P it was 82 us; with K's tokens in the order of the matrix rows, so that a
// fetch took half a line, 79.5; with V through the caches 4 to 6 us more for sequences of equal length; with three blocks a CU registers spill (151).  One sequence of 262011 tokens: 56 us with the join's 5, 5.6 TB/s.
// The matrix units also take K's numbers and powers as they lie (16x16x128, numbers of 4 bits by such of 8, q as the sum of two), 73.4 and 53.4 us, but add eight neighbouring products with no more than
// 13 bits below the largest exponent among them: where elements of q differ by 2^8 and more, scores were off by up to 2^-14.6 of what is added, in bf16 by 2^-23.6.
// What P loses by its rounding to bf16, up to 2^-8 of each, is what a bf16 result loses: 0.0021 to 0.0022 in the norm where rounding the exact result gives 0.0016.
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

// With this power and the one above it the numbers 4 and 6 are past the largest in bf16: they would become infinite, and infinite times a zero on the other side is NaN.
constexpr float kFarPower = 0x1p126f;

template <int DH, bool STREAM>
__global__ __launch_bounds__(256, 2) void attn_decode4_kernel(DecodeArgs a) {
  constexpr uint32_t TOK = 64, NT = 4, NB = DH / 32, KW = DH / 32, DT = DH / 16;      // tiles of 16 tokens; powers of a token; words of a lane's d
  const KvView& c = a.c;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;      // (steps are scalars)
  const uint32_t ht = blockIdx.x % a.head_tiles, kvh = blockIdx.x / a.head_tiles % c.kv_heads, i = blockIdx.x / a.head_tiles / c.kv_heads;
  // the query first, looked at when the first contents are on their way: from the list to the length, the table and the pages there are four round trips
  const uint32_t in_group = ht * AD_HEADS + col, head = kvh * a.group + in_group;
  const bool head_ok = in_group < a.group;
  const bf16_t* qp = a.q + (size_t)i * a.ld_q + (size_t)(head_ok ? head : kvh * a.group) * DH;
  uint4 xq[KW];
#pragma unroll
  for (uint32_t j = 0; j < KW; ++j) xq[j] = *reinterpret_cast<const uint4*>(qp + g * (DH / 4) + j * 8);
  const int32_t s = kv_listed(c, a.seqs, i);
  const DecodeSpan sp = decode_span<TOK>(s >= 0 ? kv_length(c, s) : 0u, a.window, a.sinks);
  const uint32_t parts = sp.steps == 0 ? 1u : std::min((sp.steps + a.chunk - 1) / a.chunk, a.splits), split = a.splits - 1 - blockIdx.y;      // (the last splits, which only long sequences have, first)
  auto unused = [&](uint32_t which) {
    if (threadIdx.x < std::min(a.group - ht * AD_HEADS, AD_HEADS))
      a.part[(((size_t)i * a.heads + kvh * a.group + ht * AD_HEADS + threadIdx.x) * a.splits + which) * (DH + 4) + 1] = kNoSplit;
  };
  if (split >= parts) { unused(split); return; }
  if (parts == 1 && a.splits > 1) unused(0);
  const uint32_t per = (sp.steps + parts - 1) / parts, end = std::min(sp.steps, (split + 1) * per);
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
  bf16x8 fq[KW];

  struct Tile { uint32_t k[NT][KW]; uint4 v[NB]; uint4 kpow; uint32_t vpow, base; bool there; };
  auto base_of = [&](uint32_t step) { return step < sp.sink_steps ? step * TOK : sp.from + (step - sp.sink_steps) * TOK; };
  auto page_at = [&](uint32_t token) { const uint32_t slot = token >> c.page_lg; return slot < pages ? row[slot] : -1; };
  auto fetch = [&](Tile& t, uint32_t step, int32_t kp, int32_t vp) {
    t.base = base_of(step);
    t.there = (uint32_t)vp < c.n_pages;
    const uint32_t koff = (t.base + (col >> 2) * 16 + (col & 3)) & page_mask, voff = (t.base + g * 16) & page_mask;
    const unsigned char* kp8 = kbase + (size_t)((uint32_t)kp < c.n_pages ? kp : 0) * c.page_bytes;
    const unsigned char* vp8 = vbase + (size_t)(t.there ? vp : 0) * c.page_bytes;
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n) {
      const unsigned char* at = kp8 + (koff + 4 * n) * (DH / 2) + g * (DH / 8);
      if constexpr (KW == 4) *reinterpret_cast<uint4*>(t.k[n]) = *reinterpret_cast<const uint4*>(at);
      else *reinterpret_cast<uint2*>(t.k[n]) = *reinterpret_cast<const uint2*>(at);
    }
    t.kpow = *reinterpret_cast<const uint4*>(kp8 + powers + ((g * DH / 128) << c.page_lg) + (koff & ~15u));
#pragma unroll
    for (uint32_t b = 0; b < NB; ++b) {
      const unsigned char* at = vp8 + ((b * 16 + col) << c.page_lg) + voff;
      if constexpr (STREAM) t.v[b] = fetch16(at); else t.v[b] = *reinterpret_cast<const uint4*>(at);
    }
    const unsigned char* at = vp8 + powers + (voff + col) * NB;
    if constexpr (NB == 4) t.vpow = *reinterpret_cast<const uint32_t*>(at); else t.vpow = *reinterpret_cast<const uint16_t*>(at);
  };
  auto use = [&](Tile& t) {
    floatx4 sc[NT];                                        // element e of sc[n]: token 4 n + e of the lane's sixteen
    auto score = [&](floatx4& to, const uint32_t (&k)[KW], float power) {
#pragma unroll
      for (uint32_t j = 0; j < KW; ++j)
        to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(make_uint4(e2m1x2<0>(k[j], power), e2m1x2<1>(k[j], power), e2m1x2<2>(k[j], power), e2m1x2<3>(k[j], power))), fq[j], to, 0, 0, 0);
    };
    float power[NT];
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n) {
      power[n] = e2m1_power((n == 0 ? t.kpow.x : n == 1 ? t.kpow.y : n == 2 ? t.kpow.z : t.kpow.w) >> (8 * (col & 3)) & 255u);
      sc[n] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    if (!__any(fmaxf(fmaxf(power[0], power[1]), fmaxf(power[2], power[3])) >= kFarPower)) {      // (NaN is not the largest of numbers)
#pragma unroll
      for (uint32_t n = 0; n < NT; ++n) score(sc[n], t.k[n], power[n]);
    } else {
      // such keys at a quarter of themselves, into a sum of their own
#pragma unroll
      for (uint32_t n = 0; n < NT; ++n) {
        uint32_t others[KW], those[KW];
        floatx4 quarter = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (uint32_t j = 0; j < KW; ++j) {
          others[j] = power[n] >= kFarPower ? 0u : t.k[n][j];
          those[j] = power[n] >= kFarPower ? t.k[n][j] : 0u;
        }
        score(sc[n], others, power[n]);
        score(quarter, those, 0.25f * power[n]);
        sc[n] += 4.f * quarter;
      }
    }
    float vp[NB];
#pragma unroll
    for (uint32_t b = 0; b < NB; ++b) vp[b] = e2m1_power(t.vpow >> (8 * b) & 255u);
    // masks: what is held in tokens that are not visible may be anything, and their powers NaN: scores become -inf, powers of two any number
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
        for (uint32_t e = 0; e < 4; ++e) sc[n][e] = (keep >> (n * 4 + e)) & 1u ? sc[n][e] : -INFINITY;
#pragma unroll
      for (uint32_t b = 0; b < NB; ++b) vp[b] = (keep >> col) & 1u ? vp[b] : 1.f;
    }
    // (the scale is above 0: the largest product is the largest score; the maximum is kept as a score, base 2)
    float mx = -INFINITY;
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) mx = fmaxf(mx, sc[n][e]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c2;
    const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
    if (__any(m_new > m_run)) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
      l_run *= alpha;
#pragma unroll
      for (uint32_t d = 0; d < DT; ++d) oacc[d] *= alpha;
    }
    m_run = m_new;
    // FAR: of a token and 32 d with such a power a quarter of the values, and four times P.
    auto weigh = [&](auto with_far) {
      constexpr bool FAR = decltype(with_far)::value;
      float times[NB];
#pragma unroll
      for (uint32_t b = 0; b < NB; ++b) {
        times[b] = FAR && vp[b] >= kFarPower ? 4.f : 1.f;
        if constexpr (FAR) vp[b] /= times[b];
      }
      for_each(std::make_integer_sequence<int, 4>{}, [&](auto nc) {
        constexpr int n = decltype(nc)::value;               // tokens 4 n .. 4 n + 3
        float p[4];
        uint32_t lo_p[4], hi_p[4];                           // beside d, beside d + 16
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(sc[n][e], c2, -m_use));
          l_run += p[e];
          lo_p[e] = pack_bf2(p[e], 0.f);
          hi_p[e] = lo_p[e] << 16;
        }
#pragma unroll
        for (uint32_t b = 0; b < NB; ++b) {
          const uint32_t w = n == 0 ? t.v[b].x : n == 1 ? t.v[b].y : n == 2 ? t.v[b].z : t.v[b].w;
          const bf16x8 x = as_bf16(make_uint4(e2m1x2<0>(w, of_row<4 * n>(vp[b])), e2m1x2<1>(w, of_row<4 * n + 1>(vp[b])),
                                              e2m1x2<2>(w, of_row<4 * n + 2>(vp[b])), e2m1x2<3>(w, of_row<4 * n + 3>(vp[b]))));
          if constexpr (FAR) {
            const float f[4] = {of_row<4 * n>(times[b]), of_row<4 * n + 1>(times[b]), of_row<4 * n + 2>(times[b]), of_row<4 * n + 3>(times[b])};
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
              lo_p[e] = pack_bf2(p[e] * f[e], 0.f);
              hi_p[e] = lo_p[e] << 16;
            }
          }
          oacc[2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, as_bf16(make_uint4(lo_p[0], lo_p[1], lo_p[2], lo_p[3])), oacc[2 * b], 0, 0, 0);
          oacc[2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, as_bf16(make_uint4(hi_p[0], hi_p[1], hi_p[2], hi_p[3])), oacc[2 * b + 1], 0, 0, 0);
        }
      });
    };
    float most = vp[0];
#pragma unroll
    for (uint32_t b = 1; b < NB; ++b) most = fmaxf(most, vp[b]);
    if (!__any(most >= kFarPower)) weigh(std::false_type{}); else weigh(std::true_type{});
  };
  // Every fourth of the split's steps, the next one's contents on the way, in front of them the page numbers of the one after that.  Behind the last step it is fetched
  // once more: a fetch under a condition would make every step wait for all that is under way.
  const uint32_t mine = split * per + wave;
  if (mine < end) {
    const uint32_t last = mine + (end - 1 - mine) / AD_WAVES * AD_WAVES;
    auto kpage_of = [&](uint32_t step) { return page_at(base_of(std::min(step, last)) + (col >> 2) * 16); };
    auto vpage_of = [&](uint32_t step) { return page_at(base_of(std::min(step, last)) + g * 16); };
    Tile t0, t1;
    uint32_t step = mine;
    int32_t kp = kpage_of(step), vp = vpage_of(step), kn = kpage_of(step + AD_WAVES), vn = vpage_of(step + AD_WAVES);
    fetch(t0, step, kp, vp);
#pragma unroll
    for (uint32_t j = 0; j < KW; ++j) fq[j] = as_bf16(head_ok ? xq[j] : make_uint4(0, 0, 0, 0));
    for (;;) {
      kp = kpage_of(step + 2 * AD_WAVES);
      vp = vpage_of(step + 2 * AD_WAVES);
      fetch(t1, std::min(step + AD_WAVES, last), kn, vn);
      use(t0);
      if (step == last) break;
      step += AD_WAVES;
      kn = kpage_of(step + 2 * AD_WAVES);
      vn = vpage_of(step + 2 * AD_WAVES);
      fetch(t0, std::min(step + AD_WAVES, last), kp, vp);
      use(t1);
      if (step == last) break;
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
