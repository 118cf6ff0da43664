// Attention of one new token per sequence over a paged cache: one launch, or two, per layer and token of a program that generates (no
// registered model does).
//
//   o = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale k_scale q k_j - m),   over the visible tokens j
//
// The cache is read once and nothing else is large, so the memory's rate is the bound (64 sequences of 1 to 8192 tokens, 8 kv heads of
// 128: 1.07 GB); the query heads that share a kv head are the columns of one matrix product, sixteen at a time, and cost nothing
// beside that.  A wavefront works on its own through steps of 32 tokens (64 of 8 bits) with a running maximum and sum, operands go
// from memory straight into the matrix units' registers, no LDS and no barrier until the end:
//
//   S^T = K Q^T    rows of a 16-row tile are tokens in an order of choice: row 4a + b of tile t is token a * (TOK / 4) + 4 t + b, so that a
//                  lane's results (column = query head, rows 4 (lane / 16) ..) are TOK / 4 consecutive tokens
//   O^T = V^T P^T  and these are the k elements that the next product wants from that lane; V is stored [d][token], its operand is 16
//                  consecutive bytes.
//
// Long sequences are cut over blocks, which leave (m, l, O) behind; a second launch joins them, in a fixed order.
#include <math.h>
#include <algorithm>

#include "attn_decode.h"

namespace sif {

// eight e4m3 values (two words) as bf16, exactly
__device__ __forceinline__ bf16x8 from_e4m3(uint32_t a, uint32_t b) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  u4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true));
  return __builtin_bit_cast(bf16x8, r);
}

// STREAM: a step is at least as long as a page, see fetch16.  Grid: (units = sequence x kv head x tile of 16 query heads, splits).
template <int DH, bool E4M3, bool STREAM>
__global__ __launch_bounds__(256, 2) void attn_decode_kernel(DecodeArgs a) {
  constexpr uint32_t TOK = E4M3 ? 64 : 32, NT = TOK / 16, ELT = E4M3 ? 1 : 2;
  constexpr uint32_t KL = DH * ELT / 64, DT = DH / 16;                 // 16-byte fetches of a lane per 16 keys; tiles of 16 d
  const KvView& c = a.c;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
  const uint32_t ht = blockIdx.x % a.head_tiles, kvh = blockIdx.x / a.head_tiles % c.kv_heads, i = blockIdx.x / a.head_tiles / c.kv_heads;
  const int32_t s = kv_listed(c, a.seqs, i);
  const DecodeSpan sp = decode_span<TOK>(s >= 0 ? kv_length(c, s) : 0u, a.window, a.sinks);
  const uint32_t parts = sp.steps == 0 ? 1u : std::min((sp.steps + a.chunk - 1) / a.chunk, a.splits), split = blockIdx.y;
  // what the join reads of splits that are not used
  auto unused = [&](uint32_t which) {
    if (threadIdx.x < std::min(a.group - ht * AD_HEADS, AD_HEADS))
      a.part[(((size_t)i * a.heads + kvh * a.group + ht * AD_HEADS + threadIdx.x) * a.splits + which) * (DH + 4) + 1] = kNoSplit;
  };
  if (split >= parts) { unused(split); return; }
  if (parts == 1 && a.splits > 1) unused(0);
  const uint32_t per = (sp.steps + parts - 1) / parts, end = std::min(sp.steps, (split + 1) * per);
  const uint32_t in_group = ht * AD_HEADS + col, head = kvh * a.group + in_group;
  const bool head_ok = in_group < a.group;

  bf16x8 fq[DH / 32];
  {
    const bf16_t* qp = a.q + (size_t)i * a.ld_q + (size_t)(head_ok ? head : kvh * a.group) * DH;
#pragma unroll
    for (uint32_t k = 0; k < DH / 32; ++k) {
      // the d of a k element: those of the key's fetch that lies in the same lane
      const uint32_t d = E4M3 ? (k >> 1) * 64 + g * 16 + (k & 1) * 8 : k * 32 + g * 8;
      uint4 v = *reinterpret_cast<const uint4*>(qp + d);
      if (!head_ok) v = make_uint4(0, 0, 0, 0);
      fq[k] = as_bf16(v);
    }
  }
  float c2 = a.scale * 1.44269504088896f;
  if (E4M3 && c.k_scale != nullptr) c2 *= c.k_scale[a.layer * c.kv_heads + kvh];
  const size_t head_off = (size_t)kvh * (c.page_bytes / c.kv_heads), layer_off = (size_t)a.layer * c.n_pages;
  const unsigned char* kbase = c.k + layer_off * c.page_bytes + head_off;
  const unsigned char* vbase = c.v + layer_off * c.page_bytes + head_off;
  const int32_t* row = c.table + (size_t)(s >= 0 ? s : 0) * c.table_ld;
  const uint32_t page_mask = (1u << c.page_lg) - 1u, pages = kv_pages_of(c, sp.len);

  floatx4 oacc[DT];
#pragma unroll
  for (uint32_t d = 0; d < DT; ++d) oacc[d] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;

  struct Tile { uint4 k[NT * KL], v[DT]; uint32_t base; bool there; };
  auto base_of = [&](uint32_t step) { return step < sp.sink_steps ? step * TOK : sp.from + (step - sp.sink_steps) * TOK; };
  // the pages of a step's tokens: a lane needs that of its key row's quarter and that of its own quarter
  auto page_at = [&](uint32_t token) { const uint32_t slot = token >> c.page_lg; return slot < pages ? row[slot] : -1; };
  auto fetch = [&](Tile& t, uint32_t step, int32_t kp, int32_t vp) {
    t.base = base_of(step);
    t.there = (uint32_t)vp < c.n_pages;
    const uint32_t ktok = t.base + (col >> 2) * (TOK / 4) + (col & 3), vtok = t.base + g * (TOK / 4);
    const unsigned char* kp8 = kbase + (size_t)((uint32_t)kp < c.n_pages ? kp : 0) * c.page_bytes + ((ktok & page_mask) * DH) * ELT + g * 16;
    const unsigned char* vp8 = vbase + (size_t)(t.there ? vp : 0) * c.page_bytes + ((col << c.page_lg) + (vtok & page_mask)) * ELT;
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
      for (uint32_t j = 0; j < KL; ++j) t.k[n * KL + j] = *reinterpret_cast<const uint4*>(kp8 + (n * 4 * DH) * ELT + j * 64);
    if constexpr (STREAM) {
#pragma unroll
      for (uint32_t d = 0; d < DT; ++d) t.v[d] = fetch16(vp8 + ((d * 16) << c.page_lg) * ELT);
    } else {
#pragma unroll
      for (uint32_t d = 0; d < DT; ++d) t.v[d] = *reinterpret_cast<const uint4*>(vp8 + ((d * 16) << c.page_lg) * ELT);
    }
  };
  auto use = [&](Tile& t) {
    floatx4 sc[NT];
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n) {
      sc[n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (uint32_t j = 0; j < KL; ++j) {
        const uint4& kv = t.k[n * KL + j];
        if constexpr (E4M3) {
          sc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(from_e4m3(kv.x, kv.y), fq[2 * j], sc[n], 0, 0, 0);
          sc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(from_e4m3(kv.z, kv.w), fq[2 * j + 1], sc[n], 0, 0, 0);
        } else {
          sc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(kv), fq[j], sc[n], 0, 0, 0);
        }
      }
      sc[n] *= c2;                                         // (in front of the mask: a scale of the cache may be 0 or negative)
    }
    // masks: only steps that hold the end, the border of the window or of the sinks, or a quarter without a page.  What is held there may
    // be anything, a NaN too: scores become -inf, values zero.
    const uint32_t first = t.base + g * (TOK / 4);
    const bool whole = t.base + TOK <= sp.len && (t.base >= sp.lo || t.base + TOK <= a.sinks);
    if (!whole || !__all(t.there)) {
      uint32_t keep = 0;                                   // bit e: token first + e is visible
#pragma unroll
      for (uint32_t e = 0; e < TOK / 4; ++e) {
        const uint32_t tok = first + e;
        keep |= (t.there && tok < sp.len && (tok >= sp.lo || tok < a.sinks)) ? 1u << e : 0u;
      }
#pragma unroll
      for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) sc[n][e] = (keep >> (n * 4 + e)) & 1u ? sc[n][e] : -INFINITY;
      uint32_t mk[4];
#pragma unroll
      for (uint32_t w = 0; w < 4; ++w) {
        mk[w] = 0;
        constexpr uint32_t PER = 4 / ELT, BITS = 8 * ELT;
#pragma unroll
        for (uint32_t b = 0; b < PER; ++b) mk[w] |= (keep >> (w * PER + b)) & 1u ? ((1u << BITS) - 1u) << (b * BITS) : 0u;
      }
#pragma unroll
      for (uint32_t d = 0; d < DT; ++d) { t.v[d].x &= mk[0]; t.v[d].y &= mk[1]; t.v[d].z &= mk[2]; t.v[d].w &= mk[3]; }
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
    uint32_t pk[NT * 2];
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n) {
      float p[4];
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) { p[e] = __builtin_amdgcn_exp2f(sc[n][e] - m_use); l_run += p[e]; }
      pk[2 * n] = pack_bf2(p[0], p[1]);
      pk[2 * n + 1] = pack_bf2(p[2], p[3]);
    }
#pragma unroll
    for (uint32_t d = 0; d < DT; ++d) {
      if constexpr (E4M3) {
        oacc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(from_e4m3(t.v[d].x, t.v[d].y), as_bf16(make_uint4(pk[0], pk[1], pk[2], pk[3])), oacc[d], 0, 0, 0);
        oacc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(from_e4m3(t.v[d].z, t.v[d].w), as_bf16(make_uint4(pk[4], pk[5], pk[6], pk[7])), oacc[d], 0, 0, 0);
      } else {
        oacc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(t.v[d]), as_bf16(make_uint4(pk[0], pk[1], pk[2], pk[3])), oacc[d], 0, 0, 0);
      }
    }
  };
  // A wavefront's steps: every fourth of the split's.  While one is used the next one's contents are on the way, and in front of these the
  // page numbers of the one after that: loads complete in order, so numbers asked for behind the contents would be waited for with
  // them.  (A quarter of the split's steps each, one after the other: one sequence of 262011 tokens 186 -> 207 us.)
  auto kpage_of = [&](uint32_t step) { return step < end ? page_at(base_of(step) + (col >> 2) * (TOK / 4)) : -1; };
  auto vpage_of = [&](uint32_t step) { return step < end ? page_at(base_of(step) + g * (TOK / 4)) : -1; };
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
  decode_finish<DH>(a, i, kvh, ht, split, parts, m_run, l_run, oacc, E4M3 && c.v_scale != nullptr ? c.v_scale[a.layer * c.kv_heads + kvh] : 1.f);
}

// Joins a row's splits: one block per (sequence, query head).  First every split's weight, then the weighted sum, DH / 4 lanes to a split.
template <int DH>
__global__ __launch_bounds__(256) void attn_decode_join_kernel(DecodeArgs a) {
  constexpr uint32_t LANES = DH / 4, ROWS = 256 / LANES;
  static_assert(AD_BLOCKS == 256, "a thread per split");
  __shared__ float s_w[AD_BLOCKS];
  __shared__ __align__(16) float4 s_o[256];
  __shared__ float sm[16];
  const uint32_t t = threadIdx.x, head = blockIdx.x % a.heads, i = blockIdx.x / a.heads;
  const float* from = a.part + ((size_t)i * a.heads + head) * a.splits * (DH + 4);
  // Everything that is known only on the device - how many splits the sequence has - stands in the splits themselves: the first
  // `parts` have an l, the others kNoSplit (all of them if one block did the whole sequence).  So there are two rounds of loads, and not the
  // length's and the list's before them.
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  float m, l;
  if (a.splits <= 64) {
    // A split per lane, in every wavefront: no barriers, and the splits' rows on their way beside the sums (of splits that are none too: anything, not looked at).  The same operations in the same order as
    // below.  (One sequence in 4 bits, heads of 128, the whole call: 1000 tokens 10.6 -> 8.3 us, 100000 27.9 -> 25.3; 64 of 1 to 8192 75 -> 74.)
    const uint32_t lane = t & 63, first = t / LANES;
    float2 ml = make_float2(-INFINITY, kNoSplit);
    if (lane < a.splits) ml = *reinterpret_cast<const float2*>(from + (size_t)lane * (DH + 4));
    float4 v[64 / ROWS];
#pragma unroll
    for (uint32_t round = 0; round < 64 / ROWS; ++round)
      if (round * ROWS < a.splits) v[round] = *reinterpret_cast<const float4*>(from + (size_t)std::min(round * ROWS + first, a.splits - 1) * (DH + 4) + 4 + t % LANES * 4);
    const bool here = ml.y != kNoSplit;
    const uint32_t parts = (uint32_t)__popcll(__ballot(here));
    if (parts == 0) return;
    m = wave_max(here ? ml.x : -INFINITY);
    const float w = here && m != -INFINITY ? __builtin_amdgcn_exp2f(ml.x - m) : 0.f;
    l = wave_sum(here ? w * ml.y : 0.f);
#pragma unroll
    for (uint32_t round = 0; round < 64 / ROWS; ++round)
      if (round * ROWS < parts) {
        const uint32_t p = round * ROWS + first;
        const float f = __shfl(w, p, 64);
        if (p < parts) { y.x += f * v[round].x; y.y += f * v[round].y; y.z += f * v[round].z; y.w += f * v[round].w; }
      }
  } else {
    float2 ml = make_float2(-INFINITY, kNoSplit);
    if (t < a.splits) ml = *reinterpret_cast<const float2*>(from + (size_t)t * (DH + 4));
    const bool here = ml.y != kNoSplit;
    const uint32_t parts = (uint32_t)block_sum(here ? 1.f : 0.f, sm);
    if (parts == 0) return;
    m = block_max(here ? ml.x : -INFINITY, sm);
    const float w = here && m != -INFINITY ? __builtin_amdgcn_exp2f(ml.x - m) : 0.f;
    s_w[t] = w;
    l = block_sum(here ? w * ml.y : 0.f, sm);      // (its barriers stand behind the weights too)
#pragma unroll 8
    for (uint32_t p = t / LANES; p < parts; p += ROWS) {
      const float4 v = *reinterpret_cast<const float4*>(from + (size_t)p * (DH + 4) + 4 + t % LANES * 4);
      const float f = s_w[p];
      y.x += f * v.x; y.y += f * v.y; y.z += f * v.z; y.w += f * v.w;
    }
  }
  s_o[t] = y;
  __syncthreads();
  if (t >= LANES) return;
#pragma unroll
  for (uint32_t r = 1; r < ROWS; ++r) {
    const float4 v = s_o[r * LANES + t];
    y.x += v.x; y.y += v.y; y.z += v.z; y.w += v.w;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  *reinterpret_cast<uint2*>(a.o + (size_t)i * a.ld_o + (size_t)head * DH + t * 4) = make_uint2(pack_bf2(y.x * inv, y.y * inv), pack_bf2(y.z * inv, y.w * inv));
  if (t == 0 && a.lse != nullptr) a.lse[(size_t)i * a.heads + head] = (m + __log2f(l)) * 0.693147180559945f;
}

// How the work is divided.  A CU takes in some 47 KB per us whatever its wavefronts do, so a launch wants all CUs: splits of at least one
// step per wavefront until there is a block for each of the 256 CUs.  (One sequence, 8 kv heads of 128: 1000 tokens 14.0 -> 8.5 us,
// 8000 87 -> 11.5, 30000 325 -> 26.5, the join's 4 to 5 us included.)  Past that, up to eight blocks per CU, only where there are several
// sequences, and in splits of 2048 tokens or more: where lengths differ, which is not known here, the long sequences' ends are then shared
// (pages of 16: 32 sequences of 1 to 8000 tokens 112 -> 89 us, 64 of 1 to 8192 200 -> 193, 128 of 1 to 8000 389 -> 350, three of 100 to
// 262011 375 -> 280; pages of 64: 139 -> 112, 237 -> 220, 451 -> 404, 463 -> 318), where they do not, that costs the splits' own ends and
// the join (64 of 4096 170 -> 177, of 64-token pages 188 -> 197; 16 of 8000 85 -> 89 and 99 -> 112; 32 of 4000 the same; one of 262011
// 189 -> 198 in pages of 64).  Splits that may be as short as a step cost more (128 of 500 13 -> 21), of 1024 tokens too (64 of 4096 182),
// of 4096 leave 32 of 1 to 8000 at 111.
// In 4 bits two blocks for each CU: a step is as long in time as there, but half of it is a wavefront's own work, and one wavefront on a SIMD leaves the memory idle meanwhile (one
// sequence of 262011 tokens 70 -> 56 us); splits of 1366 to 4096 tokens all take 75 to 78 us for 64 sequences of 1 to 8192.
static sif_status decode_plan(const char* who, const sif_kv_cache* c, const sif_attn_decode_args* a, DecodeArgs* out, uint64_t* bytes) {
  if (sif_status st = kv_check(who, c, &out->c)) return st;
  if (!a) return fail(SIF_E_INVAL, "%s: null arguments", who);
  if (a->struct_size != sizeof(sif_attn_decode_args)) return fail(SIF_E_INVAL, "%s: struct_size", who);
  if (a->layer >= c->layers) return fail(SIF_E_INVAL, "%s: no layer %u", who, a->layer);
  if (!a->n || !a->heads || a->heads % c->kv_heads) return fail(SIF_E_INVAL, "%s: no sequences, or heads not a multiple of kv_heads", who);
  if (!(a->scale >= 0.f) || !std::isfinite(a->scale * 1.44269504088896f)) return fail(SIF_E_INVAL, "%s: scale must be finite (in base 2 too) and not negative", who);
  const uint32_t tok = c->dtype == SIF_BF16 ? 32u : 64u;
  out->seqs = a->seqs_dev;
  out->layer = a->layer;
  out->n = a->n;
  out->heads = a->heads;
  out->group = a->heads / c->kv_heads;
  out->head_tiles = (out->group + AD_HEADS - 1) / AD_HEADS;
  out->window = a->window;
  out->sinks = a->sinks;
  const uint64_t units = (uint64_t)a->n * c->kv_heads * out->head_tiles;
  if ((uint64_t)a->n * a->heads >= 1ull << 23) return fail(SIF_E_INVAL, "%s: n * heads below 2^23", who);       // threads of a grid stay below 2^32
  uint64_t seen = a->max_tokens != 0 ? a->max_tokens : (uint64_t)c->table_ld * c->page_tokens;
  if (a->window != 0) seen = std::min<uint64_t>(seen, (uint64_t)a->window + a->sinks + 2 * tok);
  const uint64_t steps = std::max<uint64_t>(1, (seen + tok - 1) / tok);
  const uint64_t most = std::max<uint64_t>(1, steps / AD_WAVES);
  const uint64_t one = std::min<uint64_t>(most, (c->dtype == SIF_E2M1 ? 2 : 1) * AD_BLOCKS / units), eight = a->n > 1 ? std::min<uint64_t>(seen / 2048, 8 * AD_BLOCKS / units) : 0;
  out->splits = (uint32_t)std::min<uint64_t>(AD_BLOCKS, std::max<uint64_t>(1, std::max(one, eight)));
  out->chunk = (uint32_t)((steps + out->splits - 1) / out->splits);
  *bytes = out->splits > 1 ? (uint64_t)a->n * a->heads * out->splits * (c->d_head + 4) * sizeof(float) : 256;
  return SIF_OK;
}

}  // namespace sif

using namespace sif;

extern "C" {

uint64_t sif_attn_decode_workspace_bytes(const sif_kv_cache* c, const sif_attn_decode_args* a) {
  DecodeArgs d;
  uint64_t bytes;
  return decode_plan("attn_decode_workspace_bytes", c, a, &d, &bytes) == SIF_OK ? bytes : 0;
}

sif_status sif_k_attn_decode(const sif_kv_cache* c, const sif_attn_decode_args* a, void* stream) {
  DecodeArgs d;
  uint64_t bytes;
  if (sif_status st = decode_plan("attn_decode", c, a, &d, &bytes)) return st;
  const uint32_t width = a->heads * c->d_head;
  if (!a->q_dev || !a->o_dev) return fail(SIF_E_INVAL, "attn_decode: null operand");
  if (((uintptr_t)a->q_dev | (uintptr_t)a->o_dev) & 15) return fail(SIF_E_INVAL, "attn_decode: q and o must be 16-byte aligned");
  if (((uintptr_t)a->lse_dev | (uintptr_t)a->seqs_dev) & 3) return fail(SIF_E_INVAL, "attn_decode: misaligned operand");
  if (a->ld_q < width || a->ld_o < width || ((a->ld_q | a->ld_o) & 7)) return fail(SIF_E_INVAL, "attn_decode: bad leading dimensions");
  if (d.splits > 1) {
    if (!a->workspace_dev || ((uintptr_t)a->workspace_dev & 255)) return fail(SIF_E_INVAL, "attn_decode: the workspace must be 256-byte aligned");
    if (a->workspace_bytes < bytes)
      return fail(SIF_E_NOMEM, "attn_decode: the workspace holds %llu of %llu bytes", (unsigned long long)a->workspace_bytes, (unsigned long long)bytes);
  }
  d.q = (const bf16_t*)a->q_dev;
  d.o = (bf16_t*)a->o_dev;
  d.lse = a->lse_dev;
  d.part = (float*)a->workspace_dev;
  d.ld_q = a->ld_q;
  d.ld_o = a->ld_o;
  d.scale = a->scale != 0.f ? a->scale : 1.0f / sqrtf((float)c->d_head);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 grid(d.n * d.c.kv_heads * d.head_tiles, d.splits);
  const bool stream_v = c->page_tokens <= (c->dtype == SIF_BF16 ? 32u : 64u) && d.head_tiles == 1;       // see fetch16; a second tile of heads reads it again
#define AD_LAUNCH(DH, E) \
  if (stream_v) hipLaunchKernelGGL((attn_decode_kernel<DH, E, true>), grid, dim3(64 * AD_WAVES), 0, s, d); \
  else hipLaunchKernelGGL((attn_decode_kernel<DH, E, false>), grid, dim3(64 * AD_WAVES), 0, s, d)
  if (c->dtype == SIF_E2M1) {
    launch_attn_decode4(d, c->d_head, grid, stream_v, s);
  } else if (c->d_head == 64) {
    if (c->dtype == SIF_E4M3) { AD_LAUNCH(64, true); } else { AD_LAUNCH(64, false); }
  } else {
    if (c->dtype == SIF_E4M3) { AD_LAUNCH(128, true); } else { AD_LAUNCH(128, false); }
  }
#undef AD_LAUNCH
  if (sif_status st = check_launch("attn_decode")) return st;
  if (d.splits > 1) {
    if (c->d_head == 64) hipLaunchKernelGGL((attn_decode_join_kernel<64>), dim3(d.n * d.heads), dim3(256), 0, s, d);
    else hipLaunchKernelGGL((attn_decode_join_kernel<128>), dim3(d.n * d.heads), dim3(256), 0, s, d);
    return check_launch("attn_decode: join");
  }
  return SIF_OK;
}

}  // extern "C"
