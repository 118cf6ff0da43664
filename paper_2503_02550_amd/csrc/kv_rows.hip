// New keys and values into a paged cache with the rotation by position on the way, and rows back out of it, for all formats of a cache.
//
// Rows are read and written once and nothing else is large: the memory's rate is the bound, or for a token per sequence the chain of list, length,
// table and page.  A block takes sixteen rows and some of their heads: it finds the rows' sequences, positions and pages, takes the sines of its rows' angles
// once, and walks the heads.  Keys go out as the vectors they come in as; values pass through LDS, so that lanes which are neighbours in a page's
// row of tokens store neighbouring elements.
//
// Measured: 24600 rows into 4 bits, 32 heads turned and 8 key heads of 128 written, 531 MB: 122 us, 4.4 TB/s; 33000 rows read back, 171 MB: 40 us, 4.3 TB/s (values leave and come in a byte or two
// at a time).  A token for each of 128 sequences 7.5 us, for four 4.7, of which the launch is 3: in front of the heads stand the list, the length, the table and the sines, each waiting for
// the one before.  With the first vectors on their way meanwhile and the lists read sixteen entries at a time appending these 24600 rows took 126.5 us for 129.6, with four heads at a time in place of
// one reading back 43 for 69.6.
//
// Formats of 8 and 4 bits: a turned key next to the border between two values goes to one or the other by its last bits, and a step is up to a
// third of the value.  So sines, products and the search for the largest of 32 are in 64 bits there (which cost what those in 32 bits do on this chip), and what is
// rounded once more on its way to 4 bits, to fp32, is rounded to odd: fp32 numbers that are borders are even, so nothing reaches a border that did
// not lie on it.
#include <algorithm>

#include "e2m1.h"
#include "kv_rows.h"
#include "rope.h"

namespace sif {

struct KvAppend {
  KvView c;
  KvRowList l;
  const bf16_t* k;
  const bf16_t* v;
  const bf16_t* q;
  bf16_t* q_out;
  uint32_t layer, heads, ld_q, ld_q_out, ld_k, ld_v;
  uint32_t kv_blocks;                // blocks along y that write the cache; the others turn q
  uint32_t tiles_lg;                 // see kv_tile
  uint32_t q_copies;                 // units of sixteen elements of q behind the rotated ones, where q_out is not q
};

// to fp32, inexact numbers to the neighbour with an odd last bit
__device__ __forceinline__ float kv_round_odd(double x) {
  const float f = (float)x;
  const double back = (double)f;
  uint32_t u = __float_as_uint(f);
  if (back != x) u = (u - (fabs(back) > fabs(x) ? 1u : 0u)) | 1u;      // (NaN stays one: its last bit is set)
  return __uint_as_float(u);
}

// The exponent that 32 elements share, from the largest one's bits without the sign, of a number that is 2^-up of it: the smallest e with |x| <= 7 2^e.  255 as a byte: NaN.
struct KvPower { int e; uint32_t byte; };
__device__ __forceinline__ KvPower kv_power(uint32_t top, int up) {
  if (top > 0x7F800000u) return {0, 255u};
  if (top == 0x7F800000u) return {126, 253u};                                           // an infinity: as the largest number in bf16, 1.99 * 2^127
  const float x = __uint_as_float(top);
  int e = __builtin_amdgcn_frexp_expf(x) + up - (__builtin_amdgcn_frexp_mantf(x) <= 0.875f ? 3 : 2);
  if (top == 0) e = -127;
  e = std::min(std::max(e, -127), 127);
  return {e, (uint32_t)(e + 127)};
}
// eight floats over 2^e as 4-bit codes, the first in the lowest bits; infinities are held at +-6
__device__ __forceinline__ uint32_t kv_codes8(const float (&x)[8], int e) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = ldexpf(x[i], -e);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.f, 3);
  return w;
}
// the four 4-bit codes of a half word, a byte each
__device__ __forceinline__ uint32_t kv_spread4(uint32_t h) {
  h = (h | (h << 8)) & 0x00FF00FFu;
  return (h | (h << 4)) & 0x0F0F0F0Fu;
}
__device__ __forceinline__ uint32_t kv_largest_of_4(uint32_t x) {      // of four neighbouring lanes
  x = std::max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));
  return std::max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));
}
typedef uint32_t u32x4_kv __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 kv_uint4(const u32x4_kv& x) { return make_uint4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void kv_unpack8(const uint4& x, float (&f)[8]) {
  f[0] = bflo(x.x); f[1] = bfhi(x.x); f[2] = bflo(x.y); f[3] = bfhi(x.y);
  f[4] = bflo(x.z); f[5] = bfhi(x.z); f[6] = bflo(x.w); f[7] = bfhi(x.w);
}

// Bytes of a kv head's part of a page, and of the elements in front of its powers.
template <int DH, uint32_t FMT> __device__ __forceinline__ uint32_t kv_head_bytes(uint32_t page_lg) {
  return FMT == SIF_BF16 ? (DH * 2) << page_lg : FMT == SIF_E4M3 ? DH << page_lg : (DH / 32 * 17) << page_lg;
}

// Which sixteen rows a block takes.  A line of a page's values holds more tokens than these sixteen rows where pages are longer, and blocks go to the eight XCDs in turn: 2^lg tiles, a
// page's, go to one of them together, so that one L2 gets the whole line.  (16 prompts of 1024 tokens, 8 heads of 128, pages of 64, bf16: appending with 32 query heads 98.5 -> 87 us, reading back 32.6 -> 19.8;
// pages of 256: 104 -> 87, 33.7 -> 21.)
__device__ __forceinline__ uint32_t kv_tile(uint32_t x, uint32_t lg) {
  return (x >> (3 + lg) << (3 + lg)) + ((x & 7) << lg) + (x >> 3 & ((1u << lg) - 1u));
}
static uint32_t kv_tiles_lg(const KvView& c, const KvRowList& l) { return l.starts != nullptr ? c.page_lg - 4 : 0; }      // (without starts every row is another page's)
static uint32_t kv_grid_x(uint32_t tiles, uint32_t lg) { return lg == 0 ? tiles : (tiles + (8u << lg) - 1) >> (3 + lg) << (3 + lg); }

// grid: (sixteen rows, kv_blocks + blocks for q)
template <int DH, uint32_t FMT, bool TURN>
__global__ __launch_bounds__(256) void kv_append_kernel(RopeView r, KvAppend a) {
  typedef typename std::conditional<FMT == SIF_BF16, float, double>::type T;
  constexpr uint32_t CH = DH / 8, HP = 16 / CH;              // chunks of eight elements of a head; heads at once
  constexpr uint32_t ROW = FMT == SIF_BF16 ? DH * 2 + 4 : FMT == SIF_E4M3 ? DH + 4 : DH / 2 + 4;      // bytes of a row of values in LDS
  __shared__ int32_t s_page[kKvRows];
  __shared__ uint32_t s_pos[kKvRows];
  __shared__ __align__(16) unsigned char s_table[kKvRows * (DH / 2) * sizeof(CosSin<T>)];
  __shared__ __align__(16) unsigned char s_v[HP * kKvRows * ROW];
  const KvView& c = a.c;
  const uint32_t t = threadIdx.x, row0 = kv_tile(blockIdx.x, a.tiles_lg) * kKvRows;
  if (row0 >= a.l.rows) return;
  const bool of_q = blockIdx.y >= a.kv_blocks;
  if (of_q) {
    // (the first vectors are on their way while the rows are looked for)
    const uint32_t turning = r.half / 8, units = turning + a.q_copies, slots = 16 / units;
    const uint32_t unit = t % units, slot = t / units % slots, row = t / (units * slots);
    const bool turns = unit < turning;
    uint32_t x = r.interleaved ? unit * 16 : unit * 8, y = r.interleaved ? x + 8 : x + r.half;
    if (!turns) {
      x = 2 * r.half + (unit - turning) * 8;
      y = x + a.q_copies * 8 < DH ? x + a.q_copies * 8 : x;      // (of an odd number the last one twice)
    }
    const size_t at = row0 + row;
    uint32_t h = (blockIdx.y - a.kv_blocks) * slots + slot;
    const size_t safe = std::min(row0 + row, a.l.rows - 1);
    u32x4_kv nu = *reinterpret_cast<const u32x4_kv*>(a.q + safe * a.ld_q + std::min(h, a.heads - 1) * DH + x);
    u32x4_kv nw = *reinterpret_cast<const u32x4_kv*>(a.q + safe * a.ld_q + std::min(h, a.heads - 1) * DH + y);
    kv_find_rows(c, a.l, row0, false, false, s_pos);
    __syncthreads();
    CosSin<float>* cs_all = reinterpret_cast<CosSin<float>*>(s_table);
    for (uint32_t i = t; i < kKvRows * r.half; i += 256) {
      const uint32_t pos = s_pos[i / r.half];
      if (pos < kBefore) cs_all[i] = rope_cos_sin<float>(r, (double)pos, i % r.half);
    }
    __syncthreads();
    if (row >= kKvRows || s_pos[row] >= kBefore) return;
    CosSin<float> cs[8];
    if (turns) {
#pragma unroll
      for (uint32_t e = 0; e < 8; e += 2) *reinterpret_cast<float4*>(&cs[e]) = *reinterpret_cast<const float4*>(&cs_all[row * r.half + unit * 8 + e]);
    }
    while (h < a.heads) {
      const uint32_t next = h + (gridDim.y - a.kv_blocks) * slots;
      uint4 u = kv_uint4(nu), w = kv_uint4(nw);
      nu = *reinterpret_cast<const u32x4_kv*>(a.q + at * a.ld_q + std::min(next, a.heads - 1) * DH + x);
      nw = *reinterpret_cast<const u32x4_kv*>(a.q + at * a.ld_q + std::min(next, a.heads - 1) * DH + y);
      bf16_t* to = a.q_out + at * a.ld_q_out + h * DH;
      if (turns) rope_turn8(r.interleaved, cs, 1.f, u, w);
      *reinterpret_cast<uint4*>(to + x) = u;
      *reinterpret_cast<uint4*>(to + y) = w;
      h = next;
    }
    return;
  }
  const uint32_t row = t / CH % kKvRows, ch = t % CH, hp = t / (CH * kKvRows), pt = 1u << c.page_lg;
  // (of a turned chunk also the one whose elements are its partners)
  const bool turned = TURN && ch * 8 < 2 * r.half, first = ch * 8 < r.half;
  const uint32_t other = !turned || r.interleaved ? ch * 8 : first ? ch * 8 + r.half : ch * 8 - r.half;
  struct Vectors { u32x4_kv own, partner, val; };
  auto fetch = [&](uint32_t group) {
    const uint32_t head = std::min(group * HP + hp, c.kv_heads - 1);       // (a head or a row too many is the last one)
    const size_t at = std::min(row0 + row, a.l.rows - 1);
    const bf16_t* from = a.k + at * a.ld_k + head * DH;
    return Vectors{*reinterpret_cast<const u32x4_kv*>(from + ch * 8), *reinterpret_cast<const u32x4_kv*>(from + other), *reinterpret_cast<const u32x4_kv*>(a.v + at * a.ld_v + head * DH + ch * 8)};
  };
  Vectors next = fetch(blockIdx.y);                // (the first heads' vectors are on their way while the rows are looked for)
  const int32_t found = kv_find_rows(c, a.l, row0, true, true, s_pos);
  __syncthreads();
  CosSin<T>* cs_all = reinterpret_cast<CosSin<T>*>(s_table);
  if constexpr (TURN)
    for (uint32_t i = t; i < kKvRows * r.half; i += 256) {
      const uint32_t pos = s_pos[i / r.half];
      if (pos < kBefore) cs_all[i] = rope_cos_sin<T>(r, (double)pos, i % r.half);
    }
  if ((t & 15) == 0) s_page[t >> 4] = (uint32_t)found < c.n_pages ? found : -1;
  __syncthreads();
  const int32_t page = s_page[row];
  const uint32_t off = s_pos[row] & (pt - 1u);
  const size_t head_bytes = kv_head_bytes<DH, FMT>(c.page_lg), pool = ((size_t)a.layer * c.n_pages + (uint32_t)std::max(page, 0)) * c.page_bytes;
  for (uint32_t group = blockIdx.y; group * HP < c.kv_heads; group += a.kv_blocks) {
    const uint32_t head = group * HP + hp;
    const bool there = page >= 0 && head < c.kv_heads;
    const float ks = FMT == SIF_E4M3 && c.k_scale != nullptr && there ? c.k_scale[a.layer * c.kv_heads + head] : 1.f;
    const float vs = FMT == SIF_E4M3 && c.v_scale != nullptr && there ? c.v_scale[a.layer * c.kv_heads + head] : 1.f;
    const uint4 own = kv_uint4(next.own), partner = kv_uint4(next.partner), val = kv_uint4(next.val);
    next = fetch(group + a.kv_blocks);
    if (there) {
      float x[8], p[8];
      kv_unpack8(own, x);
      T y[8];
      if (turned) {
        const CosSin<T>* cs = cs_all + row * r.half;
        if (r.interleaved) {
#pragma unroll
          for (uint32_t e = 0; e < 8; e += 2) {
            const CosSin<T> f = cs[ch * 4 + e / 2];
            y[e] = fma((T)x[e], f.c, -((T)x[e + 1] * f.s));
            y[e + 1] = fma((T)x[e + 1], f.c, (T)x[e] * f.s);
          }
        } else {
          const uint32_t pair = first ? ch * 8 : other;
          kv_unpack8(partner, p);
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) {
            const CosSin<T> f = cs[pair + e];
            y[e] = fma((T)x[e], f.c, (first ? -(T)p[e] : (T)p[e]) * f.s);
          }
        }
      } else {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) y[e] = (T)x[e];
      }
      unsigned char* to = c.k + pool + head * head_bytes;
      if constexpr (FMT == SIF_BF16) {
        *reinterpret_cast<uint4*>(to + (off * DH + ch * 8) * 2) =
            turned ? make_uint4(pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3]), pack_bf2(y[4], y[5]), pack_bf2(y[6], y[7])) : own;
        uint32_t* at = reinterpret_cast<uint32_t*>(s_v + (hp * kKvRows + row) * ROW + ch * 16);
        at[0] = val.x; at[1] = val.y; at[2] = val.z; at[3] = val.w;
      } else if constexpr (FMT == SIF_E4M3) {
        // (through fp32: what lies within 2^-24 of a border counts as on it, so the reciprocal's rounding takes no quotient off a border that it is on)
        const double inv = 1.0 / (double)ks;
        float f[8], g[8];
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) f[e] = (float)(y[e] * inv);
        *reinterpret_cast<uint2*>(to + off * DH + ch * 8) =
            make_uint2(kv_e4m3x2(f[0], f[1]) | kv_e4m3x2(f[2], f[3]) << 16, kv_e4m3x2(f[4], f[5]) | kv_e4m3x2(f[6], f[7]) << 16);
        kv_unpack8(val, g);
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) g[e] = __fdiv_rn(g[e], vs);
        uint32_t* at = reinterpret_cast<uint32_t*>(s_v + (hp * kKvRows + row) * ROW + ch * 8);
        at[0] = kv_e4m3x2(g[0], g[1]) | kv_e4m3x2(g[2], g[3]) << 16;
        at[1] = kv_e4m3x2(g[4], g[5]) | kv_e4m3x2(g[6], g[7]) << 16;
      } else {
        // The largest of 32: four neighbouring lanes have them (they are all here or none is: they share the row and the head).  7 2^e is even in fp32, so it may be told from what is rounded
        // to odd; a sixteenth of the key, so that what a turn makes of the largest bf16 numbers stays one.
        float f[8], g[8];
        kv_unpack8(val, g);
        uint32_t top_k = 0, top_v = 0;
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
          f[e] = kv_round_odd((double)y[e] * 0.0625);
          top_k = std::max(top_k, __float_as_uint(f[e]) & 0x7FFFFFFFu);
          top_v = std::max(top_v, __float_as_uint(g[e]) & 0x7FFFFFFFu);
        }
        const KvPower pk = kv_power(kv_largest_of_4(top_k), 4), pv = kv_power(kv_largest_of_4(top_v), 0);
        *reinterpret_cast<uint32_t*>(to + off * (DH / 2) + ch * 4) = pk.byte == 255u ? 0u : kv_codes8(f, pk.e - 4);
        unsigned char* tv = c.v + pool + head * head_bytes;
        if (ch % 4 == 0) {
          to[((DH / 2) << c.page_lg) + ((ch / 4) << c.page_lg) + off] = (unsigned char)pk.byte;
          tv[((DH / 2) << c.page_lg) + off * (DH / 32) + ch / 4] = (unsigned char)pv.byte;
        }
        const uint32_t mine = pv.byte == 255u ? 0u : kv_codes8(g, pv.e), over = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mine, 0x4E, 0xF, 0xF, true);
        if (ch % 4 < 2) {
          uint32_t* at = reinterpret_cast<uint32_t*>(s_v + (hp * kKvRows + row) * ROW + ch / 4 * 16 + ch % 4 * 8);
          at[0] = kv_spread4(mine & 0xFFFFu) | kv_spread4(over & 0xFFFFu) << 4;
          at[1] = kv_spread4(mine >> 16) | kv_spread4(over >> 16) << 4;
        }
      }
    }
    __syncthreads();
    const uint32_t vr = t & 15;
    const int32_t vpage = s_page[vr];
    if (vpage >= 0) {
      const uint32_t voff = s_pos[vr] & (pt - 1u);
      constexpr uint32_t LINES = FMT == SIF_E2M1 ? DH / 2 : DH;             // rows of tokens of a page's head
      unsigned char* to = c.v + ((size_t)a.layer * c.n_pages + (uint32_t)vpage) * c.page_bytes;
#pragma unroll
      for (uint32_t j = 0; j < LINES * HP / 16; ++j) {
        const uint32_t line = (j * 16 + (t >> 4)) % LINES, vh = (j * 16 + (t >> 4)) / LINES;
        if (group * HP + vh >= c.kv_heads) continue;
        const unsigned char* from = s_v + (vh * kKvRows + vr) * ROW;
        unsigned char* at = to + (group * HP + vh) * head_bytes;
        if constexpr (FMT == SIF_BF16) reinterpret_cast<bf16_t*>(at)[(line << c.page_lg) + voff] = reinterpret_cast<const bf16_t*>(from)[line];
        else at[(line << c.page_lg) + voff] = from[line];
      }
    }
    __syncthreads();                               // nobody reads these heads' values any more
  }
}

struct KvRead {
  KvView c;
  KvRowList l;
  bf16_t* k;
  bf16_t* v;
  uint32_t layer, ld_k, ld_v, tiles_lg;
};

// two of e2m1, the lowest byte, times a power of two that may be NaN, as bf16
__device__ __forceinline__ uint32_t kv_e2m1x2(uint32_t byte, float power) {
  const uint32_t w = e2m1x2<0>(byte, 1.0f);
  return pack_bf2(bflo(w) * power, bfhi(w) * power);
}
typedef float floatx2_kv __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t kv_from_e4m3_lo(uint32_t w, float scale) {
  const floatx2_kv f = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
  return pack_bf2(f[0] * scale, f[1] * scale);
}
__device__ __forceinline__ uint32_t kv_from_e4m3_hi(uint32_t w, float scale) {
  const floatx2_kv f = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  return pack_bf2(f[0] * scale, f[1] * scale);
}

// grid: (sixteen rows, groups of heads).  Four heads at a time: what a block takes is not bytes but loads that wait for one another.
template <int DH, uint32_t FMT>
__global__ __launch_bounds__(256) void kv_read_kernel(KvRead a) {
  constexpr uint32_t CH = DH / 8, HP = 16 / CH, TURNS = 4 / HP;
  constexpr uint32_t ROW = FMT == SIF_BF16 ? DH * 2 + 4 : FMT == SIF_E4M3 ? DH + 4 : DH / 2 + 4;
  constexpr uint32_t LINES = FMT == SIF_E2M1 ? DH / 2 : DH, PER = LINES * HP / 16;      // rows of tokens of a page's head; of them a thread's
  typedef typename std::conditional<FMT == SIF_BF16, uint16_t, uint8_t>::type Held;
  __shared__ int32_t s_page[kKvRows];
  __shared__ uint32_t s_pos[kKvRows];
  __shared__ __align__(16) unsigned char s_v[TURNS * HP * kKvRows * ROW];
  const KvView& c = a.c;
  const uint32_t t = threadIdx.x, row0 = kv_tile(blockIdx.x, a.tiles_lg) * kKvRows;
  if (row0 >= a.l.rows) return;
  const int32_t found = kv_find_rows(c, a.l, row0, true, false, s_pos);
  if ((t & 15) == 0) s_page[t >> 4] = (uint32_t)found < c.n_pages ? found : -1;
  __syncthreads();
  const uint32_t row = t / CH % kKvRows, ch = t % CH, hp = t / (CH * kKvRows), pt = 1u << c.page_lg;
  const int32_t page = s_page[row];
  const uint32_t off = s_pos[row] & (pt - 1u);
  const bool wanted = s_pos[row] != kNoRow;
  const size_t head_bytes = kv_head_bytes<DH, FMT>(c.page_lg), layer = (size_t)a.layer * c.n_pages;
  const uint32_t vr = t & 15;                      // the row whose values this thread fetches
  const int32_t vpage = s_page[vr];
  const uint32_t voff = s_pos[vr] & (pt - 1u);
  const size_t pool = (layer + (uint32_t)std::max(page, 0)) * c.page_bytes, vpool = (layer + (uint32_t)std::max(vpage, 0)) * c.page_bytes;
  for (uint32_t group = blockIdx.y * TURNS; group * HP < c.kv_heads; group += gridDim.y * TURNS) {
    Held held[TURNS][PER];
    uint4 k[TURNS];
    uint32_t pk[TURNS], pv[TURNS];
#pragma unroll
    for (uint32_t u = 0; u < TURNS; ++u) {
#pragma unroll
      for (uint32_t j = 0; j < PER; ++j) {
        const uint32_t line = (j * 16 + (t >> 4)) % LINES, vh = (group + u) * HP + (j * 16 + (t >> 4)) / LINES;
        held[u][j] = 0;
        if (vpage >= 0 && vh < c.kv_heads) held[u][j] = reinterpret_cast<const Held*>(c.v + vpool + vh * head_bytes)[(line << c.page_lg) + voff];
      }
      const uint32_t head = (group + u) * HP + hp;
      k[u] = make_uint4(0, 0, 0, 0);
      pk[u] = pv[u] = 0;
      if (page >= 0 && head < c.kv_heads) {
        const unsigned char* from = c.k + pool + head * head_bytes;
        if constexpr (FMT == SIF_BF16) {
          k[u] = *reinterpret_cast<const uint4*>(from + (off * DH + ch * 8) * 2);
        } else if constexpr (FMT == SIF_E4M3) {
          const uint2 w = *reinterpret_cast<const uint2*>(from + off * DH + ch * 8);
          k[u].x = w.x;
          k[u].y = w.y;
        } else {
          k[u].x = *reinterpret_cast<const uint32_t*>(from + off * (DH / 2) + ch * 4);
          pk[u] = from[((DH / 2) << c.page_lg) + ((ch / 4) << c.page_lg) + off];
          pv[u] = c.v[pool + head * head_bytes + ((DH / 2) << c.page_lg) + off * (DH / 32) + ch / 4];
        }
      }
    }
#pragma unroll
    for (uint32_t u = 0; u < TURNS; ++u)
#pragma unroll
      for (uint32_t j = 0; j < PER; ++j) {
        const uint32_t line = (j * 16 + (t >> 4)) % LINES, vh = u * HP + (j * 16 + (t >> 4)) / LINES;
        reinterpret_cast<Held*>(s_v + (vh * kKvRows + vr) * ROW)[line] = held[u][j];
      }
    __syncthreads();
#pragma unroll
    for (uint32_t u = 0; u < TURNS; ++u) {
      const uint32_t head = (group + u) * HP + hp;
      if (!wanted || head >= c.kv_heads) continue;
      const uint32_t* sv = reinterpret_cast<const uint32_t*>(s_v + ((u * HP + hp) * kKvRows + row) * ROW);
      uint4 x = make_uint4(0, 0, 0, 0), y = x;
      if (page >= 0) {
        if constexpr (FMT == SIF_BF16) {
          x = k[u];
          y = make_uint4(sv[ch * 4], sv[ch * 4 + 1], sv[ch * 4 + 2], sv[ch * 4 + 3]);
        } else if constexpr (FMT == SIF_E4M3) {
          const float ks = c.k_scale != nullptr ? c.k_scale[a.layer * c.kv_heads + head] : 1.f, vs = c.v_scale != nullptr ? c.v_scale[a.layer * c.kv_heads + head] : 1.f;
          x = make_uint4(kv_from_e4m3_lo(k[u].x, ks), kv_from_e4m3_hi(k[u].x, ks), kv_from_e4m3_lo(k[u].y, ks), kv_from_e4m3_hi(k[u].y, ks));
          const uint32_t p = sv[ch * 2], q = sv[ch * 2 + 1];
          y = make_uint4(kv_from_e4m3_lo(p, vs), kv_from_e4m3_hi(p, vs), kv_from_e4m3_lo(q, vs), kv_from_e4m3_hi(q, vs));
        } else {
          const float kp = e2m1_power(pk[u]), vp = e2m1_power(pv[u]);
          const uint32_t w = k[u].x;
          x = make_uint4(kv_e2m1x2(w & 255u, kp), kv_e2m1x2(w >> 8 & 255u, kp), kv_e2m1x2(w >> 16 & 255u, kp), kv_e2m1x2(w >> 24, kp));
          // eight bytes, of each the half that belongs to this chunk; two of these to a byte
          uint32_t p = sv[ch / 4 * 4 + ch % 2 * 2], q = sv[ch / 4 * 4 + ch % 2 * 2 + 1];
          p = (ch % 4 < 2 ? p : p >> 4) & 0x0F0F0F0Fu;
          q = (ch % 4 < 2 ? q : q >> 4) & 0x0F0F0F0Fu;
          p |= p >> 4;
          q |= q >> 4;
          y = make_uint4(kv_e2m1x2(p & 255u, vp), kv_e2m1x2(p >> 16 & 255u, vp), kv_e2m1x2(q & 255u, vp), kv_e2m1x2(q >> 16 & 255u, vp));
        }
      }
      *reinterpret_cast<uint4*>(a.k + (size_t)(row0 + row) * a.ld_k + head * DH + ch * 8) = x;
      *reinterpret_cast<uint4*>(a.v + (size_t)(row0 + row) * a.ld_v + head * DH + ch * 8) = y;
    }
    __syncthreads();                               // nobody reads these heads' values any more
  }
}

// Blocks along y that share a tile's groups of heads: enough for some blocks per CU.
static uint32_t kv_share(uint32_t tiles, uint32_t groups) { return std::max(1u, std::min(groups, (1024 + tiles - 1) / tiles)); }

template <bool TURN>
static sif_status launch_append(const char* who, uint32_t dtype, uint32_t d_head, const RopeView& r, KvAppend a, hipStream_t s) {
  const uint32_t tiles = (a.l.rows + kKvRows - 1) / kKvRows, at_once = 128 / d_head, groups = (a.c.kv_heads + at_once - 1) / at_once;
  a.kv_blocks = kv_share(tiles, groups);
  uint32_t q_blocks = 0;
  if (a.heads != 0) {
    const uint32_t slots = 16 / (r.half / 8 + a.q_copies);
    // (Of four turns and more up to 4096 in all: 16384 rows, 32 query heads and 8 key heads of 64 in bf16 49.5 -> 46 us, of 128 83 -> 79; with blocks of two turns 8 query heads of 64 took 20.4 us for 18.4.)
    const uint32_t groups_q = (a.heads + slots - 1) / slots;
    q_blocks = std::max(kv_share(tiles, groups_q), std::min(groups_q / 4, (4096 + tiles - 1) / tiles));
  }
  a.tiles_lg = kv_tiles_lg(a.c, a.l);
  const dim3 grid(kv_grid_x(tiles, a.tiles_lg), a.kv_blocks + q_blocks);
#define KV_APPEND(DH, F) hipLaunchKernelGGL((kv_append_kernel<DH, F, TURN>), grid, dim3(256), 0, s, r, a)
  if constexpr (TURN) {
    if (d_head == 64) { if (dtype == SIF_BF16) KV_APPEND(64, SIF_BF16); else if (dtype == SIF_E4M3) KV_APPEND(64, SIF_E4M3); else KV_APPEND(64, SIF_E2M1); }
    else { if (dtype == SIF_BF16) KV_APPEND(128, SIF_BF16); else if (dtype == SIF_E4M3) KV_APPEND(128, SIF_E4M3); else KV_APPEND(128, SIF_E2M1); }
  } else {
    if (d_head == 64) KV_APPEND(64, SIF_E2M1); else KV_APPEND(128, SIF_E2M1);
  }
#undef KV_APPEND
  return check_launch(who);
}

sif_status kv_write_4bit(const KvView& c, uint32_t d_head, uint32_t layer, const void* k, const void* v, uint32_t ld_k, uint32_t ld_v, const KvRowList& l, hipStream_t s) {
  RopeView r = {};
  r.half = 8;                                       // (not looked at)
  KvAppend a = {};
  a.c = c;
  a.l = l;
  a.k = (const bf16_t*)k;
  a.v = (const bf16_t*)v;
  a.layer = layer;
  a.ld_k = ld_k;
  a.ld_v = ld_v;
  return launch_append<false>("kv_write", SIF_E2M1, d_head, r, a, s);
}

static sif_status check_rows(const char* who, const KvView& c, uint32_t layer, const void* k, const void* v, uint32_t ld_k, uint32_t ld_v, const KvRowList& l, bool once) {
  if (layer >= c.layers) return fail(SIF_E_INVAL, "%s: no layer %u", who, layer);
  if (!k || !v || (((uintptr_t)k | (uintptr_t)v) & 15)) return fail(SIF_E_INVAL, "%s: k and v must be 16-byte aligned", who);
  if (l.n == 0 || l.rows == 0 || l.n > (1u << 27) || l.rows > (1u << 27)) return fail(SIF_E_INVAL, "%s: entries or rows outside 1 .. 2^27", who);
  if (once && l.seqs != nullptr && l.n > kKvMaxWritten) return fail(SIF_E_INVAL, "%s: at most %u listed sequences", who, kKvMaxWritten);      // see sif_k_kv_write
  if (((uintptr_t)l.seqs | (uintptr_t)l.starts) & 3) return fail(SIF_E_INVAL, "%s: misaligned list", who);
  if (l.starts == nullptr && l.rows != l.n) return fail(SIF_E_INVAL, "%s: without starts there is one row per entry", who);
  const uint32_t width = c.kv_heads * c.d_head;
  if (ld_k < width || ld_v < width || ((ld_k | ld_v) & 7)) return fail(SIF_E_INVAL, "%s: bad leading dimensions", who);
  return SIF_OK;
}

}  // namespace sif

using namespace sif;
static inline hipStream_t S(void* s) { return reinterpret_cast<hipStream_t>(s); }

extern "C" {

sif_status sif_k_kv_append(const sif_kv_cache* c, const sif_rope* rope, const sif_kv_append_args* x, void* stream) {
  KvAppend a = {};
  if (sif_status st = kv_check("kv_append", c, &a.c)) return st;
  if (!x) return fail(SIF_E_INVAL, "kv_append: null arguments");
  if (x->struct_size != sizeof(sif_kv_append_args)) return fail(SIF_E_INVAL, "kv_append: struct_size");
  RopeView r;
  if (sif_status st = rope_check("kv_append", rope, c->d_head, &r)) return st;
  a.l = KvRowList{x->seqs_dev, x->starts_dev, x->n, x->rows};
  if (sif_status st = check_rows("kv_append", a.c, x->layer, x->k_dev, x->v_dev, x->ld_k, x->ld_v, a.l, true)) return st;
  if (x->heads > 1024) return fail(SIF_E_INVAL, "kv_append: at most 1024 heads");
  if (x->heads != 0) {
    const uint32_t width = x->heads * c->d_head;
    if (!x->q_dev || !x->q_out_dev || (((uintptr_t)x->q_dev | (uintptr_t)x->q_out_dev) & 15)) return fail(SIF_E_INVAL, "kv_append: q and q_out must be 16-byte aligned");
    if (x->ld_q < width || x->ld_q_out < width || ((x->ld_q | x->ld_q_out) & 7)) return fail(SIF_E_INVAL, "kv_append: bad leading dimensions");
    if (x->q_dev == x->q_out_dev && x->ld_q != x->ld_q_out) return fail(SIF_E_INVAL, "kv_append: in place, with one leading dimension");
  }
  a.k = (const bf16_t*)x->k_dev;
  a.v = (const bf16_t*)x->v_dev;
  a.q = (const bf16_t*)x->q_dev;
  a.q_out = (bf16_t*)x->q_out_dev;
  a.layer = x->layer;
  a.heads = x->heads;
  a.ld_q = x->ld_q;
  a.ld_q_out = x->ld_q_out;
  a.ld_k = x->ld_k;
  a.ld_v = x->ld_v;
  a.q_copies = x->q_dev == x->q_out_dev ? 0 : ((c->d_head - 2 * r.half) / 8 + 1) / 2;
  return launch_append<true>("kv_append", c->dtype, c->d_head, r, a, S(stream));
}

sif_status sif_k_kv_read(const sif_kv_cache* c, uint32_t layer, void* k, void* v, uint32_t ld_k, uint32_t ld_v, const int32_t* seqs, const int32_t* starts,
                         uint32_t n, uint32_t rows, void* stream) {
  KvRead a = {};
  if (sif_status st = kv_check("kv_read", c, &a.c)) return st;
  a.l = KvRowList{seqs, starts, n, rows};
  if (sif_status st = check_rows("kv_read", a.c, layer, k, v, ld_k, ld_v, a.l, false)) return st;
  a.k = (bf16_t*)k;
  a.v = (bf16_t*)v;
  a.layer = layer;
  a.ld_k = ld_k;
  a.ld_v = ld_v;
  const uint32_t tiles = (rows + kKvRows - 1) / kKvRows;
  a.tiles_lg = kv_tiles_lg(a.c, a.l);
  const dim3 grid(kv_grid_x(tiles, a.tiles_lg), kv_share(tiles, (a.c.kv_heads + 3) / 4));
#define KV_READ(DH, F) hipLaunchKernelGGL((kv_read_kernel<DH, F>), grid, dim3(256), 0, S(stream), a)
  if (c->d_head == 64) { if (c->dtype == SIF_BF16) KV_READ(64, SIF_BF16); else if (c->dtype == SIF_E4M3) KV_READ(64, SIF_E4M3); else KV_READ(64, SIF_E2M1); }
  else { if (c->dtype == SIF_BF16) KV_READ(128, SIF_BF16); else if (c->dtype == SIF_E4M3) KV_READ(128, SIF_E4M3); else KV_READ(128, SIF_E2M1); }
#undef KV_READ
  return check_launch("kv_read");
}

}  // extern "C"
