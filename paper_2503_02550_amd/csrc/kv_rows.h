// Which token a row of new or read-back keys and values is, for the kernels that take rows by the list of a paged cache's sequences.
#pragma once
#include <algorithm>

#include "common.h"
#include "kv_cache.h"

namespace sif {

constexpr uint32_t kKvRows = 16;         // rows of a block, sixteen threads each

// Rows row0 .. row0 + 15 of lists as in sif_k_kv_write, sixteen threads to a row: s_pos gets the row's place in its sequence (kNoRow: the row is no sequence's; kBefore: it lies
// in front of the sequence's first token).  Returns, in the first of the sixteen, the number of its page as the table has it, or -1; that load is still on its way.  With
// `once` a sequence that stands in the list before has no page either.  The lists are read sixteen entries at a time: what counts is how many loads wait for one another.
constexpr uint32_t kNoRow = 0xFFFFFFFFu, kBefore = 0xFFFFFFFEu;
struct KvRowList { const int32_t* seqs; const int32_t* starts; uint32_t n, rows; };
__device__ __forceinline__ int32_t kv_find_rows(const KvView& c, const KvRowList& l, uint32_t row0, bool pages, bool once, uint32_t* s_pos) {
  const uint32_t t = threadIdx.x, r = t >> 4, part = t & 15, row = row0 + r, shift = t & 48;
  uint32_t i = row, pos = kNoRow;
  int32_t s = -1;
  if (row < l.rows) {
    uint32_t from = row, to = row + 1;
    if (l.starts != nullptr) {
      uint32_t lo = 0, size = l.n;               // the first entry that begins behind the row is one of lo .. lo + size
      while (size > 0) {
        const uint32_t step = (size + 15) / 16, at = (part + 1) * step - 1;
        const bool upto = at < size && l.starts[lo + at] <= (int32_t)row;
        const uint32_t c16 = __popc((uint32_t)(__ballot(upto) >> shift) & 0xFFFFu), skip = c16 * step;
        lo += skip;
        size = size > skip ? std::min(step - 1, size - skip) : 0u;
      }
      i = lo - 1;
      from = lo > 0 ? (uint32_t)l.starts[i] : 0u;
      to = lo > 0 ? (uint32_t)l.starts[i + 1] : 0u;
    }
    if (i < l.n && from <= row && row < to) {
      s = kv_listed(c, l.seqs, i);
      if (s >= 0) {
        const uint32_t len = kv_length(c, s), back = to - row;
        pos = back <= len ? len - back : kBefore;
      }
    }
  }
  bool again = false;
  if (once && s >= 0 && l.seqs != nullptr) {
#pragma unroll 8
    for (uint32_t j = part; j < i; j += 16) again |= l.seqs[j] == s;
  }
  const uint32_t votes = (uint32_t)(__ballot(again) >> shift) & 0xFFFFu;
  int32_t p = -1;
  if (part == 0) {
    if (pages && pos < kBefore && votes == 0) p = c.table[(size_t)s * c.table_ld + (pos >> c.page_lg)];
    s_pos[r] = pos;
  }
  return p;
}

// float -> e4m3, held at +-448, NaN kept; two at a time into the low half of a word
__device__ __forceinline__ uint32_t kv_e4m3x2(float a, float b) {
  a = a != a ? a : fminf(fmaxf(a, -448.f), 448.f);
  b = b != b ? b : fminf(fmaxf(b, -448.f), 448.f);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}

// What sif_k_kv_write does for a cache in 4 bits (kv_rows.hip); arguments as checked there.
sif_status kv_write_4bit(const KvView& c, uint32_t d_head, uint32_t layer, const void* k, const void* v, uint32_t ld_k, uint32_t ld_v, const KvRowList& l, hipStream_t s);

}  // namespace sif
