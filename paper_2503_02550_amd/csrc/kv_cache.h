// A paged key-value cache as the kernels see it (sif_kv_cache, checked), and the rules that its operations and the attention over it
// share.  These launches are unmonitored: they belong to no registered model.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "launch.h"

namespace sif {

struct KvView {
  unsigned char* k;
  unsigned char* v;
  const float* k_scale;
  const float* v_scale;
  int32_t* table;
  int32_t* lengths;
  int32_t* refs;
  uint32_t layers, kv_heads, d_head, page_lg, n_pages, n_seqs, table_ld;
  uint32_t page_bytes;               // of K or V in one layer
};

constexpr uint32_t kKvMaxListed = 1024, kKvMaxWritten = 1u << 14, kKvMaxPages = 1u << 21;      // entries of a list (kKvMaxWritten: of tokens that are written)

// Checks a cache and fills in the view; `who` begins the error's text.
sif_status kv_check(const char* who, const sif_kv_cache* c, KvView* out);

// The i-th listed sequence, or -1 where the list names none of the table's.
__device__ __forceinline__ int32_t kv_listed(const KvView& c, const int32_t* seqs, uint32_t i) {
  const int32_t s = seqs != nullptr ? seqs[i] : (int32_t)i;
  return (uint32_t)s < c.n_seqs ? s : -1;
}
// Tokens of a sequence; a length that its row of the table cannot hold is cut there.
__device__ __forceinline__ uint32_t kv_length(const KvView& c, int32_t s) {
  const int32_t n = c.lengths[s];
  const uint32_t most = c.table_ld << c.page_lg;       // fits: kv_check
  return n <= 0 ? 0u : ((uint32_t)n < most ? (uint32_t)n : most);
}
__device__ __forceinline__ uint32_t kv_pages_of(const KvView& c, uint32_t tokens) { return (tokens + (1u << c.page_lg) - 1u) >> c.page_lg; }

}  // namespace sif
