// Page operations of a paged key-value cache: queued on a stream like every other kernel, they ask the host nothing.  Bookkeeping is integers: what it costs is launches and dependent loads, so each operation is one
// launch for the bookkeeping and, where contents move, one that moves them at the memory's rate.  Results do not depend on the
// order of blocks: reference counts are sums, and who gets which page follows from a rank in the list of free pages.
#include "common.h"
#include "kv_cache.h"

namespace sif {

sif_status kv_check(const char* who, const sif_kv_cache* c, KvView* out) {
  if (!c) return fail(SIF_E_INVAL, "%s: null cache", who);
  if (c->struct_size != sizeof(sif_kv_cache)) return fail(SIF_E_INVAL, "%s: struct_size of the cache", who);
  if (c->dtype != SIF_BF16 && c->dtype != SIF_E4M3) return fail(SIF_E_INVAL, "%s: dtype must be SIF_BF16 or SIF_E4M3", who);
  if (!c->layers || !c->kv_heads || !c->n_pages || !c->n_seqs || !c->table_ld) return fail(SIF_E_INVAL, "%s: empty extent", who);
  if (c->d_head != 64 && c->d_head != 128) return fail(SIF_E_INVAL, "%s: d_head must be 64 or 128", who);
  const uint32_t pt = c->page_tokens;
  if (pt < 16 || pt > 256 || (pt & (pt - 1))) return fail(SIF_E_INVAL, "%s: page_tokens must be 16, 32, 64, 128 or 256", who);
  if (!c->k_dev || !c->v_dev || !c->table_dev || !c->lengths_dev || !c->refs_dev) return fail(SIF_E_INVAL, "%s: null operand", who);
  if (((uintptr_t)c->k_dev | (uintptr_t)c->v_dev | (uintptr_t)c->refs_dev) & 15) return fail(SIF_E_INVAL, "%s: k, v and refs must be 16-byte aligned", who);
  if (((uintptr_t)c->table_dev | (uintptr_t)c->lengths_dev | (uintptr_t)c->k_scale_dev | (uintptr_t)c->v_scale_dev) & 3)
    return fail(SIF_E_INVAL, "%s: misaligned operand", who);
  if (c->dtype == SIF_BF16 && (c->k_scale_dev || c->v_scale_dev)) return fail(SIF_E_INVAL, "%s: scales belong to SIF_E4M3", who);
  if (c->layers > 1024 || c->kv_heads > 1024) return fail(SIF_E_INVAL, "%s: at most 1024 layers and 1024 kv_heads", who);
  if ((uint64_t)c->table_ld * pt > 0x7FFFFF00ull || c->n_seqs > 0x7FFFFF00u)
    return fail(SIF_E_INVAL, "%s: tokens of a row or sequences beyond 31 bits", who);
  if (c->n_pages > kKvMaxPages) return fail(SIF_E_INVAL, "%s: at most %u pages", who, kKvMaxPages);
  KvView v;
  v.k = (unsigned char*)c->k_dev;
  v.v = (unsigned char*)c->v_dev;
  v.k_scale = c->k_scale_dev;
  v.v_scale = c->v_scale_dev;
  v.table = c->table_dev;
  v.lengths = c->lengths_dev;
  v.refs = c->refs_dev;
  v.layers = c->layers;
  v.kv_heads = c->kv_heads;
  v.d_head = c->d_head;
  v.page_lg = (uint32_t)__builtin_ctz(pt);
  v.n_pages = c->n_pages;
  v.n_seqs = c->n_seqs;
  v.table_ld = c->table_ld;
  v.page_bytes = c->kv_heads * pt * c->d_head * (c->dtype == SIF_BF16 ? 2u : 1u);      // at most 64 MB
  *out = v;
  return SIF_OK;
}

static sif_status kv_check_list(const char* who, uint32_t n, const int32_t* x, const int32_t* y = nullptr, const int32_t* status = nullptr) {
  if (n == 0 || n > kKvMaxListed) return fail(SIF_E_INVAL, "%s: 1 to %u entries", who, kKvMaxListed);
  if (((uintptr_t)x | (uintptr_t)y | (uintptr_t)status) & 3) return fail(SIF_E_INVAL, "%s: misaligned list", who);
  return SIF_OK;
}

// Workspace of the operations that move contents: pairs (from, to), their number, and three lists of page numbers.
struct KvWork {
  uint32_t* count;                   // pairs to move (compact)
  int2* pairs;                       // [kKvMaxListed] (extend)
  int32_t* low;                      // [n_pages] free pages in ascending order
  int32_t* high;                     // [n_pages] used pages to be moved, in ascending order
  int32_t* map;                      // [n_pages] where a page goes
};
static uint64_t kv_work_bytes(const KvView& c) { return 256 + sizeof(int2) * kKvMaxListed + 3ull * sizeof(int32_t) * c.n_pages; }
static KvWork kv_work(const KvView& c, void* p) {
  unsigned char* b = (unsigned char*)p;
  KvWork w;
  w.count = (uint32_t*)b;
  w.pairs = (int2*)(b + 256);
  w.low = (int32_t*)(b + 256 + sizeof(int2) * kKvMaxListed);
  w.high = w.low + c.n_pages;
  w.map = w.high + c.n_pages;
  return w;
}
static sif_status kv_check_work(const char* who, const KvView& c, const void* p, uint64_t bytes) {
  if (!p || ((uintptr_t)p & 255)) return fail(SIF_E_INVAL, "%s: the workspace must be 256-byte aligned", who);
  if (bytes < kv_work_bytes(c)) return fail(SIF_E_NOMEM, "%s: the workspace holds %llu of %llu bytes", who, (unsigned long long)bytes, (unsigned long long)kv_work_bytes(c));
  return SIF_OK;
}

__global__ __launch_bounds__(256) void kv_reset_kernel(KvView c) {
  const uint64_t at = blockIdx.x * 256ull + threadIdx.x, step = gridDim.x * 256ull, entries = (uint64_t)c.n_seqs * c.table_ld;
  for (uint64_t i = at; i < entries; i += step) c.table[i] = -1;
  for (uint64_t i = at; i < c.n_seqs; i += step) c.lengths[i] = 0;
  for (uint64_t i = at; i < c.n_pages; i += step) c.refs[i] = 0;
}

// Whether one of the first `before` entries of a list is `x`; all threads of the block take part.
__device__ __forceinline__ bool kv_in_list(const int32_t* list, uint32_t before, int32_t x) {
  bool found = false;
  for (uint32_t j = threadIdx.x; j < before; j += blockDim.x) found |= list[j] == x;
  return __syncthreads_or(found) != 0;
}

// Free (window = 0) and trim: a block per entry.  Pages leave a sequence's row; their counts go down.
__global__ __launch_bounds__(256) void kv_release_kernel(KvView c, const int32_t* __restrict__ seqs, uint32_t window, uint32_t sinks) {
  const int32_t s = kv_listed(c, seqs, blockIdx.x);
  if (s < 0) return;
  if (seqs != nullptr && kv_in_list(seqs, blockIdx.x, s)) return;
  const uint32_t len = kv_length(c, s);
  uint32_t first = 0, last = kv_pages_of(c, len);
  if (window != 0) {
    first = sinks < len ? kv_pages_of(c, sinks) : last;
    last = len > window ? (len - window) >> c.page_lg : 0u;
  }
  int32_t* row = c.table + (size_t)s * c.table_ld;
  for (uint32_t i = first + threadIdx.x; i < last; i += 256) {
    const int32_t p = row[i];
    if ((uint32_t)p < c.n_pages) atomicSub(c.refs + p, 1);
    row[i] = -1;
  }
  if (window == 0) {
    __syncthreads();                             // every thread has read the length
    if (threadIdx.x == 0) c.lengths[s] = 0;
  }
}

__global__ __launch_bounds__(256) void kv_fork_kernel(KvView c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, uint32_t n,
                                                      int32_t* __restrict__ status) {
  const uint32_t i = blockIdx.x;
  const int32_t a = src[i], b = dst[i];
  bool bad = (uint32_t)a >= c.n_seqs || (uint32_t)b >= c.n_seqs;
  bad = kv_in_list(dst, i, b) || bad;
  bad = kv_in_list(dst, n, a) || bad;            // a source that changes in this call
  if (!bad) bad = c.lengths[b] != 0;             // only the first entry that names b gets here and writes it, below
  __syncthreads();
  if (threadIdx.x == 0 && status != nullptr) status[i] = bad ? SIF_E_INVAL : SIF_OK;
  if (bad) return;
  const uint32_t len = kv_length(c, a), pages = kv_pages_of(c, len);
  const int32_t* from = c.table + (size_t)a * c.table_ld;
  int32_t* to = c.table + (size_t)b * c.table_ld;
  for (uint32_t j = threadIdx.x; j < pages; j += 256) {
    const int32_t p = from[j];
    to[j] = p;
    if ((uint32_t)p < c.n_pages) atomicAdd(c.refs + p, 1);
  }
  if (threadIdx.x == 0) c.lengths[b] = (int32_t)len;
}

// Inclusive sum over a block of 1024 threads; `sm` holds 17 words, total = the block's sum.
__device__ __forceinline__ uint32_t kv_block_scan(uint32_t v, uint32_t* sm, uint32_t* total) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t t = __shfl_up(v, o, 64);
    if (lane >= (uint32_t)o) v += t;
  }
  __syncthreads();                               // nobody reads the last call's sums any more
  if (lane == 63) sm[wave] = v;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (uint32_t w = 0; w < 16; ++w) {
    const uint32_t t = sm[w];
    before += w < wave ? t : 0u;
    all += t;
  }
  *total = all;
  return v + before;
}

// Sixteen consecutive reference counts from page p on (p a multiple of 16): bit e says whether page p + e is used.  Pages past the end
// are neither used nor free; *here says which are there.
__device__ __forceinline__ uint32_t kv_used16(const KvView& c, uint32_t p, uint32_t* here) {
  uint32_t used = 0;
  if (p + 16 <= c.n_pages) {
    int4 r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = *reinterpret_cast<const int4*>(c.refs + p + 4 * j);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      used |= ((r[j].x > 0 ? 1u : 0u) | (r[j].y > 0 ? 2u : 0u) | (r[j].z > 0 ? 4u : 0u) | (r[j].w > 0 ? 8u : 0u)) << (4 * j);
    *here = 0xFFFFu;
    return used;
  }
  const uint32_t m = p < c.n_pages ? c.n_pages - p : 0u;
  for (uint32_t e = 0; e < m; ++e) used |= c.refs[p + e] > 0 ? 1u << e : 0u;
  *here = (1u << m) - 1u;
  return used;
}

// Extend: one block, a thread per entry for the demand, then all threads look for free pages from the lowest number on, 16384 at a time,
// only as many as are asked for.  A page's rank among the free ones decides which entry it goes to (a search in the running sums
// of the demands).
__global__ __launch_bounds__(1024) void kv_extend_kernel(KvView c, const int32_t* __restrict__ seqs, const int32_t* __restrict__ counts, uint32_t n,
                                                         int32_t* __restrict__ status, KvWork w) {
  __shared__ uint32_t sm[17];
  __shared__ int32_t s_seq[kKvMaxListed];
  __shared__ uint32_t s_end[kKvMaxListed];       // inclusive running sum of the demands
  __shared__ uint32_t s_begin[kKvMaxListed];     // first entry of the row that gets a new page
  const uint32_t i = threadIdx.x;
  const int32_t s = i < n ? kv_listed(c, seqs, i) : -1;
  s_seq[i] = s;
  __syncthreads();
  bool bad = s < 0;
  if (seqs != nullptr && !bad)
    for (uint32_t j = 0; j < i; ++j) bad |= s_seq[j] == s;
  uint32_t need = 0, begin = 0, len = 0;
  int32_t count = 0, copied = -1;
  if (!bad) {
    count = counts != nullptr ? counts[i] : 1;
    len = kv_length(c, s);
    bad = count < 0 || (uint64_t)len + (uint32_t)count > (uint64_t)c.table_ld << c.page_lg;
    if (!bad && count > 0) {
      begin = kv_pages_of(c, len);
      need = kv_pages_of(c, len + (uint32_t)count) - begin;
      if (len & ((1u << c.page_lg) - 1u)) {
        const int32_t p = c.table[(size_t)s * c.table_ld + begin - 1];
        if ((uint32_t)p >= c.n_pages) {
          bad = true;
          need = 0;
        } else if (c.refs[p] > 1) {
          copied = p;
          ++need;
          --begin;
        }
      }
    }
  }
  uint32_t wanted;
  need = need <= c.n_pages ? need : c.n_pages + 1;       // (more than there are is as good as any number above: sums stay within 32 bits)
  const uint32_t end = kv_block_scan(need, sm, &wanted);
  s_end[i] = end;
  s_begin[i] = begin;
  // the lowest free pages, as many as wanted if there are that many
  uint32_t found = 0;
  for (uint32_t base = 0; base < c.n_pages && found < wanted; base += 1024 * 16) {
    const uint32_t p = base + i * 16;
    uint32_t here, used = p < c.n_pages ? kv_used16(c, p, &here) : (here = 0u);
    uint32_t open = here & ~used, more;
    uint32_t rank = found + kv_block_scan(__popc(open), sm, &more) - __popc(open);
    while (open != 0 && rank < wanted) {
      w.low[rank++] = (int32_t)(p + __ffs(open) - 1);
      open &= open - 1;
    }
    found += more;
  }
  if (found > wanted) found = wanted;
  __syncthreads();                               // the list is written, and every count has been read
  const bool fits = !bad && (need == 0 || end <= found);
  if (i < n) {
    int2 pair = make_int2(-1, -1);
    if (fits && count > 0) {
      c.lengths[s] = (int32_t)(len + (uint32_t)count);
      if (copied >= 0) {
        pair = make_int2(copied, w.low[end - need]);
        atomicSub(c.refs + copied, 1);
      }
    }
    w.pairs[i] = pair;
    if (status != nullptr) status[i] = bad ? SIF_E_INVAL : (fits ? SIF_OK : SIF_E_NOMEM);
  }
  for (uint32_t r = i; r < found; r += 1024) {
    uint32_t lo = 0, hi = n;                     // the first entry whose running sum is above r
    while (lo < hi) {
      const uint32_t mid = (lo + hi) >> 1;
      if (s_end[mid] > r) hi = mid; else lo = mid + 1;
    }
    if (lo >= n || s_end[lo] > found) continue;  // (an entry that does not fit gets none of its pages)
    const uint32_t before = lo > 0 ? s_end[lo - 1] : 0u;
    const int32_t p = w.low[r];
    c.table[(size_t)s_seq[lo] * c.table_ld + s_begin[lo] + (r - before)] = p;
    c.refs[p] = 1;
  }
}

// One page's K or V of one layer, by one block: 16-byte vectors, eight per thread in flight.  STREAM: past the caches, for contents that
// nobody is about to read (compaction of 1.1 GB 229 -> 220 us; copies of pages that are being written to would lose by it, 29 -> 38).
template <bool STREAM>
__device__ __forceinline__ void kv_copy_page(const KvView& c, uint32_t part, int32_t from, int32_t to) {
  unsigned char* pool = ((part & 1u) ? c.v : c.k) + (size_t)(part >> 1) * c.n_pages * c.page_bytes;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4* a = reinterpret_cast<const u32x4*>(pool + (size_t)from * c.page_bytes);
  u32x4* b = reinterpret_cast<u32x4*>(pool + (size_t)to * c.page_bytes);
  const uint32_t m = c.page_bytes / 16;          // a page has at least 1 KB
  for (uint32_t base = threadIdx.x; base < m; base += 256 * 8) {
    u32x4 v[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      const u32x4* from_at = a + (base + j * 256 < m ? base + j * 256 : base);
      if constexpr (STREAM) v[j] = __builtin_nontemporal_load(from_at); else v[j] = *from_at;
    }
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j)
      if (base + j * 256 < m) {
        if constexpr (STREAM) __builtin_nontemporal_store(v[j], b + base + j * 256); else b[base + j * 256] = v[j];
      }
  }
}

// The pages that an extension copies: grid (entries, 2 * layers)
__global__ __launch_bounds__(256) void kv_copy_pairs_kernel(KvView c, const int2* __restrict__ pairs) {
  const int2 p = pairs[blockIdx.x];
  if (p.x >= 0) kv_copy_page<false>(c, blockIdx.y, p.x, p.y);
}

__global__ __launch_bounds__(256) void kv_copy_listed_kernel(KvView c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, uint32_t n,
                                                             int32_t* __restrict__ status) {
  const uint32_t i = blockIdx.x;
  const int32_t a = src[i], b = dst[i];
  bool bad = (uint32_t)a >= c.n_pages || (uint32_t)b >= c.n_pages;
  bad = kv_in_list(dst, i, b) || bad;
  bad = kv_in_list(dst, n, a) || bad;
  if (blockIdx.y == 0 && threadIdx.x == 0 && status != nullptr) status[i] = bad ? SIF_E_INVAL : SIF_OK;
  if (!bad) kv_copy_page<false>(c, blockIdx.y, a, b);
}

// Compact, the plan: one block counts the used pages (their number is where the used region will end), lists the free pages below and
// the used ones above, and notes where each of the latter goes.
__global__ __launch_bounds__(1024) void kv_plan_compact_kernel(KvView c, KvWork w) {
  __shared__ uint32_t sm[17];
  const uint32_t t = threadIdx.x;
  uint32_t mine = 0, total;
  for (uint32_t p = t * 16; p < c.n_pages; p += 1024 * 16) {
    uint32_t here;
    mine += __popc(kv_used16(c, p, &here));
  }
  kv_block_scan(mine, sm, &total);
  uint32_t holes = 0, tails = 0;
  for (uint32_t base = 0; base < c.n_pages; base += 1024 * 16) {
    const uint32_t p = base + t * 16;
    uint32_t here = 0, used = p < c.n_pages ? kv_used16(c, p, &here) : 0u;
    const uint32_t below = total <= p ? 0u : (total - p >= 16 ? 0xFFFFu : (1u << (total - p)) - 1u);
    uint32_t open = here & ~used & below, moving = used & ~below, more;
    // both ranks in one sum: at most 16384 of each a turn
    const uint32_t both = __popc(open) | (__popc(moving) << 16);
    const uint32_t upto = kv_block_scan(both, sm, &more);
    uint32_t r = holes + (upto & 0xFFFFu) - __popc(open), q = tails + (upto >> 16) - __popc(moving);
    while (open != 0) {
      w.low[r++] = (int32_t)(p + __ffs(open) - 1);
      open &= open - 1;
    }
    for (uint32_t e = 0; e < 16; ++e)
      if ((here & ~below) >> e & 1u) {
        w.map[p + e] = (int32_t)(p + e);
        if (moving >> e & 1u) w.high[q++] = (int32_t)(p + e);
      }
    holes += more & 0xFFFFu;
    tails += more >> 16;
  }
  __syncthreads();                               // the lists are written; there are as many holes as pages to move
  for (uint32_t r = t; r < tails; r += 1024) w.map[w.high[r]] = w.low[r];
  if (t == 0) {
    w.count[0] = tails;
    w.count[1] = total;
  }
}

// Compact, the moves: blocks take (page, layer, K or V) in turn; the table's entries and the counts beside them.  Sources lie above
// all destinations, so no block waits for another.
__global__ __launch_bounds__(256) void kv_move_kernel(KvView c, KvWork w) {
  const uint32_t moves = w.count[0], total = w.count[1], parts = 2 * c.layers;
  if (moves == 0) return;
  const uint64_t at = blockIdx.x * 256ull + threadIdx.x, step = gridDim.x * 256ull, entries = (uint64_t)c.n_seqs * c.table_ld;
  for (uint64_t i = at; i < entries; i += step) {
    const int32_t p = c.table[i];
    if ((uint32_t)p < c.n_pages && (uint32_t)p >= total) c.table[i] = w.map[p];
  }
  for (uint64_t i = at; i < moves; i += step) {
    const int32_t from = w.high[i];
    c.refs[w.low[i]] = c.refs[from];
    c.refs[from] = 0;
  }
  for (uint64_t i = blockIdx.x; i < (uint64_t)moves * parts; i += gridDim.x) {
    const uint32_t r = (uint32_t)(i / parts);
    kv_copy_page<true>(c, (uint32_t)(i % parts), w.high[r], w.low[r]);
  }
}

// float -> e4m3, held at +-448, NaN kept; two at a time into the low half of a word
__device__ __forceinline__ uint32_t kv_e4m3x2(float a, float b) {
  a = a != a ? a : fminf(fmaxf(a, -448.f), 448.f);
  b = b != b ? b : fminf(fmaxf(b, -448.f), 448.f);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}

// Write: a block takes 16 rows of one kv head.  Keys go out as the 16-byte vectors they come in as; values pass through LDS, so that
// lanes which are neighbours in a page's row of tokens store neighbouring elements.
template <int DH, bool E4M3>
__global__ __launch_bounds__(256) void kv_write_kernel(KvView c, uint32_t layer, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, uint32_t ld_k,
                                                       uint32_t ld_v, const int32_t* __restrict__ seqs, const int32_t* __restrict__ starts, uint32_t n, uint32_t rows) {
  constexpr int CH = DH / 8, LD = DH + 2;
  __shared__ int32_t s_page[16];
  __shared__ uint32_t s_off[16];
  __shared__ bf16_t tile[16 * LD];
  const uint32_t t = threadIdx.x, row0 = blockIdx.x * 16, head = blockIdx.y;
  {
    // sixteen threads per row look whether its sequence was listed before
    const uint32_t r = t >> 4, row = row0 + r;
    uint32_t i = row;
    int32_t s = -1;
    uint32_t pos = 0;
    if (row < rows) {
      uint32_t from = row, to = row + 1;
      if (starts != nullptr) {
        uint32_t lo = 0, hi = n;                 // the last entry that begins at or before the row
        while (lo < hi) {
          const uint32_t mid = (lo + hi) >> 1;
          if (starts[mid] <= (int32_t)row) lo = mid + 1; else hi = mid;
        }
        i = lo - 1;
        from = lo > 0 ? (uint32_t)starts[i] : 0u;
        to = lo > 0 ? (uint32_t)starts[i + 1] : 0u;
      }
      if (i < n && from <= row && row < to) {
        s = kv_listed(c, seqs, i);
        if (s >= 0) {
          const uint32_t len = kv_length(c, s), back = to - row;
          if (back <= len) pos = len - back; else s = -1;
        }
      }
    }
    bool again = false;
    if (s >= 0 && seqs != nullptr)
      for (uint32_t j = t & 15; j < i; j += 16) again |= seqs[j] == s;
    const uint64_t votes = __ballot(again);
    if ((t & 15) == 0) {
      int32_t p = -1;
      if (s >= 0 && ((votes >> (t & 63)) & 0xFFFFull) == 0) p = c.table[(size_t)s * c.table_ld + (pos >> c.page_lg)];
      s_page[r] = (uint32_t)p < c.n_pages ? p : -1;
      s_off[r] = pos & ((1u << c.page_lg) - 1u);
    }
  }
  __syncthreads();
  const size_t base = (size_t)layer * c.n_pages, head_bytes = c.page_bytes / c.kv_heads;
  constexpr uint32_t kElt = E4M3 ? 1u : 2u;
  const float ks = E4M3 && c.k_scale != nullptr ? c.k_scale[layer * c.kv_heads + head] : 1.f;
  const float vs = E4M3 && c.v_scale != nullptr ? c.v_scale[layer * c.kv_heads + head] : 1.f;
  if (t < 16 * CH) {
    const uint32_t r = t / CH, ch = t % CH;
    const int32_t p = s_page[r];
    if (p >= 0) {
      const uint4 x = *reinterpret_cast<const uint4*>(k + (size_t)(row0 + r) * ld_k + head * DH + ch * 8);
      const uint4 y = *reinterpret_cast<const uint4*>(v + (size_t)(row0 + r) * ld_v + head * DH + ch * 8);
      unsigned char* to = c.k + (base + (uint32_t)p) * c.page_bytes + head * head_bytes + (s_off[r] * DH + ch * 8) * kElt;
      if constexpr (E4M3) {
        const uint32_t lo = kv_e4m3x2(__fdiv_rn(bflo(x.x), ks), __fdiv_rn(bfhi(x.x), ks)) | kv_e4m3x2(__fdiv_rn(bflo(x.y), ks), __fdiv_rn(bfhi(x.y), ks)) << 16;
        const uint32_t hi = kv_e4m3x2(__fdiv_rn(bflo(x.z), ks), __fdiv_rn(bfhi(x.z), ks)) | kv_e4m3x2(__fdiv_rn(bflo(x.w), ks), __fdiv_rn(bfhi(x.w), ks)) << 16;
        *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
      } else {
        *reinterpret_cast<uint4*>(to) = x;
      }
      uint32_t* at = reinterpret_cast<uint32_t*>(tile + r * LD + ch * 8);
      at[0] = y.x;
      at[1] = y.y;
      at[2] = y.z;
      at[3] = y.w;
    }
  }
  __syncthreads();
  const uint32_t r = t & 15;
  const int32_t p = s_page[r];
  if (p < 0) return;
  unsigned char* to = c.v + (base + (uint32_t)p) * c.page_bytes + head * head_bytes;
#pragma unroll
  for (uint32_t j = 0; j < DH / 16; ++j) {
    const uint32_t d = j * 16 + (t >> 4), at = (d << c.page_lg) + s_off[r];
    const bf16_t x = tile[r * LD + d];
    if constexpr (E4M3) to[at] = (unsigned char)kv_e4m3x2(__fdiv_rn(bf2f(x), vs), 0.f);
    else reinterpret_cast<bf16_t*>(to)[at] = x;
  }
}

}  // namespace sif

using namespace sif;
static inline hipStream_t S(void* s) { return reinterpret_cast<hipStream_t>(s); }

extern "C" {

uint64_t sif_kv_workspace_bytes(const sif_kv_cache* c) {
  KvView v;
  return kv_check("kv_workspace_bytes", c, &v) == SIF_OK ? kv_work_bytes(v) : 0;
}

sif_status sif_k_kv_reset(const sif_kv_cache* c, void* stream) {
  KvView v;
  if (sif_status st = kv_check("kv_reset", c, &v)) return st;
  const uint64_t most = (uint64_t)v.n_seqs * v.table_ld > v.n_pages ? (uint64_t)v.n_seqs * v.table_ld : v.n_pages;
  const uint64_t blocks = (most + 1023) / 1024;
  hipLaunchKernelGGL(kv_reset_kernel, dim3((uint32_t)(blocks < 1024 ? blocks : 1024)), dim3(256), 0, S(stream), v);
  return check_launch("kv_reset");
}

sif_status sif_k_kv_extend(const sif_kv_cache* c, const int32_t* seqs, const int32_t* counts, uint32_t n, int32_t* status, void* workspace,
                           uint64_t workspace_bytes, void* stream) {
  KvView v;
  if (sif_status st = kv_check("kv_extend", c, &v)) return st;
  if (sif_status st = kv_check_list("kv_extend", n, seqs, counts, status)) return st;
  if (sif_status st = kv_check_work("kv_extend", v, workspace, workspace_bytes)) return st;
  const KvWork w = kv_work(v, workspace);
  hipLaunchKernelGGL(kv_extend_kernel, dim3(1), dim3(1024), 0, S(stream), v, seqs, counts, n, status, w);
  if (sif_status st = check_launch("kv_extend")) return st;
  hipLaunchKernelGGL(kv_copy_pairs_kernel, dim3(n, 2 * v.layers), dim3(256), 0, S(stream), v, (const int2*)w.pairs);
  return check_launch("kv_extend: copies");
}

sif_status sif_k_kv_write(const sif_kv_cache* c, uint32_t layer, const void* k, const void* v, uint32_t ld_k, uint32_t ld_v, const int32_t* seqs,
                          const int32_t* starts, uint32_t n, uint32_t rows, void* stream) {
  KvView w;
  if (sif_status st = kv_check("kv_write", c, &w)) return st;
  if (layer >= w.layers) return fail(SIF_E_INVAL, "kv_write: no layer %u", layer);
  if (!k || !v || (((uintptr_t)k | (uintptr_t)v) & 15)) return fail(SIF_E_INVAL, "kv_write: k and v must be 16-byte aligned");
  if (n == 0 || rows == 0 || n > (1u << 27) || rows > (1u << 27)) return fail(SIF_E_INVAL, "kv_write: entries or rows outside 1 .. 2^27");
  // every row looks through the list in front of its entry, for each kv head: the work grows with rows times entries (at 2^27 of each it
  // would not end in any useful time; 2^14 entries are 64 KB of list, and 2^10 reads a row and thread)
  if (seqs != nullptr && n > kKvMaxWritten) return fail(SIF_E_INVAL, "kv_write: at most %u listed sequences", kKvMaxWritten);
  if (((uintptr_t)seqs | (uintptr_t)starts) & 3) return fail(SIF_E_INVAL, "kv_write: misaligned list");
  if (starts == nullptr && rows != n) return fail(SIF_E_INVAL, "kv_write: without starts there is one row per entry");
  const uint32_t width = w.kv_heads * w.d_head;
  if (ld_k < width || ld_v < width || ((ld_k | ld_v) & 7)) return fail(SIF_E_INVAL, "kv_write: bad leading dimensions");
  const dim3 grid((rows + 15) / 16, w.kv_heads);
#define KV_LAUNCH(DH, E) hipLaunchKernelGGL((kv_write_kernel<DH, E>), grid, dim3(256), 0, S(stream), w, layer, (const bf16_t*)k, (const bf16_t*)v, ld_k, ld_v, \
                                            seqs, starts, n, rows)
  if (w.d_head == 64) { if (c->dtype == SIF_E4M3) KV_LAUNCH(64, true); else KV_LAUNCH(64, false); }
  else { if (c->dtype == SIF_E4M3) KV_LAUNCH(128, true); else KV_LAUNCH(128, false); }
#undef KV_LAUNCH
  return check_launch("kv_write");
}

sif_status sif_k_kv_fork(const sif_kv_cache* c, const int32_t* src, const int32_t* dst, uint32_t n, int32_t* status, void* stream) {
  KvView v;
  if (sif_status st = kv_check("kv_fork", c, &v)) return st;
  if (sif_status st = kv_check_list("kv_fork", n, src, dst, status)) return st;
  if (!src || !dst) return fail(SIF_E_INVAL, "kv_fork: null list");
  hipLaunchKernelGGL(kv_fork_kernel, dim3(n), dim3(256), 0, S(stream), v, src, dst, n, status);
  return check_launch("kv_fork");
}

static sif_status kv_release(const char* who, const sif_kv_cache* c, const int32_t* seqs, uint32_t n, uint32_t window, uint32_t sinks, void* stream) {
  KvView v;
  if (sif_status st = kv_check(who, c, &v)) return st;
  if (sif_status st = kv_check_list(who, n, seqs)) return st;
  hipLaunchKernelGGL(kv_release_kernel, dim3(n), dim3(256), 0, S(stream), v, seqs, window, sinks);
  return check_launch(who);
}

sif_status sif_k_kv_free(const sif_kv_cache* c, const int32_t* seqs, uint32_t n, void* stream) { return kv_release("kv_free", c, seqs, n, 0, 0, stream); }

sif_status sif_k_kv_trim(const sif_kv_cache* c, const int32_t* seqs, uint32_t n, uint32_t window, uint32_t sinks, void* stream) {
  if (window == 0) return fail(SIF_E_INVAL, "kv_trim: the window holds one token at least");
  return kv_release("kv_trim", c, seqs, n, window, sinks, stream);
}

sif_status sif_k_kv_compact(const sif_kv_cache* c, void* workspace, uint64_t workspace_bytes, void* stream) {
  KvView v;
  if (sif_status st = kv_check("kv_compact", c, &v)) return st;
  if (sif_status st = kv_check_work("kv_compact", v, workspace, workspace_bytes)) return st;
  const KvWork w = kv_work(v, workspace);
  hipLaunchKernelGGL(kv_plan_compact_kernel, dim3(1), dim3(1024), 0, S(stream), v, w);
  if (sif_status st = check_launch("kv_compact: plan")) return st;
  // as many blocks as the chip holds at once, or as there can be pieces of work
  const uint64_t pieces = ((uint64_t)v.n_pages + 1) / 2 * 2 * v.layers;
  hipLaunchKernelGGL(kv_move_kernel, dim3((uint32_t)(pieces < 2048 ? pieces : 2048)), dim3(256), 0, S(stream), v, w);
  return check_launch("kv_compact: moves");
}

sif_status sif_k_kv_copy_pages(const sif_kv_cache* c, const int32_t* src, const int32_t* dst, uint32_t n, int32_t* status, void* stream) {
  KvView v;
  if (sif_status st = kv_check("kv_copy_pages", c, &v)) return st;
  if (sif_status st = kv_check_list("kv_copy_pages", n, src, dst, status)) return st;
  if (!src || !dst) return fail(SIF_E_INVAL, "kv_copy_pages: null list");
  hipLaunchKernelGGL(kv_copy_listed_kernel, dim3(n, 2 * v.layers), dim3(256), 0, S(stream), v, src, dst, n, status);
  return check_launch("kv_copy_pages");
}

}  // extern "C"
