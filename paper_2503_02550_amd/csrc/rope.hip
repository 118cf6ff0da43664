// Rotary positions of rows of query and key heads, forward and back.  Every element is read and written once and costs three operations, so
// the memory's rate is the bound; what could get in the way are the sines: a block takes them once for its rows and all their heads.  671 MB take 119 us, 5.6 TB/s, a plain copy
// 5.1; 50 MB 13; a few rows 3.4, the launch.
#include <algorithm>

#include "rope.h"

namespace sif {

sif_status rope_check(const char* who, const sif_rope* r, uint32_t d_head, RopeView* out) {
  if (!r) return fail(SIF_E_INVAL, "%s: null rotation", who);
  if (r->struct_size != sizeof(sif_rope)) return fail(SIF_E_INVAL, "%s: struct_size of the rotation", who);
  if (r->layout != SIF_ROPE_HALF && r->layout != SIF_ROPE_INTERLEAVED) return fail(SIF_E_INVAL, "%s: the rotation's layout must be SIF_ROPE_HALF or SIF_ROPE_INTERLEAVED", who);
  if (r->rot_dim == 0 || r->rot_dim > 256 || (r->rot_dim & 15) || r->rot_dim > d_head) return fail(SIF_E_INVAL, "%s: rot_dim must be a multiple of 16, at most 256 and d_head", who);
  if (!std::isfinite(r->magnitude) || !std::isfinite((float)r->magnitude)) return fail(SIF_E_INVAL, "%s: the rotation's magnitude must be finite", who);
  out->interleaved = r->layout == SIF_ROPE_INTERLEAVED;
  out->half = r->rot_dim / 2;
  out->magnitude = r->magnitude;
  for (uint32_t i = 0; i < 128; ++i) {
    const double t = i < out->half ? r->turns[i] : 0.0;
    if (!(t >= -1.0 && t <= 1.0)) return fail(SIF_E_INVAL, "%s: turns per token must be between -1 and 1", who);
    out->turns[i] = t;
  }
  return SIF_OK;
}

struct RopeArgs {
  const int32_t* positions;
  const bf16_t* q;
  const bf16_t* k;
  bf16_t* q_out;
  bf16_t* k_out;
  uint32_t rows, heads, all_heads, d_head, seq, ld_q, ld_q_out, ld_k, ld_k_out;
  int32_t first;
  float back;
  uint32_t units, slots, tile;       // sixteen elements each of a head; heads a block takes at once; rows it takes at once
  uint32_t copies;                   // of the units, those of elements behind the rotated ones, where results do not take their operands' place
  bool copy_q, copy_k;
};

// Sixteen elements of a head and row to a thread, eight pairs or what stands behind the rotated ones, two 16-byte vectors in, two out: consecutive threads take a head's units,
// then the next heads', which lie next to it in memory, then the next row's.  (With the elements behind left to the threads that turn, 32768 rows of 16 heads of 128 of which 16 elements are
// turned took 210 us, 32 elements 98, all of them 52.)
__global__ __launch_bounds__(256) void rope_kernel(RopeView r, RopeArgs a) {
  __shared__ __align__(16) CosSin<float> s_cs[2048];      // [row][pair]
  const uint32_t tid = threadIdx.x, unit = tid % a.units, slot = tid / a.units % a.slots, row = tid / (a.units * a.slots);
  const uint32_t tiles = (a.rows + a.tile - 1) / a.tile;
  for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const uint32_t row0 = tile * a.tile;
    __syncthreads();                               // nobody reads the last tile's table any more
    for (uint32_t i = tid; i < a.tile * r.half; i += 256) {
      const uint32_t at = row0 + i / r.half;
      if (at < a.rows) {
        const double pos = a.positions != nullptr ? (double)a.positions[at] : (double)a.first + (double)(at % a.seq);
        s_cs[i] = rope_cos_sin<float>(r, pos, i % r.half);
      }
    }
    __syncthreads();
    const uint32_t at = row0 + row;
    if (row >= a.tile || at >= a.rows) continue;
    const uint32_t turning = a.units - a.copies;
    const bool turns = unit < turning;
    CosSin<float> cs[8];
    uint32_t x, y;
    if (turns) {
#pragma unroll
      for (uint32_t e = 0; e < 8; e += 2) *reinterpret_cast<float4*>(&cs[e]) = *reinterpret_cast<const float4*>(&s_cs[row * r.half + unit * 8 + e]);
      x = r.interleaved ? unit * 16 : unit * 8;
      y = r.interleaved ? x + 8 : x + r.half;
    } else {
      x = 2 * r.half + (unit - turning) * 8;
      y = x + a.copies * 8 < a.d_head ? x + a.copies * 8 : x;      // (of an odd number the last one twice)
    }
    for (uint32_t h = blockIdx.y * a.slots + slot; h < a.all_heads; h += gridDim.y * a.slots) {
      const bool of_q = h < a.heads;
      if (!turns && !(of_q ? a.copy_q : a.copy_k)) continue;
      const uint32_t c = (of_q ? h : h - a.heads) * a.d_head;
      const bf16_t* from = of_q ? a.q + (size_t)at * a.ld_q + c : a.k + (size_t)at * a.ld_k + c;
      bf16_t* to = of_q ? a.q_out + (size_t)at * a.ld_q_out + c : a.k_out + (size_t)at * a.ld_k_out + c;
      uint4 u = *reinterpret_cast<const uint4*>(from + x), v = *reinterpret_cast<const uint4*>(from + y);
      if (turns) rope_turn8(r.interleaved, cs, a.back, u, v);
      *reinterpret_cast<uint4*>(to + x) = u;
      *reinterpret_cast<uint4*>(to + y) = v;
    }
  }
}

}  // namespace sif

using namespace sif;

extern "C" {

sif_status sif_rope_plan(const sif_rope_desc* d, sif_rope* out) {
  if (!d || !out) return fail(SIF_E_INVAL, "rope_plan: null argument");
  if (d->struct_size != sizeof(sif_rope_desc)) return fail(SIF_E_INVAL, "rope_plan: struct_size");
  if (d->scaling > SIF_ROPE_PARTS) return fail(SIF_E_INVAL, "rope_plan: no scaling %u", d->scaling);
  if (d->rot_dim == 0 || d->rot_dim > 256 || (d->rot_dim & 15)) return fail(SIF_E_INVAL, "rope_plan: rot_dim must be a multiple of 16, at most 256");
  if (!(d->base >= 1.0) || !std::isfinite(d->base)) return fail(SIF_E_INVAL, "rope_plan: base must be finite and at least 1");
  if (d->scaling != SIF_ROPE_PLAIN && (!(d->factor > 0.0) || !std::isfinite(d->factor))) return fail(SIF_E_INVAL, "rope_plan: factor must be finite and above 0");
  if (d->scaling == SIF_ROPE_PARTS && (!(d->low_turns < d->high_turns) || !std::isfinite(d->high_turns - d->low_turns) || !(d->trained_tokens > 0.0) || !std::isfinite(d->trained_tokens)))
    return fail(SIF_E_INVAL, "rope_plan: low_turns must be below high_turns, trained_tokens above 0, all finite");
  constexpr double two_pi = 6.283185307179586476925;
  sif_rope r = {};
  r.struct_size = sizeof(sif_rope);
  r.layout = d->layout;
  r.rot_dim = d->rot_dim;
  r.magnitude = d->magnitude;
  const double base = d->scaling == SIF_ROPE_BASE ? d->base * pow(d->factor, (double)d->rot_dim / (d->rot_dim - 2.0)) : d->base;
  for (uint32_t i = 0; i < d->rot_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / d->rot_dim);
    if (d->scaling == SIF_ROPE_LINEAR) f /= d->factor;
    if (d->scaling == SIF_ROPE_PARTS) {
      const double turns = d->trained_tokens * f / two_pi;
      const double g = std::min(1.0, std::max(0.0, (turns - d->low_turns) / (d->high_turns - d->low_turns)));
      f = g * f + (1.0 - g) * f / d->factor;
    }
    r.turns[i] = f / two_pi;
  }
  RopeView v;
  if (sif_status st = rope_check("rope_plan", &r, 256, &v)) return st;
  *out = r;
  return SIF_OK;
}

sif_status sif_k_rope(const sif_rope* rope, const sif_rope_args* a, void* stream) {
  if (!a) return fail(SIF_E_INVAL, "rope: null arguments");
  if (a->struct_size != sizeof(sif_rope_args)) return fail(SIF_E_INVAL, "rope: struct_size");
  if (a->d_head == 0 || (a->d_head & 7) || a->d_head > 256) return fail(SIF_E_INVAL, "rope: d_head must be a multiple of 8, at most 256");
  RopeView v;
  if (sif_status st = rope_check("rope", rope, a->d_head, &v)) return st;
  if (!a->rows || !a->heads || a->rows >= 1u << 31) return fail(SIF_E_INVAL, "rope: rows below 2^31, and at least one row and one head");
  if (a->heads > 16384 || a->kv_heads > 16384) return fail(SIF_E_INVAL, "rope: at most 16384 heads");
  if (!a->positions_dev && !a->seq) return fail(SIF_E_INVAL, "rope: without positions a sequence has at least one token");
  if (a->inverse > 1) return fail(SIF_E_INVAL, "rope: inverse is 0 or 1");
  if (!a->q_dev || !a->q_out_dev || (a->kv_heads && (!a->k_dev || !a->k_out_dev))) return fail(SIF_E_INVAL, "rope: null operand");
  const uintptr_t k_ptrs = a->kv_heads ? (uintptr_t)a->k_dev | (uintptr_t)a->k_out_dev : 0;
  if (((uintptr_t)a->q_dev | (uintptr_t)a->q_out_dev | k_ptrs) & 15) return fail(SIF_E_INVAL, "rope: q and k must be 16-byte aligned");
  if ((uintptr_t)a->positions_dev & 3) return fail(SIF_E_INVAL, "rope: misaligned positions");
  const uint64_t wq = (uint64_t)a->heads * a->d_head, wk = (uint64_t)a->kv_heads * a->d_head;
  auto bad = [](uint32_t ld, uint64_t width) { return ld < width || (ld & 7) || ld >= 1u << 27; };
  if (bad(a->ld_q, wq) || bad(a->ld_q_out, wq) || (a->kv_heads && (bad(a->ld_k, wk) || bad(a->ld_k_out, wk)))) return fail(SIF_E_INVAL, "rope: bad leading dimensions");
  const bool q_there = a->q_dev == a->q_out_dev, k_there = a->kv_heads && a->k_dev == a->k_out_dev;
  if ((q_there && a->ld_q != a->ld_q_out) || (k_there && a->ld_k != a->ld_k_out)) return fail(SIF_E_INVAL, "rope: in place, with one leading dimension");
  RopeArgs x;
  x.positions = a->positions_dev;
  x.q = (const bf16_t*)a->q_dev;
  x.k = (const bf16_t*)a->k_dev;
  x.q_out = (bf16_t*)a->q_out_dev;
  x.k_out = (bf16_t*)a->k_out_dev;
  x.rows = a->rows;
  x.heads = a->heads;
  x.all_heads = a->heads + a->kv_heads;
  x.d_head = a->d_head;
  x.seq = a->seq;
  x.first = a->first;
  x.back = a->inverse ? -1.f : 1.f;
  x.ld_q = a->ld_q;
  x.ld_q_out = a->ld_q_out;
  x.ld_k = a->ld_k;
  x.ld_k_out = a->ld_k_out;
  x.copy_q = !q_there;
  x.copy_k = !k_there;
  x.copies = q_there && (k_there || !a->kv_heads) ? 0 : ((a->d_head - 2 * v.half) / 8 + 1) / 2;
  x.units = v.half / 8 + x.copies;                 // 1 .. 16
  // Two rows or more to a block, and as many heads as that leaves: they lie next to each other in its loads, and each row's sines serve them all.  (Rows to a block at least 1, 2, 4, 8: 32762 rows of
  // 40 heads of 128, half of each turned 124, 120, 125, 130 us; 16384 of 16 heads of 256 50 to 53, 49 to 51, 51, 54; 52428 of 16 heads of 80, where two rows fill 240 to 250 of a block's threads and four 192 or 200, 51, 51, 56, 54.)
  x.slots = std::min(x.all_heads, 256 / x.units / 2);
  x.tile = 256 / (x.units * x.slots);
  x.tile = std::min(x.tile, 2048 / v.half);        // the table's size
  const uint32_t tiles = (a->rows + x.tile - 1) / x.tile, rounds = (x.all_heads + x.slots - 1) / x.slots;
  const uint32_t gx = std::min(tiles, 1u << 20), gy = std::max(1u, std::min(rounds, 1024u / gx));
  hipLaunchKernelGGL(rope_kernel, dim3(gx, gy), dim3(256), 0, reinterpret_cast<hipStream_t>(stream), v, x);
  return check_launch("rope");
}

}  // extern "C"
