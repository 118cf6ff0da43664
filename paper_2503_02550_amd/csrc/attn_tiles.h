// Tiles of fused attention kernels: rows of bf16 matrices fetched into LDS, MFMA operands read from there, results written out.
// (What an operand's k elements are, and why, is said in attention.hip.)
#pragma once
#include "common.h"

namespace sif {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int AT_Q = 128, AT_KV = 128, AT_THREADS = 256;
constexpr int AT_QB = 64;                                    // query rows per step of the dk/dv kernel

__device__ __forceinline__ uint32_t at_key(uint32_t row) { return (row & 7u) ^ ((row >> 3) & 1u); }

// ROWS x DH tile of a row-major bf16 matrix (rows row0.., 16-byte aligned, ld elements apart) into LDS as [row][d] with
// the 16-byte chunks of a row XOR-swizzled, fetched from global memory straight into LDS (global_load_lds_dwordx4: no
// staging registers, the fetch of the next tile runs while the current one is used).  One instruction writes the 64 lanes' 16 bytes to
// consecutive LDS addresses, so a lane's place in the tile is fixed and the swizzle is applied to what it fetches.
// Rows >= limit cannot be zero-filled: they fetch row limit - 1 instead (finite data), and every use of such a row is
// either masked (scores) or multiplied by a probability of zero.
template <int DH, int ROWS>
__device__ __forceinline__ void at_dma_rows(bf16_t* dst, const bf16_t* src, size_t ld, uint32_t row0, uint32_t limit) {
  typedef __attribute__((address_space(3))) void* lds_void_ptr;
  typedef __attribute__((address_space(1))) const void* global_void_ptr;
  constexpr int CH = DH / 8, RPI = 64 / CH;                  // chunks per row, rows per instruction and wavefront
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < ROWS / (RPI * (AT_THREADS / 64)); ++i) {
    const uint32_t first = (i * (AT_THREADS / 64) + wave) * RPI, row = first + lane / CH, c = (lane % CH) ^ (at_key(row) % CH);
    const uint32_t r = row0 + row < limit ? row0 + row : limit - 1;
    __builtin_amdgcn_global_load_lds((global_void_ptr)(src + (size_t)r * ld + c * 8), (lds_void_ptr)(dst + first * DH), 16, 0, 0);
  }
}
// 32 rows fetched the same way by ONE wavefront into 32*DH elements of LDS of its own (rows swizzled by their number
// within the 32): whole 128-byte rows per fetch, where a lane that reads its own row from global memory fetches 16
// bytes of it per instruction.
template <int DH>
__device__ __forceinline__ void at_dma_rows_wave(bf16_t* dst, const bf16_t* src, size_t ld, uint32_t row0, uint32_t limit) {
  typedef __attribute__((address_space(3))) void* lds_void_ptr;
  typedef __attribute__((address_space(1))) const void* global_void_ptr;
  constexpr int CH = DH / 8, RPI = 64 / CH;
  const uint32_t lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 32 / RPI; ++i) {
    const uint32_t first = i * RPI, row = first + lane / CH, c = (lane % CH) ^ (at_key(row) % CH);
    const uint32_t r = row0 + row < limit ? row0 + row : limit - 1;
    __builtin_amdgcn_global_load_lds((global_void_ptr)(src + (size_t)r * ld + c * 8), (lds_void_ptr)(dst + first * DH), 16, 0, 0);
  }
}
// A wavefront's 32 x DH results, held transposed in MFMA accumulators (element r of tile d in lane (qi, h) is column
// d*32 + (r/4)*8 + h*4 + r%4 of row qi), times mul, to global memory as whole rows.  Stored straight from the
// accumulators a lane would write 8 bytes at a time and every 128-byte line of the output would be touched by eight
// store instructions, 16 bytes each.  So the tile passes through 32*DH elements of LDS that belong to this wavefront
// alone (16-byte chunks of a row swizzled with the row) and leaves as 16-byte vectors, a row of 128 bytes per eight
// lanes.  dst = row 0, column 0 of the tile; only the first `rows` rows exist.
template <int DH>
__device__ __forceinline__ void at_store_tile(bf16_t* stage, const floatx16 (&acc)[DH / 32], float mul, bf16_t* dst, size_t ld, uint32_t rows) {
  constexpr int CH = DH / 8;
  const uint32_t lane = threadIdx.x & 63, qi = lane & 31, h = lane >> 5;
#pragma unroll
  for (int d = 0; d < DH / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<uint2*>(stage + qi * DH + (((d * 4 + g) ^ (qi & 7u)) << 3) + h * 4) =
          make_uint2(pack_bf2(acc[d][4 * g] * mul, acc[d][4 * g + 1] * mul), pack_bf2(acc[d][4 * g + 2] * mul, acc[d][4 * g + 3] * mul));
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int it = 0; it < 32 * CH / 64; ++it) {
    const uint32_t idx = lane + it * 64, row = idx / CH, c = idx % CH;
    const uint4 v = *reinterpret_cast<const uint4*>(stage + row * DH + ((c ^ (row & 7u)) << 3));
    if (row < rows) *reinterpret_cast<uint4*>(dst + (size_t)row * ld + c * 8) = v;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// A operand (row, k = 8 consecutive d) from a swizzled [row][d] tile; chunk = k / 8.
template <int DH>
__device__ __forceinline__ bf16x8 at_frag(const bf16_t* tile, uint32_t row, uint32_t chunk) {
  return *reinterpret_cast<const bf16x8*>(tile + row * DH + ((chunk ^ (at_key(row) % (DH / 8))) << 3));
}
// A operand of a product that contracts over the tile's rows: operand row d (32 of them from dbase32, one per lane
// and lane + 32), k = the tile rows kb..kb+3 and kb+8..kb+11 (kb already holds the lane half's offset of 4).  The
// tile stays [row][d]; the transposing LDS read of gfx950 (ds_read_b64_tr_b16) does the rest: within a group of
// 16 lanes, source lane s supplies the address of four consecutive d at tile row kb + s/4, d = d0 + 4*(s%4).., and
// lane i receives d0 + i at the four tile rows.
template <int DH>
__device__ __forceinline__ bf16x8 at_frag_tr(const bf16_t* tile, uint32_t dbase32, uint32_t kb) {
  typedef short short4_lds __attribute__((ext_vector_type(4)));
  typedef short short8_v __attribute__((ext_vector_type(8)));
  typedef __attribute__((address_space(3))) short4_lds* lds_ptr;
  const uint32_t lane = threadIdx.x & 63, s = lane & 15;
  const uint32_t row = kb + (s >> 2), d = dbase32 + ((lane >> 4) & 1u) * 16 + 4 * (s & 3u);
  const bf16_t* p0 = tile + row * DH + ((((d >> 3) ^ (at_key(row) % (DH / 8))) << 3) | (d & 7u));
  const bf16_t* p1 = tile + (row + 8) * DH + ((((d >> 3) ^ (at_key(row + 8) % (DH / 8))) << 3) | (d & 7u));
  const short4_lds lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p0);
  const short4_lds hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p1);
  const short8_v v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, v);
}
// eight accumulator values r0..r0+7 as a B operand
__device__ __forceinline__ bf16x8 at_pack8(const float (&v)[16], int r0) {
  uint4 pv = make_uint4(pack_bf2(v[r0], v[r0 + 1]), pack_bf2(v[r0 + 2], v[r0 + 3]), pack_bf2(v[r0 + 4], v[r0 + 5]), pack_bf2(v[r0 + 6], v[r0 + 7]));
  return *reinterpret_cast<bf16x8*>(&pv);
}
__device__ __forceinline__ float at_round(float x) { return bf2f(f2bf(x)); }

}  // namespace sif
