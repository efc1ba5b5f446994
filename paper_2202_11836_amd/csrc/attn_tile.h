// Device pieces shared by the attention kernels: 32 x 32 MFMA accumulators,
// operand fragments of row-major [rows][64] bf16 tiles in LDS, and the mapping of
// work-groups to row blocks.
#pragma once
#include "kernels.h"

namespace {

typedef __attribute__((address_space(3))) void lds_void_t;

__device__ __forceinline__ f32x16_t mfma32(bf16x8_t a, bf16x8_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Row of register r in a 32x32 accumulator for lane half hf.
__device__ __forceinline__ int acc_row(int r, int hf) { return 8 * (r >> 2) + 4 * hf + (r & 3); }

__device__ __forceinline__ f32x16_t splat16(float v) {
  f32x16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = v;
  return z;
}

__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.0f;
  return z;
}

// Registers r0 .. r0+7 of an accumulator as a bf16 operand.
__device__ __forceinline__ bf16x8_t pack8(const f32x16_t& a, int r0) {
  const u32x4_t w = {pack_bf16x2(a[r0], a[r0 + 1]), pack_bf16x2(a[r0 + 2], a[r0 + 3]),
                     pack_bf16x2(a[r0 + 4], a[r0 + 5]), pack_bf16x2(a[r0 + 6], a[r0 + 7])};
  return __builtin_bit_cast(bf16x8_t, w);
}

__device__ __forceinline__ bf16x8_t ld_frag(const bf16_t* p) { return *(const bf16x8_t*)p; }

__device__ __forceinline__ u32x4_t zero4() { return u32x4_t{0, 0, 0, 0}; }

// LDS tile [64 rows][64 bf16]: 128-byte rows of 8 16-byte chunks, chunk c of
// row r stored at chunk c ^ f(u), u = (r >> 1) & 7, f(u) = (u0 << 2) |
// (u2 << 1) | u1.  The 16 rows of a row-fragment read and the 4 rows x 64
// bytes of a transposing read then fall on distinct banks.
__device__ __forceinline__ int tswz(int r) {
  const int u = (r >> 1) & 7;
  return ((u & 1) << 2) | (((u >> 2) & 1) << 1) | ((u >> 1) & 1);
}
__device__ __forceinline__ int toff(int r, int c) { return r * 128 + 16 * (c ^ tswz(r)); }

// A operand from tile rows: lane l reads row r0 + l % 32, columns
// 16 ks + 8 (l / 32) .. +7.
__device__ __forceinline__ bf16x8_t frag_rows(const char* tile, int r0, int ks, int lane) {
  return *(const bf16x8_t*)(tile + toff(r0 + (lane & 31), 2 * ks + (lane >> 5)));
}

// Transposed A operand: lane l gets column col0 + l % 32 at the tile rows
// rb + 4 hf + {0..3} and rb + 8 + 4 hf + {0..3} (hf = l / 32), which with
// rb = row base + 16 ks is the row order of accumulator registers
// 8 ks .. 8 ks + 7.  ds_read_b64_tr_b16 works on groups of 16 lanes: lane j
// supplies the address of 4 consecutive 16-bit values V[j][0..3] and lane i
// receives V[4e + i / 4][i % 4], e = 0..3; lane j points at row
// rb + 4 hf + j / 4, columns c0 + 4 (j % 4) .. +3, so lane i receives column
// c0 + i of those 4 rows.
__device__ __forceinline__ bf16x8_t frag_tr(const char* tile, int col0, int rb, int lane) {
  typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4_t;
  const int j = lane & 15;
  const int r = rb + 4 * (lane >> 5) + (j >> 2);
  const int d = col0 + 16 * ((lane >> 4) & 1) + 4 * (j & 3);
  const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
      (lds_bf16x4_t*)(tile + toff(r, d >> 3) + 2 * (d & 7)));
  const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
      (lds_bf16x4_t*)(tile + toff(r + 8, d >> 3) + 2 * (d & 7)));
  return bf16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// "vmcnt = 0 and lgkmcnt = 0" (gfx9 s_waitcnt encoding).
__device__ __forceinline__ void wait_all() { __builtin_amdgcn_s_waitcnt(0x0070); }

// The values of lanes l and l ^ 32 (as a pair, in either order) from one
// v_permlane32_swap, which exchanges the upper half of its first operand
// with the lower half of its second: no LDS round trip, unlike a shuffle.
struct HalfPair {
  float x, y;
};
__device__ __forceinline__ HalfPair half_pair(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}

// Work-group w of n -> (row block, batch * head), nq row blocks per (batch,
// head); consecutive work-groups go round robin
// over the 8 XCDs, so they are remapped such that each XCD takes a
// contiguous range and the row blocks of one (batch, head), which stream the
// same keys and values (or queries and output gradients), share that XCD's
// L2.
__device__ __forceinline__ void attn_block(int w, int n, int nq, int& rb, int& bh) {
  if ((n & 7) == 0) w = (w & 7) * (n >> 3) + (w >> 3);
  rb = w % nq;
  bh = w / nq;
}

}  // namespace
