// LDS tiles of bf16 rows that serve products along their columns and, turned, along their rows (gfx950).
//
// A tile row has DP columns (64, 128 or 256); its 16-byte pieces are permuted by the row, so that neither row-wise reads (32 rows, one
// column piece) nor transpose reads (four rows, 64 bytes) meet in a bank: no conflicts counted at width 256.  Tiles are filled by
// direct-to-LDS loads, which put a wave's 64 pieces side by side: the permutation is in the addresses that the lanes load from.
#pragma once
#include "common.h"

typedef bf16_t lds_bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t lds_bf16x4 __attribute__((ext_vector_type(4)));
typedef short lds_s16x4 __attribute__((ext_vector_type(4)));
#define LDS_AS __attribute__((address_space(3)))
typedef LDS_AS char lds_char;

template <int DP>
__host__ __device__ constexpr int lds_swizzle(int row) {
  return DP >= 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}
__device__ __forceinline__ void load_lds16(const void *g, lds_char *l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)g, (LDS_AS void *)l, 16, 0, 0);
}
// where column piece p (8 columns) of a row is
template <int DP>
__device__ __forceinline__ uint32_t lds_piece(int row, int p) {
  return (uint32_t)(row * DP * 2 + ((p ^ lds_swizzle<DP>(row)) << 4));
}
// A lane's place for the transpose reads below
template <int DP>
__device__ __forceinline__ uint32_t lds_turn_place(int lane) {
  const int h = lane >> 5, in_half = (lane >> 4) & 1, t = (lane & 15) >> 2, u = lane & 3;  // row t, 4 columns from 16 in_half + 4 u
  return (uint32_t)((4 * h + t) * DP * 2 + (((2 * in_half + (u >> 1)) ^ lds_swizzle<DP>(4 * h + t)) << 4) + (u & 1) * 8);
}
// Matrix-core operand (32 x 32 x 16) whose reduction index runs over the rows 16 t .. 16 t + 15 of the tile, and whose other index over
// the columns 32 dt .. 32 dt + 31: lane l holds column 32 dt + l % 32, and as element j the row 16 t + 8 (j / 4) + 4 (l / 32) + j % 4.
// A transpose read gives a lane four rows of one column.
template <int DP>
__device__ __forceinline__ lds_bf16x8 lds_turned(const lds_char *tile, uint32_t place, int dt, int t) {
  const uint32_t at = (place ^ ((dt & 3) * 64)) + (dt >> 2) * 256 + 16 * t * DP * 2;
  // (the second half is 8 rows on: swizzle turned over in its second bit)
  const uint32_t at2 = (place ^ ((dt & 3) * 64 + 32)) + (dt >> 2) * 256 + (16 * t + 8) * DP * 2;
  const lds_bf16x4 x = __builtin_bit_cast(lds_bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS lds_s16x4 *)(tile + at)));
  const lds_bf16x4 y = __builtin_bit_cast(lds_bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS lds_s16x4 *)(tile + at2)));
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
// The same where dt is known to the wave, not to the compiler
template <int DP>
__device__ __forceinline__ lds_bf16x8 lds_turned_at(const lds_char *tile, uint32_t place, int dt, int t) {
  const uint32_t turn = (uint32_t)(dt & 3) * 64, on = (uint32_t)(dt >> 2) * 256;
  const lds_bf16x4 x = __builtin_bit_cast(lds_bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS lds_s16x4 *)(tile + ((place ^ turn) + on + 16 * t * DP * 2))));
  const lds_bf16x4 y = __builtin_bit_cast(lds_bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS lds_s16x4 *)(tile + ((place ^ (turn | 32)) + on + (16 * t + 8) * DP * 2))));
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
// A barrier for LDS alone: what the wave has written there is there; its loads from memory stay out.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt 0 (vmcnt 63 and expcnt 7: nothing)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
