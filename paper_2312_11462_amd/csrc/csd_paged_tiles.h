// Shared by the kernels of many rows: staged key tiles, matrix products of 32 rows.
#pragma once

#include "csd_paged.h"

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

static constexpr int kKeys = 64;                             // keys per tile

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ float halves_max(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// 16-byte piece c of row `row` in a staged tile
template <int DH> __device__ __forceinline__ int k_piece(int row, int c) { return row * (DH / 8) + (c ^ (row & (DH / 8 - 1))); }
template <int DH> __device__ __forceinline__ int v_piece(int row, int c) {
    return row * (DH / 8) + (c ^ (DH == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2));
}

// The key tiles that row tile rt of a sequence goes through: those up to the last position that one of its rows attends.
__device__ __forceinline__ int row_tile_keys(int rt, int m, int t, int group, int cap) {
    const int last = min(((rt + 1) * CSD_PAGED_MANY_ROWS - 1) / group, m - 1);
    return (min(t + last + 1, cap) + kKeys - 1) / kKeys;
}
