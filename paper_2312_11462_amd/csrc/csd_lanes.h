// Sums over the lanes of a wave by data-parallel moves (a shuffle goes through LDS), of 32 and 64 bits.
#pragma once

#include "csd_internal.h"

typedef unsigned long long u64;

// what another lane of the wave has, by data-parallel moves; `old` where there is none
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t old, uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 old, u64 v) {
    return (u64)moved<CTRL, ROWS>((uint32_t)(old >> 32), (uint32_t)(v >> 32)) << 32 | moved<CTRL, ROWS>((uint32_t)old, (uint32_t)v);
}
// inclusive running sum over the wave: within sixteen lanes, then from row to row
template <typename U>
__device__ __forceinline__ U wave_scan(U v) {
    v += moved<0x111, 0xF>((U)0, v);
    v += moved<0x112, 0xF>((U)0, v);
    v += moved<0x114, 0xF>((U)0, v);
    v += moved<0x118, 0xF>((U)0, v);
    v += moved<0x142, 0xA>((U)0, v);
    v += moved<0x143, 0xC>((U)0, v);
    return v;
}
__device__ __forceinline__ uint32_t from_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ u64 from_lane(u64 v, int lane) { return (u64)from_lane((uint32_t)(v >> 32), lane) << 32 | from_lane((uint32_t)v, lane); }
// (what all lanes have alike, said so: branches on it are the scalar unit's)
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }
__device__ __forceinline__ u64 uniform(u64 v) { return (u64)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v); }
template <typename U>
__device__ __forceinline__ U wave_total(U v) { return from_lane(wave_scan(v), 63); }
