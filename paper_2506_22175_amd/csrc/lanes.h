// Sums and maxima over the lanes of a wavefront without LDS: the vector unit's lane permutations.
#pragma once
#include "common.h"

namespace moe {

// A lane's value of another lane of its 16: 1 and 2 away, mirrored in 8, mirrored in 16 (what is 4 and 8 away once the nearer
// ones agree), or rotated.  All lanes add and compare the same pairs, so that all end with the same bits.
template <int CTRL> __device__ __forceinline__ int from_lane(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
template <int CTRL> __device__ __forceinline__ float from_lane(float v) { return __int_as_float(from_lane<CTRL>(__float_as_int(v))); }
template <int CTRL> __device__ __forceinline__ double from_lane(double v) {
    const long long b = __double_as_longlong(v);
    return __longlong_as_double((long long)from_lane<CTRL>((int)(b >> 32)) << 32 | (unsigned)from_lane<CTRL>((int)b));
}
constexpr int AWAY_1 = 0xB1, AWAY_2 = 0x4E, MIRROR_8 = 0x141, MIRROR_16 = 0x140, ROTATE = 0x120;

// Two rows of 16 lanes, two halves: what both have, in every lane.
struct BothOf { unsigned a, b; };
__device__ __forceinline__ BothOf row_pairs(unsigned v) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return {r[0], r[1]};
}
__device__ __forceinline__ BothOf halves(unsigned v) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return {r[0], r[1]};
}

// over all 64 lanes
__device__ __forceinline__ float wave_sum(float v) {
    v += from_lane<AWAY_1>(v);
    v += from_lane<AWAY_2>(v);
    v += from_lane<MIRROR_8>(v);
    v += from_lane<MIRROR_16>(v);
    BothOf p = row_pairs(__float_as_uint(v));
    v = __uint_as_float(p.a) + __uint_as_float(p.b);
    p = halves(__float_as_uint(v));
    return __uint_as_float(p.a) + __uint_as_float(p.b);
}
__device__ __forceinline__ unsigned larger_bits(unsigned a, unsigned b) { return a > b ? a : b; }
// over the 16 lanes of a row
__device__ __forceinline__ unsigned row_max_bits(unsigned v) {
    v = larger_bits(v, (unsigned)from_lane<AWAY_1>((int)v));
    v = larger_bits(v, (unsigned)from_lane<AWAY_2>((int)v));
    v = larger_bits(v, (unsigned)from_lane<MIRROR_8>((int)v));
    return larger_bits(v, (unsigned)from_lane<MIRROR_16>((int)v));
}
__device__ __forceinline__ unsigned wave_max_bits(unsigned v) {
    v = row_max_bits(v);
    BothOf p = row_pairs(v);
    v = larger_bits(p.a, p.b);
    p = halves(v);
    return larger_bits(p.a, p.b);
}

}  // namespace moe
