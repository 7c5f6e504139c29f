// Wide accesses at addresses that are aligned to their elements only (the hardware does them at any address), and the
// element-by-element form for what is left at a row's end.
#pragma once
#include "common.h"

namespace moe {

template <int BYTES, int ALIGN> struct __attribute__((packed, aligned(ALIGN))) Anywhere { unsigned w[BYTES / 4]; };

// 16 bytes that nothing reads again: past the caches' keeping.  (Reading 512 MB and more: 7.0 TB/s so, 6.2 with an ordinary load.)
typedef unsigned wide_u4 __attribute__((ext_vector_type(4)));
template <typename V> __device__ __forceinline__ V load_once(const void* p) {
    static_assert(sizeof(V) == 16, "16 bytes");
    return __builtin_bit_cast(V, __builtin_nontemporal_load(reinterpret_cast<const wide_u4*>(p)));
}
// the same at any multiple of two bytes
typedef unsigned wide_u4_2 __attribute__((ext_vector_type(4), aligned(2)));
template <typename V> __device__ __forceinline__ V load_once_anywhere(const void* p) {
    static_assert(sizeof(V) == 16, "16 bytes");
    return __builtin_bit_cast(V, (wide_u4)__builtin_nontemporal_load(reinterpret_cast<const wide_u4_2*>(p)));
}

template <typename V> __device__ __forceinline__ void store_once_anywhere(void* p, const V& v) {
    static_assert(sizeof(V) == 16, "16 bytes");
    __builtin_nontemporal_store((wide_u4_2)__builtin_bit_cast(wide_u4, v), reinterpret_cast<wide_u4_2*>(p));
}

// four neighbouring columns, `left` of which are in the row
__device__ __forceinline__ void store_columns(float* p, const float* v, int left) {
    if (left >= 4) {
        Anywhere<16, 4> o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.w[i] = __float_as_uint(v[i]);
        *reinterpret_cast<Anywhere<16, 4>*>(p) = o;
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < left) p[i] = v[i];
    }
}
__device__ __forceinline__ void store_columns(bf16_t* p, const float* v, int left) {
    if (left >= 4) {
        Anywhere<8, 2> o;
        o.w[0] = pack_bf16x2(v[0], v[1]);
        o.w[1] = pack_bf16x2(v[2], v[3]);
        *reinterpret_cast<Anywhere<8, 2>*>(p) = o;
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < left) p[i] = f32_to_bf16(v[i]);
    }
}
__device__ __forceinline__ void load_columns(const float* p, float* v, int left) {
    if (left >= 4) {
        const Anywhere<16, 4> o = *reinterpret_cast<const Anywhere<16, 4>*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(o.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < left ? p[i] : 0.0f;
    }
}

}  // namespace moe
