// Wide accesses at addresses that are aligned to their elements only (the hardware does them at any address), and the
// element-by-element form for what is left at a row's end.
#pragma once
#include "common.h"

namespace moe {

template <int BYTES, int ALIGN> struct __attribute__((packed, aligned(ALIGN))) Anywhere { unsigned w[BYTES / 4]; };

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
