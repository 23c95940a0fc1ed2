// Numbers of type e4m3 and scales that are powers of two, held as the byte e + 127.
#pragma once
#include <hip/hip_runtime.h>

#include "lsm_pages.h"

namespace lsm {

// 2^e; 0 below 2^-126.
__device__ __forceinline__ float power_of_two(int e) { return e < -126 ? 0.f : __uint_as_float((uint32_t)(e + 127) << 23); }

// The byte of the smallest e from LSM_LEAST_SCALE on with 448 * 2^e >= top, which is finite: 448 = 1.75 * 2^8, so of top = m * 2^x only m > 1.75 matters.
__device__ __forceinline__ uint32_t scale_for(float top) {
    const uint32_t bits = __float_as_uint(top);
    const int x = (int)(bits >> 23), e = x - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);
    return e < LSM_LEAST_SCALE + 127 ? LSM_LEAST_SCALE + 127 : e;
}

template <int E>
struct Codes {
    uint32_t words[E / 4];
};
template <int E>
__device__ __forceinline__ Codes<E> load_codes(const uint8_t* p, bool wide) {
    Codes<E> c;
    if (wide) {
        c = *reinterpret_cast<const Codes<E>*>(__builtin_assume_aligned(p, E));
    } else {
#pragma unroll
        for (int i = 0; i < E / 4; i++) c.words[i] = p[i * 4] | p[i * 4 + 1] << 8 | p[i * 4 + 2] << 16 | (uint32_t)p[i * 4 + 3] << 24;
    }
    return c;
}
template <int E>
__device__ __forceinline__ void store_codes(uint8_t* p, const Codes<E>& c, bool wide) {
    if (wide) {
        *reinterpret_cast<Codes<E>*>(__builtin_assume_aligned(p, E)) = c;
    } else {
#pragma unroll
        for (int i = 0; i < E; i++) p[i] = (uint8_t)(c.words[i / 4] >> (i % 4 * 8));
    }
}
template <int E>
__device__ __forceinline__ void decode(const Codes<E>& c, float (&x)[E]) {
#pragma unroll
    for (int i = 0; i < E / 4; i++) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.words[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.words[i], true);
        x[i * 4] = lo[0], x[i * 4 + 1] = lo[1], x[i * 4 + 2] = hi[0], x[i * 4 + 3] = hi[1];
    }
}
// To nearest, ties to even; magnitudes up to 448, NaN stays NaN.  8 bits is what the cache holds: half a step is 2^-4 of a value.
template <int E>
__device__ __forceinline__ Codes<E> encode(const float (&x)[E]) {
    Codes<E> c;
#pragma unroll
    for (int i = 0; i < E / 4; i++) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[i * 4], x[i * 4 + 1], 0, false);
        c.words[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[i * 4 + 2], x[i * 4 + 3], w, true);
    }
    return c;
}

}  // namespace lsm
