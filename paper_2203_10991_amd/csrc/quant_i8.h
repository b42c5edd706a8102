// Rounding to 8-bit integers with a scale, shared by the kernels that do it: see quant_i8.hip for the rule.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "nm_internal.h"

namespace nm {

// factor and scale from the bits of the largest magnitude (which order like the magnitudes, with what is not finite on top)
__device__ __forceinline__ void factors(uint32_t top, float &up, float &scale)
{
    const float a = __uint_as_float(top);
    if (top >= 0x7f800000u) { up = 0.f; scale = __uint_as_float(0x7fc00000u); }
    else if (a < 0x1p-110f) { up = 0.f; scale = 0.f; }
    else                    { up = 127.f * (1.f / a); scale = a / 127.f; }
}
__device__ __forceinline__ uint32_t code(float x, float up)
{
    // (a product may pass 127 by a rounding: it still rounds to 127.  Where up is 0 a value that is not finite gives a NaN: code 0)
    return (uint32_t)(int)rintf(up == 0.f ? 0.f : x * up) & 0xffu;
}
__device__ __forceinline__ uint32_t wave_max_u(uint32_t v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return v;
}

// eight consecutive elements as binary32, of which `left` are there (the rest: zeros).  Rows start on any element's boundary, which vector loads do not mind.
typedef unsigned int quad_t __attribute__((ext_vector_type(4)));
template <int DT> __device__ __forceinline__ void load8(const void *p, int64_t at, int64_t left, float (&v)[8])
{
    if constexpr (DT == NM_DT_F32) {
        typedef quad_t any __attribute__((aligned(4)));
        const float *from = (const float *)p + at;
        if (left >= 8) {
            const quad_t a = *(const any *)from, b = *(const any *)(from + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(a[i]); v[4 + i] = __uint_as_float(b[i]); }
        } else if (left > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = from[min((int64_t)i, left - 1)];  // (no branches: all on their way at once)
#pragma unroll
            for (int i = 1; i < 8; ++i) v[i] = i < left ? v[i] : 0.f;
        } else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
    } else {
        typedef quad_t any __attribute__((aligned(2)));
        const uint16_t *from = (const uint16_t *)p + at;
        if (left >= 8) {
            const quad_t a = *(const any *)from;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(i & 1 ? a[i / 2] & 0xffff0000u : a[i / 2] << 16);
        } else if (left > 0) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = from[min((int64_t)i, left - 1)];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < left ? __uint_as_float(w[i] << 16) : 0.f;
        } else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
}

}  // namespace nm
