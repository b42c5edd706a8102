// Eight elements of a row, binary32 or bf16, at any element's boundary.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "nm_internal.h"
#include "prune_common.h"        // pack_bf16_rne

namespace nm {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int EW = 8;            // elements of a row that a thread takes at a time: 16 bytes of bf16, 32 of binary32

// EW elements of a row as they are stored, as binary32, and back.  Rows start on any element's boundary, which vector loads and stores here do not mind.  The last
// of a row's threads takes the row's last EW elements, those that its neighbour has too among them, and leaves them alone where it adds (`skip`: how many).
// NARROW: a row has fewer, `left`.
template <int DT> struct Raw;
template <> struct Raw<NM_DT_F32> { u32x4 v[2]; };
template <> struct Raw<NM_DT_BF16> { u32x4 v[1]; };
template <int DT, bool NARROW = false> __device__ __forceinline__ Raw<DT> load_raw(const void *p, int64_t at, int left = EW)
{
    Raw<DT> r;
    if constexpr (DT == NM_DT_F32) {
        typedef u32x4 any __attribute__((aligned(4)));
        const uint32_t *from = (const uint32_t *)p + at;
        if constexpr (!NARROW) { r.v[0] = *(const any *)from; r.v[1] = *(const any *)(from + 4); }
        else
#pragma unroll
            for (int i = 0; i < EW; ++i) r.v[i / 4][i % 4] = i < left ? from[i] : 0u;
    } else {
        typedef u32x4 any __attribute__((aligned(2)));
        const uint16_t *from = (const uint16_t *)p + at;
        if constexpr (!NARROW) r.v[0] = *(const any *)from;
        else
#pragma unroll
            for (int i = 0; i < EW; i += 2) r.v[0][i / 2] = (i < left ? (uint32_t)from[i] : 0u) | (i + 1 < left ? (uint32_t)from[i + 1] << 16 : 0u);
    }
    return r;
}
template <int DT> __device__ __forceinline__ float element(const Raw<DT> &r, int i)
{
    if constexpr (DT == NM_DT_F32) return __uint_as_float(r.v[i / 4][i % 4]);
    else return __uint_as_float(i & 1 ? r.v[0][i / 2] & 0xffff0000u : r.v[0][i / 2] << 16);
}
template <int DT> __device__ __forceinline__ void store_row(void *p, int64_t at, int skip, int left, const float (&v)[EW])
{
    if constexpr (DT == NM_DT_F32) {
        typedef u32x4 any __attribute__((aligned(4)));
        float *to = (float *)p + at;
        if (skip == 0 && left >= EW)
#pragma unroll
            for (int i = 0; i < EW; i += 4) *(any *)(to + i) = u32x4{__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])};
        else
#pragma unroll
            for (int i = 0; i < EW; ++i)
                if (i >= skip && i < left) to[i] = v[i];
    } else {
        typedef u32x4 any __attribute__((aligned(2)));
        uint16_t *to = (uint16_t *)p + at;
        const u32x4 w = {pack_bf16_rne(v[0], v[1]), pack_bf16_rne(v[2], v[3]), pack_bf16_rne(v[4], v[5]), pack_bf16_rne(v[6], v[7])};
        if (skip == 0 && left >= EW) *(any *)to = w;
        else
#pragma unroll
            for (int i = 0; i < EW; ++i)
                if (i >= skip && i < left) to[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
}

}  // namespace

}  // namespace nm
