// Rows, or columns, of a matrix as 8-bit integers with a scale each:
//     a = max |x|        q = the integer nearest to x * (127 * (1 / a)), ties to even        scale = a / 127
// (binary32, one rounding an operation).  A row of zeros, and one whose largest magnitude is below 2^-110 (1 / a would overflow), has zero codes and scale
// 0; a row with a value that is not finite has zero codes and a NaN for its scale, so that every product with it is NaN.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "nm_internal.h"
#include "prune_common.h"        // Row

namespace nm {

namespace {

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

// eight consecutive elements as binary32; VEC: on a 16-byte boundary.  Elements from `left` on are zeros
template <int DT, bool VEC> __device__ __forceinline__ void load8(const void *p, int64_t at, int64_t left, float (&v)[8])
{
    if (VEC && left >= 8) {
        if constexpr (DT == NM_DT_F32) {
            const float4 a = *(const float4 *)((const float *)p + at), b = *(const float4 *)((const float *)p + at + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = *(const uint4 *)((const uint16_t *)p + at);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = Row<NM_DT_BF16>::get(a, i);
        }
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.f;
            if (i < left) v[i] = DT == NM_DT_F32 ? ((const float *)p)[at + i] : __uint_as_float((uint32_t)((const uint16_t *)p)[at + i] << 16);
        }
}

// ---- rows: T threads to a row, T * 8 elements at a time; up to KEEP of them stay in registers between the two passes
template <int DT, bool VEC, int T, int KEEP>
__global__ __launch_bounds__(256) void quant_rows_kernel(const void *x, int64_t R, int64_t C, int64_t ld, int8_t *q, int64_t ldq, float *scale)
{
    __shared__ uint32_t tops[256 / T][T / 64];
    const int lane = threadIdx.x % T, mine = threadIdx.x / T;
    const int64_t r = (int64_t)blockIdx.x * (256 / T) + mine;
    const bool there = r < R;
    float v[KEEP][8];
    uint32_t top = 0;
    if (there)
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
            const int64_t c = ((int64_t)k * T + lane) * 8;
            load8<DT, VEC>(x, r * ld + c, C - c, v[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[k][i]) & 0x7fffffffu);
        }
    if (there)
        for (int64_t c = ((int64_t)KEEP * T + lane) * 8; c < C; c += T * 8) {
            float w[8];
            load8<DT, VEC>(x, r * ld + c, C - c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(w[i]) & 0x7fffffffu);
        }
    top = wave_max_u(top);
    if constexpr (T > 64) {
        if (threadIdx.x % 64 == 0) tops[mine][lane / 64] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < T / 64; ++w) top = max(top, tops[mine][w]);
    }
    if (!there) return;
    float up, s;
    factors(top, up, s);
    if (lane == 0) scale[r] = s;
    auto put = [&](int64_t c, const float (&w)[8]) {
        uint32_t word[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) word[i / 4] |= code(w[i], up) << (8 * (i % 4));
        if (c + 8 <= ldq) *(uint2 *)(q + r * ldq + c) = make_uint2(word[0], word[1]);       // (ldq: a multiple of 16)
    };
#pragma unroll
    for (int k = 0; k < KEEP; ++k) put(((int64_t)k * T + lane) * 8, v[k]);
    for (int64_t c = ((int64_t)KEEP * T + lane) * 8; c < ldq; c += T * 8) {
        float w[8];
        load8<DT, VEC>(x, r * ld + c, C - c, w);
        put(c, w);
    }
}

// ---- columns, transposed.  First the largest magnitudes of a slab of rows for eight columns a thread
constexpr int TILE = 64;         // rows and columns of a tile that is turned
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void column_top_kernel(const void *x, int64_t R, int64_t C, int64_t ld, uint32_t *part, int64_t rows_per_slab)
{
    const int64_t c = ((int64_t)blockIdx.x * 32 + threadIdx.x % 32) * 8;
    const int64_t from = (int64_t)blockIdx.y * rows_per_slab, to = min(from + rows_per_slab, R);
    uint32_t top[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c < C)
#pragma unroll 4
        for (int64_t r = from + threadIdx.x / 32; r < to; r += 8) {
            float v[8];
            load8<DT, VEC>(x, r * ld + c, C - c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) top[i] = max(top[i], __float_as_uint(v[i]) & 0x7fffffffu);
        }
    __shared__ uint32_t all[8][32][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) all[threadIdx.x / 32][threadIdx.x % 32][i] = top[i];
    __syncthreads();
    const int col = threadIdx.x;
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, all[w][col / 8][col % 8]);
    const int64_t at = (int64_t)blockIdx.x * 256 + col;
    if (at < C) part[(int64_t)blockIdx.y * C + at] = m;
}
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void quant_turn_kernel(const void *x, int64_t R, int64_t C, int64_t ld, int8_t *q, int64_t ldq, float *scale, const uint32_t *part, int slabs)
{
    __shared__ float ups[TILE];
    __shared__ __attribute__((aligned(16))) uint8_t turned[TILE][TILE + 16];         // [column][row]
    const int tid = threadIdx.x;
    const int64_t r0 = (int64_t)blockIdx.x * TILE, c0 = (int64_t)blockIdx.y * TILE;
    if (tid < TILE && c0 + tid < C) {
        uint32_t top = 0;
        for (int s = 0; s < slabs; ++s) top = max(top, part[(int64_t)s * C + c0 + tid]);
        float up, sc;
        factors(top, up, sc);
        ups[tid] = up;
        if (blockIdx.x == 0) scale[c0 + tid] = sc;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int row = k * 32 + tid / 8, col = tid % 8 * 8;
        float v[8];
        load8<DT, VEC>(x, (r0 + row) * ld + c0 + col, r0 + row < R ? C - c0 - col : 0, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) turned[col + i][row] = c0 + col + i < C ? (uint8_t)code(v[i], ups[col + i]) : 0;
    }
    __syncthreads();
    const int col = tid / 4, row = tid % 4 * 16;
    if (c0 + col < C && r0 + row < ldq) *(uint4 *)(q + (c0 + col) * ldq + r0 + row) = *(const uint4 *)&turned[col][row];
}

}  // namespace

hipError_t launch_quant_i8(int dt, const void *x, int64_t R, int64_t C, int64_t ld, int8_t *q, int64_t ldq, float *scale, hipStream_t st)
{
    if (R == 0) return hipSuccess;
    const int64_t e = dt == NM_DT_F32 ? 4 : 2;
    const bool vec = (uintptr_t)x % 16 == 0 && ld * e % 16 == 0;
#define NM_QUANT_D(DT, T, KEEP)                                                                                                                  \
    do {                                                                                                                                         \
        if (vec) hipLaunchKernelGGL((quant_rows_kernel<DT, true, T, KEEP>), dim3((unsigned)wgs), dim3(256), 0, st, x, R, C, ld, q, ldq, scale);  \
        else hipLaunchKernelGGL((quant_rows_kernel<DT, false, T, KEEP>), dim3((unsigned)wgs), dim3(256), 0, st, x, R, C, ld, q, ldq, scale);     \
    } while (0)
#define NM_QUANT(T, KEEP)                                                                       \
    do {                                                                                        \
        const int64_t wgs = (R + 256 / T - 1) / (256 / T);                                      \
        if (wgs > 0x7fffffff) return hipErrorInvalidConfiguration;                              \
        if (dt == NM_DT_F32) NM_QUANT_D(NM_DT_F32, T, KEEP); else NM_QUANT_D(NM_DT_BF16, T, KEEP); \
    } while (0)
    if (C <= 512) NM_QUANT(64, 1);
    else if (C <= 1024) NM_QUANT(64, 2);
    else if (C <= 4096) NM_QUANT(256, 2);
    else NM_QUANT(256, 4);
#undef NM_QUANT
#undef NM_QUANT_D
    return hipGetLastError();
}

int quant_i8_slabs(int64_t R, int64_t C)
{
    // slabs of at least 64 rows, about four workgroups to a CU
    const int64_t panels = (C + 255) / 256;
    return (int)std::max<int64_t>(1, std::min<int64_t>({(R + 63) / 64, 1024 / std::max<int64_t>(panels, 1), 64}));
}

hipError_t launch_quant_i8_t(int dt, const void *x, int64_t R, int64_t C, int64_t ld, int8_t *q, int64_t ldq, float *scale, uint32_t *part, hipStream_t st)
{
    if (C == 0) return hipSuccess;
    const int64_t e = dt == NM_DT_F32 ? 4 : 2;
    const bool vec = (uintptr_t)x % 16 == 0 && ld * e % 16 == 0;
    const int slabs = quant_i8_slabs(R, C);
    const int64_t per = (R + slabs - 1) / slabs, panels = (C + 255) / 256, tr = std::max<int64_t>((ldq + TILE - 1) / TILE, 1), tc = (C + TILE - 1) / TILE;
    if (panels > 0x7fffffff || tr > 0x7fffffff || tc > 65535) return hipErrorInvalidConfiguration;
#define NM_TURN(DT, VEC)                                                                                                                             \
    do {                                                                                                                                             \
        hipLaunchKernelGGL((column_top_kernel<DT, VEC>), dim3((unsigned)panels, (unsigned)slabs), dim3(256), 0, st, x, R, C, ld, part, per);         \
        hipLaunchKernelGGL((quant_turn_kernel<DT, VEC>), dim3((unsigned)tr, (unsigned)tc), dim3(256), 0, st, x, R, C, ld, q, ldq, scale, part, slabs); \
    } while (0)
    if (dt == NM_DT_F32) { if (vec) NM_TURN(NM_DT_F32, true); else NM_TURN(NM_DT_F32, false); }
    else                 { if (vec) NM_TURN(NM_DT_BF16, true); else NM_TURN(NM_DT_BF16, false); }
#undef NM_TURN
    return hipGetLastError();
}

}  // namespace nm
