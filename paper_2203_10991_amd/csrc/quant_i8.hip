// Rows, or columns, of a matrix as 8-bit integers with a scale each:
//     a = max |x|        q = the integer nearest to x * (127 * (1 / a)), ties to even        scale = a / 127
// (binary32, one rounding an operation).  A row of zeros, and one whose largest magnitude is below 2^-110 (1 / a would overflow), has zero codes and scale
// 0; a row with a value that is not finite has zero codes and a NaN for its scale, so that every product with it is NaN.
// Bound: HBM; rows are read once (they stay in registers up to 8192 columns), columns twice.  Rows of bf16, us: 32768 x 8192 145 (805 MB, 5.6 TB/s), 16384 x 4096 37,
// 16384 x 1024 13.5, 4096 x 1024 6.0; columns, tops and turn: 28672 x 8192 243 (1.17 GB from and to memory, 4.8 TB/s), 4096 x 1024 9.0 back to back, 15 from memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "nm_internal.h"
#include "grid_row.h"
#include "quant_i8.h"

namespace nm {

namespace {

// ---- rows: T threads to a row, T * 8 elements at a time; up to KEEP of them stay in registers between the two passes.  A wave to a row up to 1024
// columns, which needs no barrier; the workgroup to a row beyond, where a wave would hold 32 elements a lane and more.
constexpr int ROWS_WG = 256;
template <int DT, int T, int KEEP>
__global__ __launch_bounds__(ROWS_WG) void quant_rows_kernel(const void *x, int64_t R, int64_t C, int64_t ld, int8_t *q, int64_t ldq, float *scale)
{
    __shared__ uint32_t tops[ROWS_WG / T][T / 64];
    const int lane = threadIdx.x % T, mine = threadIdx.x / T;
    const int64_t r = (int64_t)grid_place(blockIdx.x, blockIdx.y) * (ROWS_WG / T) + mine;
    const bool there = r < R;
    float v[KEEP][8];
    uint32_t top = 0;
    if (there)
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
            const int64_t c = ((int64_t)k * T + lane) * 8;
            load8<DT>(x, r * ld + c, C - c, v[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[k][i]) & 0x7fffffffu);
        }
    if (there)
        for (int64_t c = ((int64_t)KEEP * T + lane) * 8; c < C; c += T * 8) {
            float w[8];
            load8<DT>(x, r * ld + c, C - c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(w[i]) & 0x7fffffffu);
        }
    top = wave_max_u(top);
    if constexpr (T > 64) {
        if (lane % 64 == 0) tops[mine][lane / 64] = top;
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
        load8<DT>(x, r * ld + c, C - c, w);
        put(c, w);
    }
}

// ---- columns, transposed.  First the largest magnitudes of a slab of rows for 64 columns, eight threads side by side to a row
constexpr int TILE = 64;         // rows and columns of a tile that is turned
template <int DT>
__global__ __launch_bounds__(256) void column_top_kernel(const void *x, int64_t R, int64_t C, int64_t ld, uint32_t *part, int64_t rows_per_slab)
{
    constexpr int H = 256 / 8;
    const int across = threadIdx.x % 8, down = threadIdx.x / 8;
    const int64_t c0 = (int64_t)blockIdx.x * TILE, c = c0 + across * 8;
    const int64_t from = (int64_t)blockIdx.y * rows_per_slab, to = min(from + rows_per_slab, R);
    uint32_t top[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c < C)
#pragma unroll 4
        for (int64_t r = from + down; r < to; r += H) {
            float v[8];
            load8<DT>(x, r * ld + c, C - c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) top[i] = max(top[i], __float_as_uint(v[i]) & 0x7fffffffu);
        }
    __shared__ uint32_t all[H][TILE];
#pragma unroll
    for (int i = 0; i < 8; ++i) all[down][across * 8 + i] = top[i];
    __syncthreads();
    const int col = threadIdx.x;
    if (col >= TILE || c0 + col >= C) return;
    uint32_t m = 0;
#pragma unroll
    for (int h = 0; h < H; ++h) m = max(m, all[h][col]);
    part[(int64_t)blockIdx.y * C + c0 + col] = m;
}
// Then tiles of 64 x 64, turned through LDS in blocks of four columns by four rows: a thread packs four rows of a column into a word.  In order, `side` tiles side by
// side, then the rows below: 32 where rows are whole lines of 128 bytes apart, so that no two tiles read one line, otherwise 1.  (us, both kernels, 32 / 1: 4096 x
// 1024 bf16 9.0 / 12.0, 28672 x 8192 bf16 243 / 279, binary32 408 / 485, 7168 x 7680 binary32 77 / 77, 7064 x 7510 binary32 102 / 91.)
template <int DT>
__global__ __launch_bounds__(256) void quant_turn_kernel(const void *x, int64_t R, int64_t C, int64_t ld, int8_t *q, int64_t ldq, float *scale, const uint32_t *part, int slabs,
                                                         int tiles_r, int tiles_c, int side)
{
    __shared__ uint32_t tops[4][TILE];
    __shared__ float ups[TILE];
    __shared__ uint32_t turned[TILE][TILE / 4 + 1];                                  // [column][four rows]
    const int tid = threadIdx.x;
    const uint32_t first = blockIdx.y * (uint32_t)side, wide = min((uint32_t)side, (uint32_t)tiles_c - first), down = blockIdx.x / wide;
    if (down >= (uint32_t)tiles_r) return;
    const int64_t r0 = (int64_t)down * TILE, c0 = (int64_t)(first + blockIdx.x - down * wide) * TILE;
    // eight columns of rows 4 k .. 4 k + 3, on their way while the slabs' tops are compared
    const int k = tid / 8 % 16, col = tid % 8 * 8, half = tid / 128;                 // (a thread loads two of the four rows, and gets the others from its partner)
    float v[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = 4 * k + 2 * half + i;
        load8<DT>(x, (r0 + row) * ld + c0 + col, r0 + row < R ? C - c0 - col : 0, v[i]);
    }
    uint32_t top = 0;
    if (c0 + tid % TILE < C)
        for (int s = tid / TILE; s < slabs; s += 4) top = max(top, part[(int64_t)s * C + c0 + tid % TILE]);
    tops[tid / TILE][tid % TILE] = top;
    __syncthreads();
    if (tid < TILE) {
        float up, sc;
        factors(max(max(tops[0][tid], tops[1][tid]), max(tops[2][tid], tops[3][tid])), up, sc);
        ups[tid] = up;
        if (r0 == 0 && c0 + tid < C) scale[c0 + tid] = sc;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float up = ups[col + i];
        ((uint16_t *)&turned[col + i][k])[half] = (uint16_t)(code(v[0][i], up) | code(v[1][i], up) << 8);
    }
    __syncthreads();
    const int out = tid / 4, word = tid % 4 * 4;
    if (c0 + out < C && r0 + 4 * word < ldq)
        *(uint4 *)(q + (c0 + out) * ldq + r0 + 4 * word) = make_uint4(turned[out][word], turned[out][word + 1], turned[out][word + 2], turned[out][word + 3]);
}

}  // namespace

hipError_t launch_quant_i8(int dt, const void *x, int64_t R, int64_t C, int64_t ld, int8_t *q, int64_t ldq, float *scale, hipStream_t st)
{
    if (R == 0) return hipSuccess;
#define NM_QUANT_D(DT, T, KEEP) hipLaunchKernelGGL((quant_rows_kernel<DT, T, KEEP>), dim3(grid_row(wgs), grid_rows(wgs)), dim3(ROWS_WG), 0, st, x, R, C, ld, q, ldq, scale)
#define NM_QUANT(T, KEEP)                                                                       \
    do {                                                                                        \
        const int64_t wgs = (R + ROWS_WG / T - 1) / (ROWS_WG / T);                        \
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
    const int64_t panels = (C + TILE - 1) / TILE;
    return (int)std::max<int64_t>(1, std::min<int64_t>({(R + 63) / 64, 1024 / std::max<int64_t>(panels, 1), 64}));
}

hipError_t launch_quant_i8_t(int dt, const void *x, int64_t R, int64_t C, int64_t ld, int8_t *q, int64_t ldq, float *scale, uint32_t *part, hipStream_t st)
{
    if (C == 0) return hipSuccess;
    const int slabs = quant_i8_slabs(R, C);
    const int64_t per = (R + slabs - 1) / slabs, tr = std::max<int64_t>((ldq + TILE - 1) / TILE, 1), tc = (C + TILE - 1) / TILE;
    const int side = ld * (dt == NM_DT_F32 ? 4 : 2) % 128 == 0 && tr < 65536 ? (int)std::min<int64_t>(tc, 32) : 1;
    if (tr > 0xffffff || tc > 65535) return hipErrorInvalidConfiguration;
#define NM_TURN(DT)                                                                                                                              \
    do {                                                                                                                                         \
        hipLaunchKernelGGL((column_top_kernel<DT>), dim3((unsigned)tc, (unsigned)slabs), dim3(256), 0, st, x, R, C, ld, part, per);              \
        hipLaunchKernelGGL((quant_turn_kernel<DT>), dim3((unsigned)(tr * side), (unsigned)((tc + side - 1) / side)), dim3(256), 0, st, x, R, C, ld, q, ldq, scale, part, slabs, (int)tr, (int)tc, side); \
    } while (0)
    if (dt == NM_DT_F32) NM_TURN(NM_DT_F32); else NM_TURN(NM_DT_BF16);
#undef NM_TURN
    return hipGetLastError();
}

}  // namespace nm
