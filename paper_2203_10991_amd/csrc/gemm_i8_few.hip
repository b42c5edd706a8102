// The 8-bit integer product (gemm_i8.hip) for few tokens, where the weights' one way from memory is what it takes.
//
// Instruction: v_mfma_i32_16x16x64_i8, both operands with 16 rows (lane % 16) and 16 bytes of the reduction axis to a lane; which ones does not matter, since both
// hold the same.  A workgroup takes 16 or 32 features and 16 or 32 tokens, its four waves a quarter of the reduction axis each, straight from memory into registers
// in groups of 256 bytes of a row, the next groups on their way while one is multiplied.  The quarters meet in LDS.
// What bounds a CU here is its address path: the four lanes of a quad in one 64-byte piece take one cycle, in four rows, as the instruction has its lanes, four.  So
// the quads load whole pieces (four loads of a group: four rows each, 256 bytes of a row) and turn 4 x 4 blocks of 16 bytes among their lanes then, 32 moves
// a group: 16 tokens x 28672 -> 8192 43 us with the instruction's own layout, 36 with the turn (6.6 TB/s), 16 x 8192 -> 2048 10.2 and 6.9, 64 x 8192 -> 1024
// 13.6 and 7.8.  Eight waves to a workgroup instead of four: 35 to 38 us, 7.0 and 8.4.
// x: codes from memory (L2), or (FUSED, up to 4 tokens) the tokens themselves, which each workgroup rounds into LDS while its first weights are on
// their way: that saves the launch.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "nm_internal.h"
#include "gemm_plan.h"           // NM_CUS
#include "quant_i8.h"            // load8, factors, code
#include "smfmac_common.h"       // vector types
#include "prune_common.h"        // pack_bf16_rne

namespace nm {

namespace {

constexpr int FEW_LDS = 16384;   // bytes of codes that a FUSED workgroup holds
constexpr int NW = 4, WG = 64 * NW;
constexpr int GROUP = 256;       // bytes of the reduction axis to four instructions

// v[j] of lane 4 i + m is then what v[m] of lane 4 i + j was
__device__ __forceinline__ void turn(i32x4 (&v)[4], int lane)
{
    const bool one = lane & 1, two = lane & 2;
#pragma unroll
    for (int p = 0; p < 4; p += 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int a = v[p][i], b = v[p + 1][i];
            const int from_a = __builtin_amdgcn_mov_dpp(a, 0xb1, 0xf, 0xf, true), from_b = __builtin_amdgcn_mov_dpp(b, 0xb1, 0xf, 0xf, true);       // of lane ^ 1
            v[p][i] = one ? from_b : a;
            v[p + 1][i] = one ? b : from_a;
        }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int a = v[p][i], b = v[p + 2][i];
            const int from_a = __builtin_amdgcn_mov_dpp(a, 0x4e, 0xf, 0xf, true), from_b = __builtin_amdgcn_mov_dpp(b, 0x4e, 0xf, 0xf, true);       // of lane ^ 2
            v[p][i] = two ? from_b : a;
            v[p + 2][i] = two ? b : from_a;
        }
}

struct FewArg {
    I8Arg a;
    const void *raw;             // FUSED: the tokens, row stride ldraw in elements
    int64_t ldraw;
    int raw_dt, groups;          // of a wave
};

// TT: blocks of 16 tokens; FT: blocks of 16 features
template <int TT, int FT, bool FUSED>
__global__ __launch_bounds__(WG) void gemm_i8_few_kernel(FewArg p)
{
    constexpr int G = FT == 1 ? 2 : 1, F = 16 * FT;                              // G: groups of a wave that are on their way
    __shared__ int sums[NW / 2][TT][16][F + 4];                                       // [wave][..][token][feature], rows padded against bank conflicts
    __shared__ uint32_t tops[NW];
    __shared__ float row_scale[4];
    extern __shared__ __attribute__((aligned(16))) char codes[];                 // FUSED: [token][row]
    const I8Arg &a = p.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, q = lane >> 4;
    const int64_t f0 = (int64_t)blockIdx.x * F, t0 = (int64_t)blockIdx.y * 16 * TT;
    const int K = (int)a.K, k_first = wave * p.groups * GROUP, row = (K + 63) / 64 * 64 + 16;        // FUSED: bytes of a token's row in LDS
    const int k_end = (K + 15) / 16 * 16;                                        // a row can be read up to here; past it its last chunk again: x has zeros there
    const int r_load = l16 & ~3, k_load = 64 * q + 16 * (lane & 3);              // load u of a group: row r_load + u, from k_load on
    const char *wp = (const char *)(a.w + f0 * a.ldw), *xp = (const char *)(a.x + t0 * a.ldx);
    uint32_t w_row[FT][4];
#pragma unroll
    for (int ft = 0; ft < FT; ++ft)
#pragma unroll
        for (int u = 0; u < 4; ++u) w_row[ft][u] = (uint32_t)min((int64_t)(16 * ft + r_load + u), a.N - 1 - f0) * (uint32_t)a.ldw;
    auto w_group = [&](int ft, int k, i32x4 (&v)[4]) {
        const uint32_t at = (uint32_t)min(k + k_load, k_end - 16);
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = *(const i32x4 *)(wp + (w_row[ft][u] + at));
    };
    i32x4 wv[FT][G][4];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) w_group(ft, k_first + GROUP * g, wv[ft][g]);
    // scales and bias of the results a thread will store, ahead of time: feature tid % F of the tokens tid / F + o * WG / F
    constexpr int OUT = TT * 16 * F / WG;
    const int64_t my_f = min(f0 + tid % F, a.N - 1);
    const float my_ws = a.ws[my_f];
    uint32_t my_add = 0;
    if (a.bias) my_add = a.bias_dt == NM_DT_F32 ? ((const uint32_t *)a.bias)[my_f] : ((const uint16_t *)a.bias)[my_f];
    float my_xs[OUT];
    if constexpr (!FUSED)
#pragma unroll
        for (int o = 0; o < OUT; ++o) my_xs[o] = a.xs[min(t0 + tid / F + o * (WG / F), a.M - 1)];
    if constexpr (FUSED) {
        for (int t = 0; t < (int)a.M; ++t) {
            auto take = [&](int c, float (&v)[8]) {
                if (p.raw_dt == NM_DT_F32) load8<NM_DT_F32>(p.raw, t * p.ldraw + c, K - c, v); else load8<NM_DT_BF16>(p.raw, t * p.ldraw + c, K - c, v);
            };
            constexpr int KEEP = 2;
            float keep[KEEP][8];
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < KEEP; ++k) {
                take((k * WG + tid) * 8, keep[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(keep[k][i]) & 0x7fffffffu);
            }
            for (int c = (KEEP * WG + tid) * 8; c < K; c += WG * 8) {
                float v[8];
                take(c, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
            }
            top = wave_max_u(top);
            __syncthreads();                                                     // (the token before is done with tops)
            if (lane == 0) tops[wave] = top;
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NW; ++v) top = max(top, tops[v]);
            float up, s;
            factors(top, up, s);
            if (tid == 0) row_scale[t] = s;
            auto put = [&](int c, const float (&v)[8]) {
                uint32_t word[2] = {0, 0};
#pragma unroll
                for (int i = 0; i < 8; ++i) word[i / 4] |= code(v[i], up) << (8 * (i % 4));
                if (c + 8 <= row) *(uint2 *)(codes + t * row + c) = make_uint2(word[0], word[1]);
            };
#pragma unroll
            for (int k = 0; k < KEEP; ++k) put((k * WG + tid) * 8, keep[k]);
            for (int c = (KEEP * WG + tid) * 8; c < row; c += WG * 8) {
                float v[8];
                take(c, v);
                put(c, v);
            }
        }
        __syncthreads();
    }
    uint32_t x_row[TT][4];
    if constexpr (!FUSED)                                                        // (tokens past the end: the last one's again, not stored)
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int u = 0; u < 4; ++u) x_row[tt][u] = (uint32_t)min((int64_t)(16 * tt + r_load + u), a.M - 1 - t0) * (uint32_t)a.ldx;
    auto x_group = [&](int tt, int k, i32x4 (&v)[4]) {
        if constexpr (FUSED) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = k + 64 * q + 16 * j;
                v[j] = l16 < (int)a.M && at < row ? *(const i32x4 *)(codes + l16 * row + at) : i32x4{0, 0, 0, 0};
            }
        } else {
            const uint32_t at = (uint32_t)min(k + k_load, k_end - 16);
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = *(const i32x4 *)(xp + (x_row[tt][u] + at));
        }
    };
    auto x_turn = [&](int k, i32x4 (&v)[4]) {
        if constexpr (FUSED) return;
        turn(v, lane);
        if (k + GROUP > K)                                                       // zeros behind the axis
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int left = K - (k + 64 * q + 16 * j);                      // bytes of the chunk that count
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j][i] &= left >= 4 * i + 4 ? -1 : left <= 4 * i ? 0 : (int)((1u << (8 * (left - 4 * i))) - 1u);
            }
    };
    i32x4 acc[TT][FT];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) acc[tt][ft] = i32x4{0, 0, 0, 0};
    i32x4 xv[TT][G][4];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) x_group(tt, k_first + GROUP * g, xv[tt][g]);
    auto round = [&](int s, auto more_c) {                                       // the groups s .. s + G - 1, and the loads of the next ones if there are any
        constexpr bool more = decltype(more_c)::value;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int k = k_first + GROUP * (s + g);
            i32x4 x_now[TT][4];
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) {
#pragma unroll
                for (int j = 0; j < 4; ++j) x_now[tt][j] = xv[tt][g][j];
                if constexpr (more) x_group(tt, k + GROUP * G, xv[tt][g]);
                x_turn(k, x_now[tt]);
            }
#pragma unroll
            for (int ft = 0; ft < FT; ++ft) {
                i32x4 w_now[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w_now[j] = wv[ft][g][j];
                if constexpr (more) w_group(ft, k + GROUP * G, wv[ft][g]);
                turn(w_now, lane);
                if (g == 0 || s + g < p.groups)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int tt = 0; tt < TT; ++tt) acc[tt][ft] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w_now[j], x_now[tt][j], acc[tt][ft], 0, 0, 0);
            }
        }
    };
    int s = 0;
    for (; s + G < p.groups; s += G) round(s, std::true_type{});
    round(s, std::false_type{});
    // a lane holds the features 4 q .. + 3 of token l16.  Half of the waves hand their sums to the others, whose own then meet
    if (wave >= NW / 2)
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int ft = 0; ft < FT; ++ft) *(i32x4 *)&sums[wave - NW / 2][tt][l16][16 * ft + 4 * q] = acc[tt][ft];
    __syncthreads();
    if (wave < NW / 2)
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int ft = 0; ft < FT; ++ft) {
                i32x4 *const at = (i32x4 *)&sums[wave][tt][l16][16 * ft + 4 * q];
                *at += acc[tt][ft];
            }
    __syncthreads();
    if (f0 + tid % F >= a.N) return;
    const float add = a.bias_dt == NM_DT_F32 ? __uint_as_float(my_add) : __uint_as_float(my_add << 16);
#pragma unroll
    for (int o = 0; o < OUT; ++o) {
        const int token = tid / F + o * (WG / F), f = tid % F;
        if (t0 + token >= a.M) break;
        int sum = 0;
#pragma unroll
        for (int v = 0; v < NW / 2; ++v) sum += sums[v][token / 16][token % 16][f];
        const float xs = FUSED ? row_scale[token] : my_xs[o];
        float v = (float)sum * (xs * my_ws) + add;
        if (a.relu) v = v <= 0.f ? 0.f : v;                                      // (a NaN stays one)
        const int64_t at = (t0 + token) * a.ldy + f0 + f;
        if (a.y_dt == NM_DT_F32) ((float *)a.y)[at] = v; else ((uint16_t *)a.y)[at] = (uint16_t)pack_bf16_rne(v, v);
    }
}

}  // namespace

// The forms, and a model of their times: a line in the groups of a wave, and what each further workgroup of a CU adds to it (in us).  Fitted to 260 products of 5 to
// 2048 tokens, 64 to 28672 features and 64 to 28672 inputs; the launch takes the form or the tile (gemm_i8.hip) with the least, which over these products is 2.4 %
// from the best of twelve forms and the five tiles.  (us, 1 x 1 blocks / 1 x 2 / 2 x 2 / best tile: 16 x 1024 -> 16384 8.0 / 6.1 / - / 8.0, 16 x 4096 -> 4096 6.1 / 7.2 / -
// / 15.0, 64 x 4096 -> 1024 5.1 / 6.3 / 7.8 / 14.8, 128 x 4096 -> 4096 17.0 / 13.0 / 10.9 / 15.3, 512 x 4096 -> 1024 15.9 / 12.7 / 10.5 / 15.1, 32 x 28672 -> 8192
// 67 / 53 / 37.7 / 73, 64 x 4096 -> 12288 30.1 / 22.6 / 16.4 / 15.7, 1024 x 4096 -> 1024 28.9 / 21.7 / 17.7 / 15.5.)
I8FewPlan gemm_i8_few_plan(int64_t M, int64_t N, int64_t K)
{
    constexpr I8FewPlan forms[3] = {{1, 1, 0.}, {1, 2, 0.}, {2, 2, 0.}};
    constexpr double fit[3][4] = {{3.8, 0.53, 0.52, 0.56}, {3.2, 0.87, 0., 0.96}, {4.4, 1.12, 0.34, 1.22}};
    const double groups = (double)((K + GROUP * NW - 1) / (GROUP * NW));
    I8FewPlan best{0, 0, 1e300};
    for (int i = 0; i < 3; ++i) {
        const int64_t blocks = (M + 16 * forms[i].tt - 1) / (16 * forms[i].tt);
        if (blocks > 65535 || (forms[i].tt > 1 && M <= 16)) continue;
        const double wgs = (double)((N + 16 * forms[i].ft - 1) / (16 * forms[i].ft)) * (double)blocks, more = std::max(wgs / NM_CUS - 1., 0.);
        const double us = fit[i][0] + fit[i][1] * groups + more * (fit[i][2] + fit[i][3] * groups);
        if (us < best.us) { best = forms[i]; best.us = us; }
    }
    return best;
}
bool gemm_i8_few_fused(int64_t M, int64_t K) { return M <= 4 && M * ((K + 63) / 64 * 64 + 16) <= FEW_LDS; }

hipError_t launch_gemm_i8_few(const I8Arg &a, const void *raw, int64_t ldraw, int raw_dt, hipStream_t st)
{
    if (a.M == 0 || a.N == 0) return hipSuccess;
    const I8FewPlan plan = gemm_i8_few_plan(a.M, a.N, a.K);
    const int64_t wgs = (a.N + 16 * plan.ft - 1) / (16 * plan.ft), blocks = (a.M + 16 * plan.tt - 1) / (16 * plan.tt);
    const FewArg p{a, raw, ldraw, raw_dt, (int)((a.K + GROUP * NW - 1) / (GROUP * NW))};
    const size_t lds = raw ? (size_t)(a.M * ((a.K + 63) / 64 * 64 + 16)) : 0;
#define NM_FEW(TT, FT, FUSED) hipLaunchKernelGGL((gemm_i8_few_kernel<TT, FT, FUSED>), dim3((unsigned)wgs, (unsigned)blocks), dim3(WG), lds, st, p)
    if (raw) { if (plan.ft == 1) NM_FEW(1, 1, true); else NM_FEW(1, 2, true); }
    else if (plan.tt == 2) NM_FEW(2, 2, false);
    else if (plan.ft == 2) NM_FEW(1, 2, false);
    else NM_FEW(1, 1, false);
#undef NM_FEW
    return hipGetLastError();
}

}  // namespace nm
