// The 8-bit integer product (gemm_i8.hip) for few tokens, where the weights' one way from memory is what it takes.
//
// Instruction: v_mfma_i32_16x16x64_i8, both operands with 16 rows (lane % 16) and 16 consecutive bytes of the reduction axis to a lane (16 * (lane / 16) on).
// A workgroup takes 16 or 32 features, its four waves a quarter of the reduction axis each, straight from memory into registers: 28672 x 8192 are 1792 workgroups
// that are all on the chip at once with U loads of 1 KB from each wave on their way.  The quarters meet in LDS.
// x: codes from memory (L2), or (FUSED, up to 4 tokens) the tokens themselves, which each workgroup rounds into LDS while its first weights are on
// their way: that saves the launch.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "nm_internal.h"
#include "gemm_plan.h"           // NM_CUS
#include "quant_i8.h"            // load8, factors, code
#include "smfmac_common.h"       // vector types
#include "prune_common.h"        // pack_bf16_rne

namespace nm {

namespace {

constexpr int FEW_LDS = 16384;   // bytes of codes that a FUSED workgroup holds

struct FewArg {
    I8Arg a;
    const void *raw;             // FUSED: the tokens, row stride ldraw in elements
    int64_t ldraw;
    int raw_dt, steps;           // steps of 64 bytes of a wave
};

// TT: blocks of 16 tokens; FT: blocks of 16 features
template <int TT, int FT, bool FUSED>
__global__ __launch_bounds__(256) void gemm_i8_few_kernel(FewArg p)
{
    constexpr int U = FT == 1 ? 8 : 4, F = 16 * FT;
    __shared__ int sums[4][TT][16][F + 4];                                       // [wave][..][token][feature], rows padded against bank conflicts
    __shared__ uint32_t tops[4];
    __shared__ float row_scale[4];
    extern __shared__ __attribute__((aligned(16))) char codes[];                 // FUSED: [token][row]
    const I8Arg &a = p.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, q = lane >> 4;
    const int64_t f0 = (int64_t)blockIdx.x * F, t0 = (int64_t)blockIdx.y * 16 * TT;
    const int K = (int)a.K, k_first = wave * p.steps * 64 + 16 * q, row = (K + 63) / 64 * 64 + 16;        // FUSED: bytes of a token's row in LDS
    const int8_t *w[FT];
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) w[ft] = a.w + min(f0 + 16 * ft + l16, a.N - 1) * a.ldw;
    const int k_end = (K + 15) / 16 * 16;                                        // a row of w can be read up to here
    // (past the end of the axis the row's last chunk again: x has zeros there)
    auto w_at = [&](int ft, int k) { return *(const i32x4 *)(w[ft] + min(k, k_end - 16)); };
    i32x4 wv[FT][U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) wv[ft][u] = w_at(ft, k_first + 64 * u);
    if constexpr (FUSED) {
        for (int t = 0; t < (int)a.M; ++t) {
            auto take = [&](int c, float (&v)[8]) {
                if (p.raw_dt == NM_DT_F32) load8<NM_DT_F32>(p.raw, t * p.ldraw + c, K - c, v); else load8<NM_DT_BF16>(p.raw, t * p.ldraw + c, K - c, v);
            };
            float keep[2][8];
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                take((k * 256 + tid) * 8, keep[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(keep[k][i]) & 0x7fffffffu);
            }
            for (int c = (512 + tid) * 8; c < K; c += 2048) {
                float v[8];
                take(c, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
            }
            top = wave_max_u(top);
            __syncthreads();                                                     // (the token before is done with tops)
            if (lane == 0) tops[wave] = top;
            __syncthreads();
            top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
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
            for (int k = 0; k < 2; ++k) put((k * 256 + tid) * 8, keep[k]);
            for (int c = (512 + tid) * 8; c < row; c += 2048) {
                float v[8];
                take(c, v);
                put(c, v);
            }
        }
        __syncthreads();
    }
    auto x_at = [&](int tt, int k) {
        const i32x4 zero = {0, 0, 0, 0};
        if constexpr (FUSED) return l16 < (int)a.M && k < row ? *(const i32x4 *)(codes + l16 * row + k) : zero;
        else {
            const int64_t t = min(t0 + 16 * tt + l16, a.M - 1);            // (tokens past the end: the last one's again, not stored)
            i32x4 v = *(const i32x4 *)(a.x + t * a.ldx + min(k, k_end - 16));
            const int left = K - k;                                              // bytes of the chunk that count
            if (left < 16)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] &= left >= 4 * j + 4 ? -1 : left <= 4 * j ? 0 : (int)((1u << (8 * (left - 4 * j))) - 1u);
            return v;
        }
    };
    i32x4 acc[TT][FT];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) acc[tt][ft] = i32x4{0, 0, 0, 0};
    for (int s = 0; s < p.steps; s += U) {
        i32x4 xv[TT][U];
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int u = 0; u < U; ++u) xv[tt][u] = s + u < p.steps ? x_at(tt, k_first + 64 * (s + u)) : i32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int ft = 0; ft < FT; ++ft) {
                const i32x4 now = wv[ft][u];
                wv[ft][u] = w_at(ft, k_first + 64 * (s + U + u));                // (behind the last step: the row's last chunk, which is not used)
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) acc[tt][ft] = __builtin_amdgcn_mfma_i32_16x16x64_i8(now, xv[tt][u], acc[tt][ft], 0, 0, 0);
            }
    }
    // a lane holds the features 4 q .. + 3 of token l16
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) *(i32x4 *)&sums[wave][tt][l16][16 * ft + 4 * q] = acc[tt][ft];
    __syncthreads();
    const int tokens = (int)min(a.M - t0, (int64_t)(16 * TT));
    for (int i = tid; i < TT * 16 * F; i += 256) {
        const int tt = i / (16 * F), t = i / F % 16, f = i % F;
        if (16 * tt + t >= tokens || f0 + f >= a.N) continue;
        const int sum = sums[0][tt][t][f] + sums[1][tt][t][f] + sums[2][tt][t][f] + sums[3][tt][t][f];
        const float xs = FUSED ? row_scale[t] : a.xs[t0 + 16 * tt + t];
        float v = (float)sum * (xs * a.ws[f0 + f]);
        if (a.bias) v += a.bias_dt == NM_DT_F32 ? ((const float *)a.bias)[f0 + f] : __uint_as_float((uint32_t)((const uint16_t *)a.bias)[f0 + f] << 16);
        if (a.relu) v = v <= 0.f ? 0.f : v;                                      // (a NaN stays one)
        const int64_t at = (t0 + 16 * tt + t) * a.ldy + f0 + f;
        if (a.y_dt == NM_DT_F32) ((float *)a.y)[at] = v; else ((uint16_t *)a.y)[at] = (uint16_t)pack_bf16_rne(v, v);
    }
}

}  // namespace

// Where this way is the faster one: its workgroups run through the whole reduction axis, 1.3 ns a byte (tiles: 2.3, behind barriers), so where they all have a CU of
// their own; and for up to 32 tokens where the weights are what takes the time, unless the tiles fill the chip and read x once for 64 features (us, this
// way / tiles: 1 x 1024 -> 4096 3.8 / 7.0, 16 x 8192 -> 2048 11.7 / 23.6, 16 x 28672 -> 8192 47.7 / 74.7, 16 x 8192 -> 28672 53.0 / 46.8, 64 x 8192 -> 1024
// 15.1 / 23.9, 64 x 1024 -> 4096 5.6 / 7.1, 96 x 1024 -> 4096 7.5 / 7.2, 512 x 8192 -> 256 15.7 / 23.6).
bool gemm_i8_few_takes(int64_t M, int64_t N)
{
    const int64_t blocks = (M + 31) / 32;
    return (N + 31) / 32 * blocks <= NM_CUS || (M <= I8_FEW && (M <= 8 || N < 16384));
}
bool gemm_i8_few_fused(int64_t M, int64_t K) { return M <= 4 && M * ((K + 63) / 64 * 64 + 16) <= FEW_LDS; }

hipError_t launch_gemm_i8_few(const I8Arg &a, const void *raw, int64_t ldraw, int raw_dt, hipStream_t st)
{
    const int64_t wgs = (a.N + 15) / 16, pairs = (a.N + 31) / 32, blocks = (a.M + 31) / 32;
    if (a.M == 0 || a.N == 0) return hipSuccess;
    if (wgs > 0x7fffffff || blocks > 65535) return hipErrorInvalidConfiguration;
    const FewArg p{a, raw, ldraw, raw_dt, (int)((a.K + 255) / 256)};
    // Two blocks of features read x once for both, and take half as many workgroups: where there are more than a CU each, or little to read
    const bool two = wgs * blocks > NM_CUS || a.K <= 1024;
#define NM_FEW(TT, FT, FUSED, X, LDS) hipLaunchKernelGGL((gemm_i8_few_kernel<TT, FT, FUSED>), dim3((unsigned)(X), (unsigned)blocks), dim3(256), LDS, st, p)
    if (raw) NM_FEW(1, 1, true, wgs, (size_t)(a.M * ((a.K + 63) / 64 * 64 + 16)));
    else if (a.M <= 16) { if (two) NM_FEW(1, 2, false, pairs, 0); else NM_FEW(1, 1, false, wgs, 0); }
    else                { if (two) NM_FEW(2, 2, false, pairs, 0); else NM_FEW(2, 1, false, wgs, 0); }
#undef NM_FEW
    return hipGetLastError();
}

}  // namespace nm
