// One AdamW step (decoupled weight decay) over many tensors in one launch:
//     m <- b1 m + (1 - b1) g        v <- b2 v + (1 - b2) g^2        p <- p (1 - lr wd) - rate m / (sqrt(v) grow + eps)
// with rate = lr / (1 - b1^step), grow = 1 / sqrt(1 - b2^step); g is multiplied by the caller's factors first.  Every operation is binary32 with
// one rounding, in this order; a bf16 parameter is rounded once, from its master copy where it has one.
//
// 8-bit states hold m and r = sqrt(v) (whose range is half of v's in powers of two) as e4m3 codes with a power-of-two scale for every 256 elements:
// the smallest that brings the block's largest finite magnitude to 448 or below, so that a scale that moves leaves the grid of all but the smallest
// values where it was.  A state moves by less than half a step of that grid (v by 0.1 % of itself), which rounding to nearest would drop each time: codes are
// rounded to one of their two neighbours with 16 random bits, without bias.  The random words are Philox4x32-10 (key: the seed, counter:
// quad of elements, tensor, step; word i for element i of the quad, low half for m, high half for r).  r > 0 keeps the smallest code at least: m over a
// vanished r would be a step of any size.  What is not finite gets the NaN code and stays out of the block's scale.
//
// Bound: HBM.  A wave takes 256 elements, each lane a quad of them with one load per array, and all tensors of up to ADAMW_MOST share a launch.  A transformer
// block of width 768 with binary32 states and masters: 213 MB in 36 us (5.9 TB/s; a copy reaches 4.75); of width 4096 with 8-bit states: 2.43 GB in 410 to 480 us
// (5.0 to 5.9 TB/s); of width 768 with 8-bit states and bf16 gradients 71 MB in 17 to 19 us, where the launch's fill and the arithmetic (Philox, rounding) show.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "nm_internal.h"
#include "grid_row.h"
#include "prune_common.h"        // philox4x32_10_uniform_c123, pack_bf16_rne

namespace nm {

namespace {

constexpr int AB = 256;          // elements of a block with one scale: a quad for each lane of a wave, which takes one block

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    // (rows of 16 lanes, then across the rows: the last lane holds the maximum)
#define NM_STEP(CTRL) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false))
    NM_STEP(0x111); NM_STEP(0x112); NM_STEP(0x114); NM_STEP(0x118); NM_STEP(0x142); NM_STEP(0x143);
#undef NM_STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

template <int DT, bool VEC> __device__ __forceinline__ void load4(const void *p, int64_t at, int left, float (&out)[4])
{
    if constexpr (VEC) {
        if constexpr (DT == NM_DT_F32) {
            const float4 v = *(const float4 *)((const float *)p + at);
            out[0] = v.x; out[1] = v.y; out[2] = v.z; out[3] = v.w;
        } else {
            const uint2 v = *(const uint2 *)((const uint16_t *)p + at);
            out[0] = __uint_as_float(v.x << 16); out[1] = __uint_as_float(v.x & 0xffff0000u);
            out[2] = __uint_as_float(v.y << 16); out[3] = __uint_as_float(v.y & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            out[i] = 0.f;
            if (i < left) out[i] = DT == NM_DT_F32 ? ((const float *)p)[at + i] : __uint_as_float((uint32_t)((const uint16_t *)p)[at + i] << 16);
        }
    }
}
template <int DT, bool VEC> __device__ __forceinline__ void store4(void *p, int64_t at, int left, const float (&v)[4])
{
    if constexpr (VEC) {
        if constexpr (DT == NM_DT_F32) *(float4 *)((float *)p + at) = make_float4(v[0], v[1], v[2], v[3]);
        else                           *(uint2 *)((uint16_t *)p + at) = make_uint2(pack_bf16_rne(v[0], v[1]), pack_bf16_rne(v[2], v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) {
                if constexpr (DT == NM_DT_F32) ((float *)p)[at + i] = v[i];
                else                           ((uint16_t *)p)[at + i] = (uint16_t)pack_bf16_rne(v[i], v[i]);
            }
    }
}

// the power of two of a block, as an exponent: largest finite magnitude (bits) over 2^e at most 448 = 1.75 * 2^8
__device__ __forceinline__ int block_exponent(uint32_t top)
{
    const int e = (int)(top >> 23) - 135 + ((top & 0x7fffffu) > 0x600000u);
    return top ? min(max(e, -126), 126) : 0;
}
// r over its block's scale: at most 448 (a root that is a unit too large must not pass it), and where v > 0 at least the smallest code's value; infinities and
// NaN as they are
__device__ __forceinline__ float code_input(float y, float v)
{
    const float least = v > 0.f ? 0x1p-9f : 0.f;
    return v < __builtin_inff() ? __builtin_amdgcn_fmed3f(y, least, 448.f) : v;
}

struct AdamwArg {
    AdamwTensor t[ADAMW_MOST];
    uint32_t first[ADAMW_MOST];  // first workgroup of a tensor
    int count;
    float b1, c1, b2, c2, rate, grow, eps, keep, scale;
    const float *scale_dev;
    uint32_t seed_lo, seed_hi, step;
};

struct Quad { float p[4], g[4], m[4], v[4]; };

template <int PT, int GT, bool Q8, bool MASTER, bool VEC>
__device__ __forceinline__ void load_block(const AdamwTensor &t, int64_t at, int left, Quad &x)
{
    if constexpr (MASTER) load4<NM_DT_F32, VEC>(t.master, at, left, x.p);
    else                  load4<PT, VEC>(t.param, at, left, x.p);
    load4<GT, VEC>(t.grad, at, left, x.g);
    if constexpr (Q8) {
        uint32_t mc = 0, vc = 0;
        if constexpr (VEC) {
            mc = *(const uint32_t *)((const uint8_t *)t.m + at);
            vc = *(const uint32_t *)((const uint8_t *)t.v + at);
        } else {
            for (int i = 0; i < 4; ++i)
                if (i < left) {
                    mc |= (uint32_t)((const uint8_t *)t.m)[at + i] << (8 * i);
                    vc |= (uint32_t)((const uint8_t *)t.v)[at + i] << (8 * i);
                }
        }
        const float ms = t.m_scale[at / AB], vs = t.v_scale[at / AB];
        const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc, true),
                   v01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vc, false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vc, true);
        x.m[0] = m01[0] * ms; x.m[1] = m01[1] * ms; x.m[2] = m23[0] * ms; x.m[3] = m23[1] * ms;
        x.v[0] = v01[0] * vs; x.v[1] = v01[1] * vs; x.v[2] = v23[0] * vs; x.v[3] = v23[1] * vs;
#pragma unroll
        for (int i = 0; i < 4; ++i) x.v[i] = x.v[i] * x.v[i];
    } else {
        load4<NM_DT_F32, VEC>(t.m, at, left, x.m);
        load4<NM_DT_F32, VEC>(t.v, at, left, x.v);
    }
}

template <int PT, int GT, bool Q8, bool MASTER, bool VEC>
__device__ __forceinline__ void step_block(const AdamwArg &a, const AdamwTensor &t, float gs, int64_t at, int left, Quad &x)
{
    float r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float g = x.g[i] * gs;
        x.m[i] = x.m[i] * a.b1 + g * a.c1;
        x.v[i] = x.v[i] * a.b2 + (g * g) * a.c2;
        // (the root and the quotient to a unit in the last place: correctly rounded they took a quarter of the kernel's instructions)
        r[i] = __builtin_amdgcn_sqrtf(x.v[i]);
    }
    // The instruction takes numbers below 2^-126 for zeros, over which a step is infinite where eps is small
    if (min(min(__float_as_uint(x.v[0]), __float_as_uint(x.v[1])), min(__float_as_uint(x.v[2]), __float_as_uint(x.v[3]))) < 0x800000u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (x.v[i] < 0x1p-126f) r[i] = __builtin_amdgcn_sqrtf(x.v[i] * 0x1p64f) * 0x1p-32f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.p[i] = x.p[i] * a.keep - (x.m[i] * a.rate) * __builtin_amdgcn_rcpf(r[i] * a.grow + a.eps);
    if constexpr (Q8) {
        uint32_t mt = 0, vt = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t mb = __float_as_uint(x.m[i]) & 0x7fffffffu, vb = __float_as_uint(x.v[i]);
            if (i < left) {
                mt = max(mt, mb < 0x7f800000u ? mb : 0u);
                vt = max(vt, vb < 0x7f800000u ? vb : 0u);
            }
        }
        // (the block's root is rounded correctly, so that its scale is the one of the definition to the last bit)
        const int me = block_exponent(wave_max(mt)), ve = block_exponent(__float_as_uint(sqrtf(__uint_as_float(wave_max(vt)))));
        const float down_m = __uint_as_float((uint32_t)(127 - me) << 23), down_v = __uint_as_float((uint32_t)(127 - ve) << 23);
        uint32_t w[4];
        const uint64_t quad = (uint64_t)at >> 2;
        philox4x32_10_uniform_c123((uint32_t)quad, __builtin_amdgcn_readfirstlane((uint32_t)(quad >> 32)), t.number, 0x80000000u + a.step, a.seed_lo, a.seed_hi, w);
        // v_cvt_sr_fp8_f32 adds the upper 20 bits of its random word to what lies behind the bits that stay, and cuts: what is not finite becomes a NaN
        int mc = 0, vc = 0;
#define NM_CODE(I)                                                                                                                          \
        mc = __builtin_amdgcn_cvt_sr_fp8_f32(x.m[I] * down_m, (int)(w[I] << 16), mc, I);                                                    \
        vc = __builtin_amdgcn_cvt_sr_fp8_f32(code_input(r[I] * down_v, x.v[I]), (int)(w[I] & 0xffff0000u), vc, I)
        NM_CODE(0); NM_CODE(1); NM_CODE(2); NM_CODE(3);
#undef NM_CODE
        if constexpr (VEC) {
            *(int *)((uint8_t *)t.m + at) = mc;
            *(int *)((uint8_t *)t.v + at) = vc;
        } else {
            for (int i = 0; i < 4; ++i)
                if (i < left) {
                    ((uint8_t *)t.m)[at + i] = (uint8_t)(mc >> (8 * i));
                    ((uint8_t *)t.v)[at + i] = (uint8_t)(vc >> (8 * i));
                }
        }
        if ((threadIdx.x & 63) == 0) {
            t.m_scale[at / AB] = __uint_as_float((uint32_t)(127 + me) << 23);
            t.v_scale[at / AB] = __uint_as_float((uint32_t)(127 + ve) << 23);
        }
    } else {
        store4<NM_DT_F32, VEC>(t.m, at, left, x.m);
        store4<NM_DT_F32, VEC>(t.v, at, left, x.v);
    }
    if constexpr (MASTER) store4<NM_DT_F32, VEC>(t.master, at, left, x.p);
    store4<PT, VEC>(t.param, at, left, x.p);
}

template <int PT, int GT, bool Q8, bool MASTER>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwArg a)
{
    const uint32_t place = grid_place(blockIdx.x, blockIdx.y);
    int k = 0;
    for (int lo = 0, hi = a.count; lo < hi;) {                                   // the last tensor whose first workgroup is not behind this one
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= place) { k = mid; lo = mid + 1; } else hi = mid;
    }
    const AdamwTensor t = a.t[k];
    const float gs = a.scale_dev ? a.scale * *a.scale_dev : a.scale;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t base = ((int64_t)(place - a.first[k]) * 4 + wave) * AB, at = base + 4 * lane;
    if (base >= t.n) return;
    Quad x;
    if (t.aligned && base + AB <= t.n) {
        load_block<PT, GT, Q8, MASTER, true>(t, at, 4, x);
        step_block<PT, GT, Q8, MASTER, true>(a, t, gs, at, 4, x);
    } else {
        const int left = (int)max(min(t.n - at, (int64_t)4), (int64_t)0);
        load_block<PT, GT, Q8, MASTER, false>(t, at, left, x);
        step_block<PT, GT, Q8, MASTER, false>(a, t, gs, at, left, x);
    }
}

}  // namespace

hipError_t launch_adamw(const AdamwTensor *tensors, int count, int param_dt, int grad_dt, bool q8, bool master, const AdamwRates &r, uint64_t seed,
                        hipStream_t st)
{
    AdamwArg a{};
    a.b1 = (float)r.beta1; a.c1 = (float)(1.0 - r.beta1); a.b2 = (float)r.beta2; a.c2 = (float)(1.0 - r.beta2);
    a.rate = (float)(r.lr / (1.0 - pow(r.beta1, (double)r.step)));
    a.grow = (float)(1.0 / sqrt(1.0 - pow(r.beta2, (double)r.step)));
    a.eps = (float)r.eps; a.keep = (float)(1.0 - r.lr * r.weight_decay);
    a.scale = r.grad_scale; a.scale_dev = r.grad_scale_dev;
    a.seed_lo = (uint32_t)seed; a.seed_hi = (uint32_t)(seed >> 32); a.step = (uint32_t)r.step;
    a.count = count;
    int64_t wgs = 0;
    for (int k = 0; k < count; ++k) {
        a.t[k] = tensors[k];
        a.first[k] = (uint32_t)wgs;
        wgs += (tensors[k].n + AB * 4 - 1) / (AB * 4);
        if (wgs > 0x7fffffff) return hipErrorInvalidConfiguration;
    }
    if (!wgs) return hipSuccess;
#define NM_ADAMW(PT, GT, Q8, MASTER) hipLaunchKernelGGL((adamw_kernel<PT, GT, Q8, MASTER>), dim3(grid_row(wgs), grid_rows(wgs)), dim3(256), 0, st, a)
#define NM_ADAMW_S(PT, GT, MASTER) do { if (q8) NM_ADAMW(PT, GT, true, MASTER); else NM_ADAMW(PT, GT, false, MASTER); } while (0)
    if (param_dt == NM_DT_F32) {
        if (grad_dt == NM_DT_F32) NM_ADAMW_S(NM_DT_F32, NM_DT_F32, false); else NM_ADAMW_S(NM_DT_F32, NM_DT_BF16, false);
    } else if (master) {
        if (grad_dt == NM_DT_F32) NM_ADAMW_S(NM_DT_BF16, NM_DT_F32, true); else NM_ADAMW_S(NM_DT_BF16, NM_DT_BF16, true);
    } else {
        if (grad_dt == NM_DT_F32) NM_ADAMW_S(NM_DT_BF16, NM_DT_F32, false); else NM_ADAMW_S(NM_DT_BF16, NM_DT_BF16, false);
    }
#undef NM_ADAMW_S
#undef NM_ADAMW
    return hipGetLastError();
}

}  // namespace nm
