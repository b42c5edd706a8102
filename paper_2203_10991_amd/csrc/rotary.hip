// Rotary positions: pairs (a, b) of a head's first `part` elements become s (a cos - b sin, a sin + b cos), the angle being position times the pair's frequency; pairs are
// neighbours (interleaved) or lie half of `part` apart.  The gradient is the same with the angle negated (sign).
//
// The angle is formed in binary64 turns and brought into half a turn, and what rounding it to binary32 takes goes into cosine and sine: at position 10^6 a binary32 angle would be off by
// 0.06, a binary32 fraction of a turn by up to 1.6 half steps of one, more than the functions' own errors.  Cosines and sines are made once for a token, in LDS, and serve all its heads; a
// thread then turns 8 pairs (two vectors of 8 elements), or 4 interleaved ones, at a time, fewer at the end of the part.  Bound: HBM: 32768 tokens of 72 heads of 128 in bf16 219 us,
// 5.5 TB/s; a flat list of vectors with four heads' to a thread 246.  Few tokens: a launch, 2.9 us for 8.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "grid_row.h"
#include "nm_internal.h"
#include "row_vec.h"

namespace nm {

namespace {

constexpr int V = EW;            // elements of a vector

// the first `left` of V elements at an element's boundary
template <int DT> __device__ __forceinline__ Raw<DT> load_v(const void *p, int64_t at, int left) { return left >= V ? load_raw<DT>(p, at) : load_raw<DT, true>(p, at, left); }

// 2^lane_bits threads to a head, 2^head_bits heads, and what is left of 256 threads as tokens of a workgroup; `turned` vectors (or pairs of them), `copied` vectors behind the part.
// A thread's first vectors are on their way while the angles are made.
template <int DT, bool INTERLEAVED> __global__ __launch_bounds__(256) void rotary_kernel(const RotaryArg p, int lane_bits, int head_bits, int turned, int copied)
{
    extern __shared__ float2 turns[];
    const int tokens = 256 >> (lane_bits + head_bits), pairs = p.part / 2;
    const int64_t first = (int64_t)grid_place(blockIdx.x, blockIdx.y) * tokens, n = p.B * p.T;
    if (first >= n) return;
    const int lane = (int)threadIdx.x & ((1 << lane_bits) - 1), head0 = (int)threadIdx.x >> lane_bits & ((1 << head_bits) - 1), token = (int)threadIdx.x >> (lane_bits + head_bits);
    const bool there = first + token < n;
    const uint32_t at_token = (uint32_t)(there ? first + token : first), b = at_token / (uint32_t)p.T, t = at_token - b * (uint32_t)p.T;
    const int64_t x0 = b * p.sx.b + t * p.sx.t, y0 = b * p.sy.b + t * p.sy.t;
    // elements of a head that chunk c has, and where they begin
    auto begin = [&](int c) { return c < turned ? c * V : p.part + (c - turned) * V; };
    auto left_of = [&](int c) { return c >= turned ? p.D - begin(c) : INTERLEAVED ? p.part - begin(c) : pairs - begin(c); };
    Raw<DT> v, w;
    auto load = [&](int head, int c) {
        v = load_v<DT>(p.x, x0 + head * p.sx.h + begin(c), left_of(c));
        if (!INTERLEAVED && c < turned) w = load_v<DT>(p.x, x0 + head * p.sx.h + begin(c) + pairs, left_of(c));
    };
    if (there && head0 < p.H && lane < turned + copied) load(head0, lane);
    for (int i = threadIdx.x; i < tokens * pairs; i += 256) {
        const int k = i / pairs, j = i - k * pairs;
        if (first + k >= n) break;
        const uint32_t at = (uint32_t)(first + k), kb = at / (uint32_t)p.T, kt = at - kb * (uint32_t)p.T;
        const int64_t pos = !p.positions ? (int64_t)kt : p.wide ? ((const int64_t *)p.positions)[kb * p.pos_b + kt] : ((const int32_t *)p.positions)[kb * p.pos_b + kt];
        // (the fraction of a turn as two binary32 numbers: the library's functions take the first, and what the second one turns, 2^-23 at most, is their first derivative's share)
        const double turn = (double)pos * (p.freqs[j] * 0.15915494309189533577), part_of_turn = turn - rint(turn);
        const float first_part = (float)part_of_turn, d = (float)(part_of_turn - (double)first_part) * 6.28318530717958647693f;
        float sn, cs;
        sincospif(2.0f * first_part, &sn, &cs);
        const float sn1 = sn;
        sn = __builtin_fmaf(cs, d, sn);
        cs = __builtin_fmaf(-sn1, d, cs);
        turns[i] = make_float2(cs * p.scale, sn * p.scale * p.sign);
    }
    __syncthreads();
    if (!there) return;
    const float2 *cs = turns + token * pairs;
    for (int head = head0; head < p.H; head += 1 << head_bits) {
        const int64_t to = y0 + head * p.sy.h;
        for (int c = lane; c < turned + copied; c += 1 << lane_bits) {
            if (head != head0 || c != lane) load(head, c);
            const int at = begin(c), left = left_of(c);
            float y[V];
            if (c >= turned) {
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = element(v, i);
            } else if constexpr (INTERLEAVED) {
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const float2 k = cs[min(at / 2 + i / 2, pairs - 1)];
                    y[i] = element(v, i) * k.x - element(v, i + 1) * k.y;
                    y[i + 1] = element(v, i) * k.y + element(v, i + 1) * k.x;
                }
            } else {
                float z[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float2 k = cs[min(at + i, pairs - 1)];
                    y[i] = element(v, i) * k.x - element(w, i) * k.y;
                    z[i] = element(v, i) * k.y + element(w, i) * k.x;
                }
                store_row<DT>(p.y, to + pairs + at, 0, left, z);
            }
            store_row<DT>(p.y, to + at, 0, left, y);
        }
    }
}

inline int bits_for(int n) { int b = 0; while ((1 << b) < n) ++b; return b; }

template <int DT, bool IL> hipError_t launch_rotary_as(const RotaryArg &a, hipStream_t st)
{
    const int turned = ((IL ? a.part : a.part / 2) + V - 1) / V, copied = a.x == a.y ? 0 : (a.D - a.part + V - 1) / V;
    const int lane_bits = std::min(8, bits_for(turned + copied)), head_bits = std::min(8 - lane_bits, bits_for(a.H)), tokens = 256 >> (lane_bits + head_bits);
    const int64_t wgs = (a.B * a.T + tokens - 1) / tokens;
    if (wgs > 0x7fffffff) return hipErrorInvalidConfiguration;
    rotary_kernel<DT, IL><<<dim3(grid_row(wgs), grid_rows(wgs)), dim3(256), (size_t)tokens * (a.part / 2) * sizeof(float2), st>>>(a, lane_bits, head_bits, turned, copied);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArg &a, hipStream_t st)
{
    if (a.dt == NM_DT_BF16) return a.interleaved ? launch_rotary_as<NM_DT_BF16, true>(a, st) : launch_rotary_as<NM_DT_BF16, false>(a, st);
    return a.interleaved ? launch_rotary_as<NM_DT_F32, true>(a, st) : launch_rotary_as<NM_DT_F32, false>(a, st);
}

}  // namespace nm
