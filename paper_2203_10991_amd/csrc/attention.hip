// Attention, forward: for each head o = softmax(scale q k^T) v over the keys that a query sees, lse = log of the sum of exponentials.
//
// One pass over the keys with the running maximum and sum.  A wave keeps 32 rows (attention.h) as columns: S^T = K Q^T from rows of K in LDS, P^T = 2^(c S^T - m) where it
// lies, O^T += V^T P^T from columns of V in LDS.  The maximum m of a column moves only when a score is 2^8 times beyond it (P then stays below 2^8, sums and products in
// binary32 are as near), so that the sums O are scaled only a few times.  In bf16 O is divided by the sum of the probabilities as they were rounded for the second product, so
// that they add up to one: what rounding moves is then a difference between keys.  lse takes their sum unrounded.  Tiles of keys go through the registers of the workgroup into
// one of two LDS buffers while the other is read; one barrier a tile.  A row that sees no key: o = 0, lse = -infinity.  Rows behind their sequence's queries: the same.
// Bound: many tokens, the matrix instructions and the exponentials beside them, and power: 2 x 8192 tokens, 64 heads of 128 over 8, causal 2.65 ms, 830 TFLOP/s (the vendor library's largest product
// 1400).  Short sequences, each workgroup's beginning and end: 32 x 512, 16 heads of 64 51 us, 340.  Single tokens, HBM: 16 over up to 8192 keys, 64 heads of 128 over 8 79 us, 5.2 TB/s, and the join 5.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "attention.h"
#include "gemm_plan.h"           // NM_CUS

namespace nm {

namespace attn {

constexpr float MOVE = 8.0f;     // a maximum moves when it is beaten by this power of two

// WAVES blocks of 32 rows; PARTS: two waves to a block, each with one half of a tile's keys, whose results are joined at the end
template <int DT, int BLOCKS, int WAVES, int KEYS, int PARTS>
__global__ __launch_bounds__(64 * WAVES * PARTS, DT == NM_DT_F32 && BLOCKS + (WAVES == 1) > 2 ? 1 : 2) void attention_kernel(const AttnArg p, int row_tiles)
{
    typedef Lane<DT, BLOCKS, KEYS> F;
    constexpr int ES = DT == NM_DT_BF16 ? 2 : 4, THREADS = 64 * WAVES * PARTS, ROWS = 32 * WAVES, SB = KEYS / 32 / PARTS;
    __shared__ __align__(F::ALIGN) char lds[2][2][F::BYTES];
    const int lane = (int)threadIdx.x & 63, wave = ((int)threadIdx.x >> 6) % WAVES, part = ((int)threadIdx.x >> 6) / WAVES, hi = lane >> 5;
    // the tiles of a head side by side, those with most keys first
    const Place place(p, row_tiles, p.splits, DT == NM_DT_BF16 || BLOCKS < 3);
    const int tile = row_tiles - 1 - place.tile, split = place.split;
    const Sequence s(p, (int)place.bh);
    const int total = p.Tq * p.group, r0 = tile * ROWS;
    const int row = r0 + wave * 32 + (lane & 31), query = query_of(min(row, total - 1), p), head = s.h * p.group + min(row, total - 1) - query * p.group;
    const bool there = row < total && query < s.nq;
    // keys that the workgroup, the wave (its last and its first row) and the lane see
    const int last_query = query_of(min(r0 + ROWS, total) - 1, p);
    const int most = s.nq == 0 || query_of(r0, p) >= s.nq ? 0 : s.seen(p, min(last_query, s.nq - 1));
    const int wave_first = query_of(min(r0 + wave * 32, total - 1), p), wave_last = query_of(min(r0 + wave * 32 + 31, total - 1), p);
    const int wave_most = r0 + wave * 32 >= total || wave_first >= s.nq ? 0 : s.seen(p, min(wave_last, s.nq - 1)), wave_least = s.seen(p, wave_first);
    const int seen = s.seen(p, query);
    const int tiles = (most + KEYS - 1) / KEYS;
    const int first_tile = part_of(tiles, split, p.splits), end_tile = part_of(tiles, split + 1, p.splits);

    const char *k0 = row_at(p.k, p.sk, s.b, 0, s.h, ES), *v0 = row_at(p.v, p.sv, s.b, 0, s.h, ES);
    Stage<DT, BLOCKS, KEYS, THREADS> ks, vs;
    auto load = [&](int t) {
        const int64_t key0 = (int64_t)t * KEYS;
        const int rows = min(KEYS, s.nk - t * KEYS);
        ks.load([&](int r) { return k0 + (key0 + r) * p.sk.t * ES; }, rows, p.D);
        vs.load([&](int r) { return v0 + (key0 + r) * p.sv.t * ES; }, rows, p.D);
    };
    auto store = [&](int t, int to) {
        const int rows = min(KEYS, s.nk - t * KEYS);
        ks.store(lds[to][0], rows, p.D);
        vs.store(lds[to][1], rows, p.D);
    };
    if (first_tile < end_tile) load(first_tile);
    Frag<DT> q[2 * BLOCKS];
    load_fragments<DT, BLOCKS>(q, row_at(p.q, p.sq, s.b, query, head, ES), there, p.D, lane);
    f32x16 o[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) o[b] = f32x16{};
    float m = -INFINITY, sum = 0.0f, rounded = 0.0f;                     // the sums of P, and of P as rounded
    const float c = p.scale * LOG2E;
    const F at_lane(lane);
    if (first_tile < end_tile) store(first_tile, 0);
    __syncthreads();
    for (int t = first_tile; t < end_tile; ++t) {
        const uint32_t mine = (uint32_t)(part * 32 * SB * Tile<BLOCKS>::ROW);
        const uint32_t kt = at_lane.rows_of(lds_address(lds[t - first_tile & 1][0]) + mine), vt = at_lane.columns_of(lds_address(lds[t - first_tile & 1][1]) + mine);
        const int key0 = t * KEYS + part * 32 * SB;
        if (t + 1 < end_tile) load(t + 1);
        if (key0 < wave_most) {
            f32x16 x[SB];
#pragma unroll
            for (int a = 0; a < SB; ++a) {
                x[a] = f32x16{};
#pragma unroll
                for (int kk = 0; kk < 2 * BLOCKS; ++kk) mma(x[a], F::rows(kt, 32 * a, kk), q[kk]);
            }
            if (key0 + 32 * SB > wave_least) {
#pragma unroll
                for (int a = 0; a < SB; ++a)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (key0 + 32 * a + row_of(i, hi) >= seen) x[a][i] = -INFINITY;
            }
            float top = x[0][0];
#pragma unroll
            for (int a = 0; a < SB; ++a)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, x[a][i]);
            top = fmaxf(top, other_half(top)) * c;
            const bool move = top > m + MOVE;                            // (m = -infinity: any score)
            if (__any(move)) {
                const float by = move ? exp2_of(m - top) : 1.0f;
                if (move) m = top;
                sum *= by;
                rounded *= by;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[b][i] *= by;
            }
            const float base = m == -INFINITY ? 0.0f : m;                // (nothing seen so far)
#pragma unroll
            for (int a = 0; a < SB; ++a)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[a][i] = exp2_of(__builtin_fmaf(x[a][i], c, -base));
            if (DT == NM_DT_F32 || p.lse)
#pragma unroll
                for (int a = 0; a < SB; ++a)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum += x[a][i];
#pragma unroll
            for (int a = 0; a < SB; ++a)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const Frag<DT> w = as_fragment<DT>(x[a], 8 * g);
                    if constexpr (DT == NM_DT_BF16) rounded = sum_of(w, rounded);
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) mma(o[b], F::columns(vt, 32 * a + 16 * g, b), w);
                }
        }
        if (t + 1 < end_tile) store(t + 1, (t - first_tile & 1) ^ 1);
        __syncthreads();
    }
    if constexpr (PARTS == 2) {
        float *other = (float *)&lds[0][0][0] + (wave * BLOCKS * 16) * 64 + lane;
        static_assert(sizeof lds >= (size_t)WAVES * BLOCKS * 16 * 64 * 4, "a block's sums go through the tiles' place");
        __shared__ float stats[3][64 * WAVES];
        if (part) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) other[(16 * b + i) * 64] = o[b][i];
            stats[0][wave * 64 + lane] = m;
            stats[1][wave * 64 + lane] = sum;
            stats[2][wave * 64 + lane] = rounded;
        }
        __syncthreads();
        if (part) return;
        const float m2 = stats[0][wave * 64 + lane], top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top, w1 = exp2_of(m - base), w2 = exp2_of(m2 - base);
        m = top;
        sum = sum * w1 + stats[1][wave * 64 + lane] * w2;
        rounded = rounded * w1 + stats[2][wave * 64 + lane] * w2;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] = o[b][i] * w1 + other[(16 * b + i) * 64] * w2;
    }
    sum += other_half(sum);
    rounded = DT == NM_DT_BF16 ? rounded + other_half(rounded) : sum;
    if (row >= total) return;
    if (!there) {                                                        // (a column that was not there has taken part with zeros)
        m = -INFINITY;
        sum = rounded = 0.0f;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) o[b] = f32x16{};
    }
    const int64_t at = ((int64_t)s.b * p.Hq + head) * p.Tq + query;
    if (p.splits == 1) {
        store_column<DT, BLOCKS>((char *)row_at(p.o, p.so, s.b, query, head, ES), o, rounded != 0.0f ? 1.0f / rounded : 0.0f, p.D, lane, rest_at(p, at));
        if (p.lse && hi == 0) p.lse[at] = (m + __builtin_amdgcn_logf(sum)) * LN2;             // (log2; -infinity of a sum of zero)
    } else {
        // O, m and the sums of this part of the keys
        const int64_t rows = (int64_t)p.B * p.Hq * p.Tq;
        float *to = p.part + ((int64_t)split * rows + at) * p.D;
        store_column<NM_DT_F32, BLOCKS>((char *)to, o, 1.0f, p.D, lane);
        if (hi == 0) {
            float4 *st = (float4 *)(p.part + (int64_t)p.splits * rows * p.D) + (int64_t)split * rows + at;
            *st = make_float4(m, sum, rounded, 0.0f);
        }
    }
}

// the parts of a row together: 2^shift threads to a row, 4 elements each
template <int DT> __global__ __launch_bounds__(256) void attention_join_kernel(const AttnArg p, int shift)
{
    const int64_t rows = (int64_t)p.B * p.Hq * p.Tq, at = (int64_t)blockIdx.x * (256 >> shift) + (threadIdx.x >> shift);
    const int e = ((int)threadIdx.x & ((1 << shift) - 1)) * 4;
    if (at >= rows || e >= p.D) return;
    const int64_t bh = at / p.Tq;
    const int query = (int)(at - bh * p.Tq), b = (int)(bh / p.Hq), head = (int)(bh - (int64_t)b * p.Hq);
    const float4 *st = (const float4 *)(p.part + (int64_t)p.splits * rows * p.D) + at;
    float m = -INFINITY;
#pragma unroll 8
    for (int k = 0; k < p.splits; ++k) m = fmaxf(m, st[k * rows].x);
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0.0f, rounded = 0.0f;
    f32x4 o = {0, 0, 0, 0};
#pragma unroll 8
    for (int k = 0; k < p.splits; ++k) {
        const float4 part = st[k * rows];
        const float w = exp2_of(part.x - base);
        const f32x4 x = *(const f32x4 *)(p.part + (k * rows + at) * p.D + e);
        sum += w * part.y;
        rounded += w * part.z;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += w * x[i];
    }
    const float by = rounded != 0.0f ? 1.0f / rounded : 0.0f;
    char *to = (char *)row_at(p.o, p.so, b, query, head, DT == NM_DT_BF16 ? 2 : 4);
    store_four<DT>(to, rest_at(p, at), e, f32x4{o[0] * by, o[1] * by, o[2] * by, o[3] * by});
    if (p.lse && e == 0) p.lse[at] = (base + __builtin_amdgcn_logf(sum)) * LN2;
}

// How many rows a workgroup takes, and in how many parts the keys go.
// A block of rows (single tokens): a workgroup of one wave with small tiles, or, where keys are many, of four, three of which only load and store: 16 x 1 token over 8192 keys, 64 heads of 128 over 8,
// 110 us with one and 106 with four, 1 x 1 over 32768, 32 heads over 8, 54 and 35, in binary32 8 x 1 over 8192 363 and 229; but 1 x 1 over 1000 keys 10.8 and 13.9 (binary32 20 and 34), 8 x 1 over 2000,
// 32 heads of 64, 28.6 and 31.6, over 3000 to 4000 as much either way.
// Parts: until there are workgroups for every CU, of keys enough to be worth their place in the join.  Unsplit: 353, 198 and 46 us where it is 106, 35 and 11.  Parts of at least 64 and 256 keys: 1 x 1 over 1000 10.8 us
// (128: 12.5, 256: 18.6), 2 x 100 over 3000, 8 heads of 128, 21 (512: 24, 1024: 34); 32 parts at most, since one thread joins all parts of its elements (2 x 4 over 4000, 32 heads over 4: 16.8, with 63 parts 23).
struct Plan { int waves, splits, parts; int64_t row_tiles; };
inline Plan plan_of(const AttnArg &a)
{
    Plan p;
    const int64_t total = (int64_t)a.Tq * a.group, heads = (int64_t)a.B * a.Hk;
    const bool one = total <= 32;
    p.waves = one && a.Tk < 4000 ? 1 : 4;
    p.row_tiles = (total + 32 * p.waves - 1) / (32 * p.waves);
    const int64_t wgs = heads * p.row_tiles, want = (p.waves == 1 ? 8 : one ? 4 : 2) * NM_CUS;
    const int64_t least = p.waves == 1 ? 64 : 256;                      // keys to a part
    p.splits = wgs >= want / 2 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({want / wgs, (a.Tk + least - 1) / least, 32}));
    // two waves to a block of rows where a CU has one workgroup at most, in binary32 (full attention, one wave and two, in us: 8 x 197 tokens of 12 heads of 64 17.6 and 15.4,
    // 2 x 1000 of 4 heads on one 37.7 and 29.9; with two workgroups to a CU, 2 x 1333 of 12 on one of 48, 74 and 77).  In bf16, where a tile is a third of the work, there is nothing
    // in it (8 x 197: 9.5 and 9.5, 6 x 256 of 16 of 128: 14.5 and 15.3)
    p.parts = a.dt == NM_DT_F32 && a.D <= 64 && a.Tk > 64 && p.waves == 4 && wgs * p.splits < NM_CUS ? 2 : 1;
    return p;
}

template <int DT, int BLOCKS> hipError_t launch(const AttnArg &a, const Plan &p, hipStream_t st)
{
    const int64_t wgs = (int64_t)a.B * a.Hk * p.row_tiles * p.splits;
    if (!grid_holds(wgs, 64 * p.waves * p.parts) || wgs > 0x7fffffff) return hipErrorInvalidConfiguration;
    if (p.waves == 1) attention_kernel<DT, BLOCKS, 1, 32, 1><<<dim3((unsigned)wgs), dim3(64), 0, st>>>(a, (int)p.row_tiles);
    else if (p.parts == 1) attention_kernel<DT, BLOCKS, 4, DT == NM_DT_F32 ? 32 : 64, 1><<<dim3((unsigned)wgs), dim3(256), 0, st>>>(a, (int)p.row_tiles);
    else if constexpr (DT == NM_DT_F32 && BLOCKS <= 2) attention_kernel<DT, BLOCKS, 4, 64, 2><<<dim3((unsigned)wgs), dim3(512), 0, st>>>(a, (int)p.row_tiles);
    return hipGetLastError();
}
template <int DT> hipError_t launch(const AttnArg &a, const Plan &p, hipStream_t st)
{
    switch ((a.D + 31) / 32) {
        case 1: return launch<DT, 1>(a, p, st);
        case 2: return launch<DT, 2>(a, p, st);
        case 3: return launch<DT, 3>(a, p, st);
        default: return launch<DT, 4>(a, p, st);
    }
}

}  // namespace attn

size_t attention_workspace(const AttnArg &a)
{
    const attn::Plan p = attn::plan_of(a);
    return p.splits == 1 ? 0 : (size_t)p.splits * a.B * a.Hq * a.Tq * (a.D + 4) * 4;
}

hipError_t launch_attention(AttnArg a, void *workspace, hipStream_t st)
{
    const attn::Plan p = attn::plan_of(a);
    a.splits = p.splits;
    a.part = (float *)workspace;
    a.mix = attn::mix_of(a, (int64_t)a.B * a.Hk, p.row_tiles);
    hipError_t e = a.dt == NM_DT_BF16 ? attn::launch<NM_DT_BF16>(a, p, st) : attn::launch<NM_DT_F32>(a, p, st);
    if (e != hipSuccess || p.splits == 1) return e;
    const int shift = a.D <= 32 ? 3 : a.D <= 64 ? 4 : 5;
    const int64_t rows = (int64_t)a.B * a.Hq * a.Tq, wgs = (rows + (256 >> shift) - 1) / (256 >> shift);
    if (!grid_holds(wgs, 256)) return hipErrorInvalidConfiguration;
    if (a.dt == NM_DT_BF16) attn::attention_join_kernel<NM_DT_BF16><<<dim3((unsigned)wgs), dim3(256), 0, st>>>(a, shift);
    else attn::attention_join_kernel<NM_DT_F32><<<dim3((unsigned)wgs), dim3(256), 0, st>>>(a, shift);
    return hipGetLastError();
}

}  // namespace nm
