// Attention, gradients.  With P = 2^(c S - lse) recomputed from q, k and the forward pass's lse, delta = sum over the head of g o, dP = g v^T:
//     dS = P (dP - delta)      dq = scale dS k      dk = scale dS^T q      dv = P^T g
// Where a row looks at few keys, dP and delta nearly cancel, and a bf16 o makes delta too coarse; `rest` holds what its rounding took.  16 heads of 512 tokens, scores of a deviation
// of 0.4 to 2.7: 2-norm of dq's and dk's errors 0.27 and 0.29 % without it, 0.24 % with it and with an exact delta alike, before LARGE below (0.17 % is the rounding of the results).
// Two kernels, each with its results in registers from beginning to end, so that no sum crosses workgroups and the same call gives the same bits:
//   dq      a wave keeps 32 rows (attention.h) of q and g as columns: S^T = K Q^T, dP^T = V G^T, dQ^T += K^T dS^T over tiles of keys; delta comes from its own rows first
//   dk dv   a wave keeps 32 keys as columns: S = Q K^T, dP = G V^T, dV^T += G^T P, dK^T += Q^T dS over tiles of the rows of all heads that share the keys
// Both recompute S and dP: seven products instead of five, and neither atomics nor a matrix in memory (dS of a pair, written and read in bf16, would take 4 bytes
// at about 5 TB/s against 4 D operations).  Bound: as the forward pass.  2 x 8192 tokens, 64 heads of 128 over 8, causal: dq 3.3 ms (1000 TFLOP/s of its three products), dk dv 4.6 (950
// of four); 32 x 512, 16 heads of 64: 67 and 82 us (385 and 420); 6 x up to 1333, 12 heads of 80 over 1: 55 and 82, and 12 for the sum of the parts.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "attention.h"
#include "gemm_plan.h"           // NM_CUS

namespace nm {

namespace attn {

// In bf16 dS is rounded for the products with k and q.  Where a probability is large, few keys make up a row's sums, rounding does not average out, and dS nearly cancels: blocks that hold one
// above 1/8 (LARGE, as a power of two) take what rounding took from their dS in a further product, one of seven.  3 heads of 32, 3332 tokens, scores of a deviation of 6: 2-norm of dq's and dk's
// errors 0.272 and 0.249 % without, 0.20 and 0.19 with; scores of a deviation of 2 over 2898 keys 0.25 and 0.243.  It costs 71 + 76 -> 74 + 81 us at 32 x 512 tokens, 16 heads of 64 (a fifth of the blocks),
// 3.40 + 4.45 -> 3.48 + 4.65 ms at 2 x 8192, 64 heads of 128 over 8 (one in 500); from 1/16 on 78 + 84 us, and 0.236 %.  The column fragments are read again there: held, they spill.
constexpr float LARGE = -3.0f;

// PARTS: two waves to a block of rows, each with one half of a tile's keys, whose sums are added up at the end
// (heads of 64 in bf16: three waves to a SIMD, 168 registers and four spilled in front of the loop; with 172 registers and two waves, 32 x 512 tokens of 16 heads take 78 us instead of 65)
template <int DT, int BLOCKS, int KEYS, int PARTS>
__global__ __launch_bounds__(256 * PARTS, DT == NM_DT_F32 && BLOCKS > 2 ? 1 : DT == NM_DT_BF16 && BLOCKS == 2 && PARTS == 1 ? 3 : 2) void attention_dq_kernel(const AttnArg p, int row_tiles)
{
    typedef Lane<DT, BLOCKS, KEYS> F;
    constexpr int ES = DT == NM_DT_BF16 ? 2 : 4, ROWS = 128, SB = KEYS / 32 / PARTS;
    __shared__ __align__(F::ALIGN) char lds[2][2][F::BYTES];
    const int lane = (int)threadIdx.x & 63, wave = ((int)threadIdx.x >> 6) % 4, part = ((int)threadIdx.x >> 6) / 4, hi = lane >> 5;
    const Place place(p, row_tiles, 1, DT == NM_DT_BF16 || BLOCKS < 3);
    const uint32_t bh = place.bh;
    const int tile = row_tiles - 1 - place.tile;
    const Sequence s(p, (int)bh);
    const int total = p.Tq * p.group, r0 = tile * ROWS;
    const int row = r0 + wave * 32 + (lane & 31), query = query_of(min(row, total - 1), p), head = s.h * p.group + min(row, total - 1) - query * p.group;
    const bool there = row < total && query < s.nq;
    const int last_query = query_of(min(r0 + ROWS, total) - 1, p);
    const int most = s.nq == 0 || query_of(r0, p) >= s.nq ? 0 : s.seen(p, min(last_query, s.nq - 1));
    const int wave_first = query_of(min(r0 + wave * 32, total - 1), p), wave_last = query_of(min(r0 + wave * 32 + 31, total - 1), p);
    const int wave_most = r0 + wave * 32 >= total || wave_first >= s.nq ? 0 : s.seen(p, min(wave_last, s.nq - 1)), wave_least = s.seen(p, wave_first);
    const int seen = s.seen(p, query), tiles = (most + KEYS - 1) / KEYS;

    const char *k0 = row_at(p.k, p.sk, s.b, 0, s.h, ES), *v0 = row_at(p.v, p.sv, s.b, 0, s.h, ES);
    Stage<DT, BLOCKS, KEYS, 256 * PARTS> ks, vs;
    auto load = [&](int t) {
        const int64_t key0 = (int64_t)t * KEYS;
        const int rows = min(KEYS, s.nk - t * KEYS);
        ks.load([&](int r) { return k0 + (key0 + r) * p.sk.t * ES; }, rows, p.D);
        vs.load([&](int r) { return v0 + (key0 + r) * p.sv.t * ES; }, rows, p.D);
    };
    auto store = [&](int t) {
        const int rows = min(KEYS, s.nk - t * KEYS);
        ks.store(lds[t & 1][0], rows, p.D);
        vs.store(lds[t & 1][1], rows, p.D);
    };
    if (tiles > 0) load(0);
    Frag<DT> q[2 * BLOCKS], g[2 * BLOCKS];
    const char *g_row = row_at(p.g, p.sg, s.b, query, head, ES);
    load_fragments<DT, BLOCKS>(g, g_row, there, p.D, lane);
    const int64_t row_of_lse = ((int64_t)s.b * p.Hq + head) * p.Tq + query;
    const float part_of_delta = row_product<DT, BLOCKS>(g, g_row, row_at(p.o, p.so, s.b, query, head, ES), rest_at(p, row_of_lse), p.D, lane);
    float delta = there ? part_of_delta : 0.0f;
    delta += other_half(delta);
    load_fragments<DT, BLOCKS>(q, row_at(p.q, p.sq, s.b, query, head, ES), there, p.D, lane);
    // (a row that sees nothing has lse = -infinity: with +infinity in its place P is zero)
    const float l = there ? p.lse[row_of_lse] : -INFINITY, lse = l == -INFINITY ? INFINITY : l * LOG2E, c = p.scale * LOG2E;
    if (hi == 0 && part == 0 && row < total) p.rows[(int64_t)bh * total + row] = make_float2(lse, delta);
    f32x16 dq[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) dq[b] = f32x16{};

    const F at_lane(lane);
    if (tiles > 0) store(0);
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
        const uint32_t mine = (uint32_t)(part * 32 * SB * Tile<BLOCKS>::ROW), k_at = lds_address(lds[t & 1][0]) + mine;
        const uint32_t kt = at_lane.rows_of(k_at), vt = at_lane.rows_of(lds_address(lds[t & 1][1]) + mine), kc = at_lane.columns_of(k_at);
        const int key0 = t * KEYS + part * 32 * SB;
        if (t + 1 < tiles) load(t + 1);
        if (key0 < wave_most) {
            const bool edge = key0 + 32 * SB > wave_least;
#pragma unroll
            for (int a = 0; a < SB; ++a) {
                f32x16 x = f32x16{}, dp = f32x16{};
                float top = -INFINITY;
#pragma unroll
                for (int kk = 0; kk < 2 * BLOCKS; ++kk) {
                    mma(x, F::rows(kt, 32 * a, kk), q[kk]);
                    mma(dp, F::rows(vt, 32 * a, kk), g[kk]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float e = __builtin_fmaf(x[i], c, -lse);
                    top = fmaxf(top, e);
                    x[i] = exp2_of(e) * (dp[i] - delta);
                }
                if (edge) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (key0 + 32 * a + row_of(i, hi) >= seen) x[i] = 0.0f;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const Frag<DT> w = as_fragment<DT>(x, 8 * h);
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) mma(dq[b], F::columns(kc, 32 * a + 16 * h, b), w);
                }
                if (DT == NM_DT_BF16 && __any(top > LARGE)) {
                    uint32_t again = kc;                                 // (read again, not held)
                    asm volatile("" : "+v"(again));
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        take_rounded<DT>(x, 8 * h, as_fragment<DT>(x, 8 * h));
                        const Frag<DT> w = as_fragment<DT>(x, 8 * h);
#pragma unroll
                        for (int b = 0; b < BLOCKS; ++b) mma(dq[b], F::columns(again, 32 * a + 16 * h, b), w);
                    }
                }
            }
        }
        if (t + 1 < tiles) store(t + 1);
        __syncthreads();
    }
    if constexpr (PARTS == 2) {
        float *other = (float *)&lds[0][0][0] + (wave * BLOCKS * 16) * 64 + lane;
        static_assert(sizeof lds >= (size_t)4 * BLOCKS * 16 * 64 * 4, "a block's sums go through the tiles' place");
        if (part) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) other[(16 * b + i) * 64] = dq[b][i];
        }
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) dq[b][i] += other[(16 * b + i) * 64];
    }
    if (!there)
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) dq[b] = f32x16{};
    if (row < total) store_column<DT, BLOCKS>((char *)row_at(p.dq, p.sdq, s.b, query, head, ES), dq, p.scale, p.D, lane);
}

// Whether two waves share a block of rows in attention_dq_kernel: where CUs stay without a workgroup and the keys are many.  All gradients, one wave and two, in us: 1 x 2000 tokens of 8 heads
// of 64 95 and 87 (binary32 275 and 254), 2 x 1333 of 12 heads on one of 48 74 and 69, 500 of 16 on four of 128 57 and 55; but 2 x 300 of 8 of 64 26.3 and 26.8, 4 x 256 of 16 23.2 and 24.3
inline bool two_parts(const AttnArg &a, int64_t wgs) { return wgs < NM_CUS && a.Tk >= 512 && (a.dt == NM_DT_BF16 || a.D <= 64); }

// the tiles of rows that see any key from key0 on: those of queries from a first one on
struct RowTiles {
    int first, count;
    __device__ __forceinline__ RowTiles(const AttnArg &p, const Sequence &s, int key0, int rows)
    {
        const int total = s.nq * p.group, query = p.causal ? max(0, key0 - (s.nk - s.nq)) : 0;
        first = (int)(min((int64_t)total, (int64_t)query * p.group) / rows);
        count = key0 < s.nk ? max(0, (total + rows - 1) / rows - first) : 0;
    }
};

template <int DT, int BLOCKS, int ROWS, int WAVES, int PER_SIMD, bool VL, int BUFFERS>
__global__ __launch_bounds__(64 * WAVES, PER_SIMD) void attention_dkdv_kernel(const AttnArg p, int key_tiles)
{
    typedef Lane<DT, BLOCKS, ROWS> F;
    typedef Lane<DT, BLOCKS, 32 * WAVES> FV;
    constexpr int ES = DT == NM_DT_BF16 ? 2 : 4, KEYS = 32 * WAVES, SB = ROWS / 32, THREADS = 64 * WAVES;
    constexpr uint32_t G = F::BYTES;                                     // from q's tile to g's
    __shared__ __align__(F::ALIGN) char lds[BUFFERS][2][F::BYTES];
    __shared__ __align__(FV::ALIGN) char v_lds[VL ? FV::BYTES : 16];
    __shared__ __align__(16) float lse_of[BUFFERS][ROWS], delta_of[BUFFERS][ROWS];          // (read four at a time)
    __shared__ int seen_of[BUFFERS][ROWS];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, hi = lane >> 5;
    const Place place(p, key_tiles, p.splits, PER_SIMD * 4 >= 2 * WAVES);
    const uint32_t bh = place.bh;
    const int tile = place.tile, split = place.split;                    // (the first keys have most rows)
    const Sequence s(p, (int)bh);
    const int key0 = tile * KEYS, wave_key = key0 + wave * 32, key = wave_key + (lane & 31);
    const int total = s.nq * p.group;
    const RowTiles tiles(p, s, key0, ROWS);
    const int first_tile = tiles.first + min(tiles.count, split * p.chunk), end_tile = tiles.first + min(tiles.count, (split + 1) * p.chunk);
    if (split > 0 && first_tile >= end_tile) return;
    const int blind = p.causal ? max(0, s.nq - s.nk) * p.group : 0;       // rows that see nothing: what their q and g hold does not count

    const char *q0 = row_at(p.q, p.sq, s.b, 0, s.h * p.group, ES), *g0 = row_at(p.g, p.sg, s.b, 0, s.h * p.group, ES);
    Stage<DT, BLOCKS, ROWS, THREADS> qs, gs;
    float2 row_next = make_float2(0.0f, 0.0f);
    const float2 *rows_of_head = p.rows + (int64_t)bh * p.Tq * p.group;
    auto load = [&](int t) {
        const int r0 = t * ROWS, rows = min(ROWS, total - r0);
        auto at = [&](const char *from, const AttnStride &st, int r) {
            const int query = query_of(r0 + r, p);
            return from + (query * st.t + (r0 + r - query * p.group) * st.h) * ES;
        };
        qs.load([&](int r) { return at(q0, p.sq, r); }, rows, p.D);
        gs.load([&](int r) { return at(g0, p.sg, r); }, rows, p.D);
        if ((int)threadIdx.x < ROWS) row_next = rows_of_head[r0 + min((int)threadIdx.x, rows - 1)];
    };
    auto store = [&](int t, int to) {
        const int r0 = t * ROWS, rows = min(ROWS, total - r0);
        qs.store(lds[to][0], rows, p.D, blind - r0);
        gs.store(lds[to][1], rows, p.D, blind - r0);
        if ((int)threadIdx.x < ROWS) {
            const bool ok = (int)threadIdx.x < rows;
            lse_of[to][threadIdx.x] = ok ? row_next.x : INFINITY;        // (P = 0)
            delta_of[to][threadIdx.x] = ok ? row_next.y : 0.0f;
            seen_of[to][threadIdx.x] = ok ? s.seen(p, query_of(r0 + (int)threadIdx.x, p)) : 0;
        }
    };
    Frag<DT> k[2 * BLOCKS], v[VL ? 1 : 2 * BLOCKS];
    f32x16 dk[BLOCKS], dv[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) dk[b] = dv[b] = f32x16{};
    if (first_tile < end_tile) {
        const int safe_key = min(key, s.nk - 1);
        load(first_tile);
        load_fragments<DT, BLOCKS>(k, row_at(p.k, p.sk, s.b, safe_key, s.h, ES), key < s.nk, p.D, lane);
        if constexpr (VL) {
            const char *v0 = row_at(p.v, p.sv, s.b, key0, s.h, ES);
            const int rows = min(KEYS, s.nk - key0);
            Stage<DT, BLOCKS, KEYS, THREADS> vs;
            vs.load([&](int r) { return v0 + r * p.sv.t * ES; }, rows, p.D);
            vs.store(v_lds, rows, p.D);
        } else load_fragments<DT, BLOCKS>(v, row_at(p.v, p.sv, s.b, safe_key, s.h, ES), key < s.nk, p.D, lane);
        store(first_tile, 0);
    }
    const float c = p.scale * LOG2E;
    const F at_lane(lane);
    __syncthreads();
    for (int t = first_tile; t < end_tile; ++t) {
        const int buf = t - first_tile & (BUFFERS - 1);
        // (one register for the rows of both tiles and one for their columns: the second tile is a constant away)
        [[maybe_unused]] const uint32_t v_rows = VL ? at_lane.rows_of(lds_address(v_lds) + (uint32_t)(wave * 32 * Tile<BLOCKS>::ROW)) : 0u;
        const uint32_t rows = at_lane.rows_of(lds_address(lds[buf][0])), columns = at_lane.columns_of(lds_address(lds[buf][0]));
        if (t + 1 < end_tile) load(t + 1);
        // the tile's last row sees most keys, its first one fewest
        const int tile_most = s.seen(p, query_of(min(t * ROWS + ROWS, total) - 1, p)), tile_least = s.seen(p, query_of(t * ROWS, p));
        if (wave_key < tile_most) {
            const bool edge = tile_least < wave_key + 32;
#pragma unroll
            for (int a = 0; a < SB; ++a) {
                f32x16 x = f32x16{}, dp = f32x16{};
                float top = -INFINITY;
#pragma unroll
                for (int kk = 0; kk < 2 * BLOCKS; ++kk) {
                    mma(x, F::rows(rows, 32 * a, kk), k[kk]);
                    if constexpr (VL) mma(dp, F::rows(rows + G, 32 * a, kk), FV::rows(v_rows, 0, kk));
                    else mma(dp, F::rows(rows + G, 32 * a, kk), v[kk]);
                }
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const f32x4 l = *(const f32x4 *)&lse_of[buf][32 * a + row_of(i, hi)], d = *(const f32x4 *)&delta_of[buf][32 * a + row_of(i, hi)];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float e = __builtin_fmaf(x[i + j], c, -l[j]);
                        top = fmaxf(top, e);
                        x[i + j] = exp2_of(e);
                        dp[i + j] = x[i + j] * (dp[i + j] - d[j]);
                    }
                }
                if (edge) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (key >= seen_of[buf][32 * a + row_of(i, hi)]) x[i] = dp[i] = 0.0f;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const Frag<DT> w = as_fragment<DT>(x, 8 * h), ds = as_fragment<DT>(dp, 8 * h);
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) {
                        mma(dv[b], F::columns(columns + G, 32 * a + 16 * h, b), w);
                        mma(dk[b], F::columns(columns, 32 * a + 16 * h, b), ds);
                    }
                }
                if (DT == NM_DT_BF16 && __any(top > LARGE)) {
                    uint32_t again = columns;                            // (read again, not held)
                    asm volatile("" : "+v"(again));
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        take_rounded<DT>(dp, 8 * h, as_fragment<DT>(dp, 8 * h));
                        const Frag<DT> w = as_fragment<DT>(dp, 8 * h);
#pragma unroll
                        for (int b = 0; b < BLOCKS; ++b) mma(dk[b], F::columns(again, 32 * a + 16 * h, b), w);
                    }
                }
            }
        }
        if constexpr (BUFFERS == 1) __syncthreads();
        if (t + 1 < end_tile) store(t + 1, buf ^ (BUFFERS - 1));
        __syncthreads();
    }
    if (key >= p.Tk) return;
    if (key >= s.nk)                                                     // (what stands in the columns of keys that are not there)
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) dk[b] = dv[b] = f32x16{};
    if (p.splits == 1) {
        store_column<DT, BLOCKS>((char *)row_at(p.dk, p.sdk, s.b, key, s.h, ES), dk, p.scale, p.D, lane);
        store_column<DT, BLOCKS>((char *)row_at(p.dv, p.sdv, s.b, key, s.h, ES), dv, 1.0f, p.D, lane);
    } else {
        const int64_t keys = (int64_t)p.B * p.Hk * p.Tk, at = ((int64_t)s.b * p.Hk + s.h) * p.Tk + key;
        store_column<NM_DT_F32, BLOCKS>((char *)(p.part + ((int64_t)split * 2 * keys + at) * p.D), dk, p.scale, p.D, lane);
        store_column<NM_DT_F32, BLOCKS>((char *)(p.part + ((int64_t)(split * 2 + 1) * keys + at) * p.D), dv, 1.0f, p.D, lane);
    }
}

// the parts of dk and dv added up in their order: 4 elements to a thread; blockIdx.y: dk, dv
template <int DT> __global__ __launch_bounds__(256) void attention_sum_kernel(const AttnArg p, int tile_keys, int tile_rows)
{
    const int64_t keys = (int64_t)p.B * p.Hk * p.Tk, n4 = keys * p.D / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n4) return;
    const int which = (int)blockIdx.y;
    const int64_t at = 4 * i / p.D, bh = at / p.Tk;
    const int e = (int)(4 * i - at * p.D), b = (int)(bh / p.Hk), key = (int)(at - bh * p.Tk);
    // (the parts that were made: one at least)
    const RowTiles tiles(p, Sequence(p, (int)bh), key / tile_keys * tile_keys, tile_rows);
    const int parts = min(p.splits, max(1, (tiles.count + p.chunk - 1) / p.chunk));
    f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
    for (int k = 0; k < parts; ++k) {
        const f32x4 y = *(const f32x4 *)(p.part + (int64_t)(2 * k + which) * keys * p.D + 4 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] += y[j];
    }
    const AttnStride st = which ? p.sdv : p.sdk;
    char *to = (char *)row_at(which ? p.dv : p.dk, st, b, key, bh - (int64_t)b * p.Hk, DT == NM_DT_BF16 ? 2 : 4);
    if constexpr (DT == NM_DT_BF16) *(u32x2 *)(to + e * 2) = u32x2{pack_bf16_rne(x[0], x[1]), pack_bf16_rne(x[2], x[3])};
    else *(f32x4 *)(to + e * 4) = x;
}

// Waves of a workgroup of the dk dv kernel, waves to a SIMD, and whether v's fragments come from LDS each time instead of staying in registers; tiles have 32 rows.
// In bf16: 128 elements to a head have 128 registers of sums; with v in LDS the rest fits two waves to a SIMD, with 64 three.  WIDE: eight waves share a tile of rows instead of
// four, for heads of more than 64 elements where keys and workgroups are many.  2 x 8192 tokens, 64 heads of 128 over 8: one wave to a SIMD with everything in registers 8.1 ms,
// four waves 5.1, eight 4.6; 32 x 512 tokens, 16 heads of 64: 105 us with two to a SIMD, 94 with three.
template <int DT, int BLOCKS, bool WIDE> struct KeyShape { static constexpr int waves = 4, per_simd = DT == NM_DT_F32 ? 1 : 2; static constexpr bool v_in_lds = false; static constexpr int buffers = 2; };
template <> struct KeyShape<NM_DT_F32, 4, false> { static constexpr int waves = 4, per_simd = 1; static constexpr bool v_in_lds = true; static constexpr int buffers = 1; };
template <bool WIDE> struct KeyShape<NM_DT_BF16, 2, WIDE> { static constexpr int waves = 4, per_simd = 3; static constexpr bool v_in_lds = true; static constexpr int buffers = 2; };
template <bool WIDE> struct KeyShape<NM_DT_BF16, 3, WIDE> { static constexpr int waves = WIDE ? 8 : 4, per_simd = 2; static constexpr bool v_in_lds = true; static constexpr int buffers = 2; };
template <bool WIDE> struct KeyShape<NM_DT_BF16, 4, WIDE> { static constexpr int waves = WIDE ? 8 : 4, per_simd = 2; static constexpr bool v_in_lds = true; static constexpr int buffers = 2; };
constexpr int KEY_ROWS = 32;
// 2 x 8192 tokens, 16 heads of 96, all gradients: eight waves 2986 us (causal 1677), four 3172 (1886); 4 x 2048 tokens, 16 heads of 96 over 4, causal: 333 and 304;
// 32 x 512 tokens, 16 heads of 80, causal: 228 and 220
inline bool wide_keys(const AttnArg &a) { return a.dt == NM_DT_BF16 && a.D > 64 && a.Tk >= 2048 && (int64_t)a.B * a.Hk * ((a.Tk + 255) / 256) >= NM_CUS; }

template <int DT, int BLOCKS, bool WIDE> struct KeyPlan {
    typedef KeyShape<DT, BLOCKS, WIDE> W;
    static constexpr int dt = DT, blocks = BLOCKS;
    // How many parts the rows go in where keys are few, and how long one is: rows divided evenly where every key is seen, so that a key's part is as long whether many
    // rows see it or few (parts that nothing is left for end at once).  Twice as many workgroups as have room, since they are all as long: 6 x up to 1333 tokens, 12 heads of
    // 80 over 1, causal: 125 us with as many as have room, 80 with twice, 79 with three and four times.  A part has eight tiles at least, or three where
    // that still leaves half of the room: all gradients, 1 x 375 tokens of 2 heads of 40 29 us and 22, 3 x 247 of 4 over 1 of 56 31 and 23, 2 x 1150 of one of 40 in binary32 96 and 88; with the room full, 10 x 221 of 42
    // over 21 of 88 75 and 100.
    static void plan(AttnArg &a)
    {
        const int64_t keys = 32 * W::waves, wgs = (int64_t)a.B * a.Hk * ((a.Tk + keys - 1) / keys), tiles = ((int64_t)a.Tq * a.group + KEY_ROWS - 1) / KEY_ROWS;
        const int64_t room = (int64_t)NM_CUS * W::per_simd * 4 / W::waves;
        a.splits = wgs >= room || wgs == 0 ? 1 : (int)std::max<int64_t>({1, std::min<int64_t>({room * (a.causal ? 4 : 2) / wgs, tiles / 8, 32}), std::min<int64_t>({room / 2 / wgs, tiles / 3, 32})});
        a.chunk = (int)std::max<int64_t>(1, (tiles + a.splits - 1) / a.splits);
    }
};
template <typename F> auto with_plan(const AttnArg &a, F &&f)
{
    const int blocks = (a.D + 31) / 32;
    if (a.dt == NM_DT_F32) return blocks == 1 ? f(KeyPlan<NM_DT_F32, 1, false>{}) : blocks == 2 ? f(KeyPlan<NM_DT_F32, 2, false>{}) : blocks == 3 ? f(KeyPlan<NM_DT_F32, 3, false>{}) : f(KeyPlan<NM_DT_F32, 4, false>{});
    if (wide_keys(a)) return blocks == 3 ? f(KeyPlan<NM_DT_BF16, 3, true>{}) : f(KeyPlan<NM_DT_BF16, 4, true>{});
    return blocks == 1 ? f(KeyPlan<NM_DT_BF16, 1, false>{}) : blocks == 2 ? f(KeyPlan<NM_DT_BF16, 2, false>{}) : blocks == 3 ? f(KeyPlan<NM_DT_BF16, 3, false>{}) : f(KeyPlan<NM_DT_BF16, 4, false>{});
}

template <typename P> hipError_t launch_grads(AttnArg a, P, hipStream_t st)
{
    constexpr int DT = P::dt, BLOCKS = P::blocks, KEYS = DT == NM_DT_F32 ? 32 : 64;
    typedef typename P::W W;
    const int64_t heads = (int64_t)a.B * a.Hk, row_tiles = ((int64_t)a.Tq * a.group + 127) / 128, kt = ((int64_t)a.Tk + 32 * W::waves - 1) / (32 * W::waves);
    const int64_t wq = heads * row_tiles, wk = heads * kt * a.splits, ws = (heads * a.Tk * a.D / 4 + 255) / 256;
    if (std::max(wq, wk) > 0x7fffffff || !grid_holds(std::max(wq, wk), 64 * W::waves) || !grid_holds(wq, 512) || !grid_holds(ws, 256)) return hipErrorInvalidConfiguration;
    if (wq > 0) {
        a.mix = mix_of(a, heads, row_tiles);
        if constexpr (DT == NM_DT_BF16 || BLOCKS <= 2) {
            if (two_parts(a, wq)) attention_dq_kernel<DT, BLOCKS, 64, 2><<<dim3((unsigned)wq), dim3(512), 0, st>>>(a, (int)row_tiles);
            else attention_dq_kernel<DT, BLOCKS, KEYS, 1><<<dim3((unsigned)wq), dim3(256), 0, st>>>(a, (int)row_tiles);
        } else attention_dq_kernel<DT, BLOCKS, KEYS, 1><<<dim3((unsigned)wq), dim3(256), 0, st>>>(a, (int)row_tiles);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || wk == 0) return e;
    a.mix = a.splits == 1 ? mix_of(a, heads, kt) : 1;
    attention_dkdv_kernel<DT, BLOCKS, KEY_ROWS, W::waves, W::per_simd, W::v_in_lds, W::buffers><<<dim3((unsigned)wk), dim3(64 * W::waves), 0, st>>>(a, (int)kt);
    e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    attention_sum_kernel<DT><<<dim3((unsigned)ws, 2), dim3(256), 0, st>>>(a, 32 * W::waves, KEY_ROWS);
    return hipGetLastError();
}
inline size_t row_bytes(const AttnArg &a) { return ((size_t)a.B * a.Hq * a.Tq * 8 + 15) / 16 * 16; }

}  // namespace attn

// (the number of parts follows from the sizes and from whether the call is causal; a workspace holds either)
size_t attention_grad_workspace(const AttnArg &a)
{
    AttnArg b = a;
    b.causal = 1;
    attn::with_plan(b, [&](auto plan) { plan.plan(b); });
    return attn::row_bytes(a) + (b.splits == 1 ? 0 : (size_t)b.splits * 2 * a.B * a.Hk * a.Tk * a.D * 4);
}

hipError_t launch_attention_grad(AttnArg a, void *workspace, hipStream_t st)
{
    a.rows = (float2 *)workspace;
    a.part = (float *)((char *)workspace + attn::row_bytes(a));
    return attn::with_plan(a, [&](auto plan) {
        plan.plan(a);
        return attn::launch_grads(a, plan, st);
    });
}

}  // namespace nm
