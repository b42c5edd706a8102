// Product of 8-bit integers with a scale for each token and each output channel (T = M tokens, N outputs, K inputs):
//     y[M x N] = act((x[M x K] w[N x K]^T) xs[M] ws[N] + bias[N])
// 32-bit integer sums (K at most 131072: 127 * 128 K stays below 2^31; -128 against -128 does up to K = 131071), then one conversion, the product with xs ws, bias
// and ReLU in binary32, one rounding.
//
// Instruction: v_mfma_i32_32x32x32_i8, both operands with 32 rows (lane % 32) and 16 consecutive bytes of the reduction axis to a lane.  Which of the 32 steps
// of the axis those are does not matter, since both operands hold the same ones.  bf16 results: the weights are the first operand, so a lane holds four
// consecutive features of a token and stores them together.  binary32 results: x is the first one, and the lanes of half a wave store 32 features of a token.
//
// Workgroup = WM x WN waves, each AM x AN blocks of 32 tokens x 32 features.  The reduction axis advances in stages of 128 bytes, NS of which rotate through
// LDS, filled by direct loads.  A row of a stage is eight chunks of 16 bytes, chunk c at position c ^ (row / 2 % 8), which makes the 16-byte reads
// of consecutive rows free of bank conflicts.  A workgroup takes tiles one after the other, and the stages run on across them.
// A stage is four MFMA steps.  Behind the second the next stage has to have landed (one barrier) and this stage's last fragments are in
// registers, so its buffer is free and the loads of the stage NS later go there; the next stage's first fragments are read under the last two steps.
// x has zeros from K to the next whole stage, so whatever stands there in w's rows, or in LDS where w's chunks are not loaded, adds nothing: the rows of a layer's
// call hold them, those of a caller's own codes get them in LDS when the stage has landed.
//
// Bound: 32768 x 8192 -> 28672 the matrix pipelines under the power limit, 6.37 to 6.44 ms, 2.4 POP/s (the vendor's product with raw 32-bit results 6.78 ms).
// 16384 x 1024 -> 4096 in bf16 82 us (vendor's, raw, 97): the eight stages of a tile take 59, what a tile's results take is the rest (their stores alone 8 to 14).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "nm_internal.h"
#include "gemm_plan.h"
#include "smfmac_common.h"
#include "prune_common.h"        // pack_bf16_rne

namespace nm {

namespace {

// (the sums are 32-bit integers; the type only names the registers)
__device__ __forceinline__ void mfma_i8_32x32x32(f32x16 &acc, const u32x4 &a, const u32x4 &b)
{
    asm volatile("v_mfma_i32_32x32x32_i8 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
// zeros into the registers the block lives in
__device__ __forceinline__ void acc_clear(f32x16 &acc)
{
    const bf16x8 z = {0, 0, 0, 0, 0, 0, 0, 0};
    asm volatile("s_nop 4\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %1, 0" : "+a"(acc) : "v"(z));
}

// one sum of a block.  (Read by itself: left to the compiler whole blocks are copied first, to registers that it has not got.)
__device__ __forceinline__ float sum_of(float acc)
{
    int sum;
    asm("v_accvgpr_read_b32 %0, %1" : "=v"(sum) : "a"(acc));
    return (float)sum;
}

struct I8Tiles { I8Arg a; int tiles_m, tiles_n; };

// eight bf16 features of a token, of which `left` are there (WHOLE: all or none).  Rows start anywhere: the stores of whole groups need
// no alignment.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(2)));
template <bool WHOLE> __device__ __forceinline__ void store_features(char *at, int left, const u32x4 &v)
{
    if (WHOLE ? left > 0 : left >= 8) *(u32x4_any *)at = v;
    else if (!WHOLE && left > 0) {
        uint32_t w0 = v[0], w1 = v[1];
        if (left & 4) { *(u32x2_any *)at = u32x2{w0, w1}; at += 8; w0 = v[2]; w1 = v[3]; }
        if (left & 2) { *(u32_any *)at = w0; at += 4; w0 = w1; }
        if (left & 1) *(uint16_t *)at = (uint16_t)w0;
    }
}
// WHOLE: N is a multiple of 8 (bf16 results only)
template <int WM, int WN, int AM, int AN, int NS, int OT, bool WHOLE>
__global__ __launch_bounds__(WM * WN * 64) void gemm_i8_kernel(I8Tiles p)
{
    constexpr int NW = WM * WN, TM = WM * AM * 32, TN = WN * AN * 32;
    constexpr int X_BYTES = TM * I8_K, STAGE = X_BYTES + TN * I8_K;
    constexpr int RPL = 8;                                                       // rows of a direct load
    constexpr int XL = TM / RPL / NW, WL = TN / RPL / NW, LPS = XL + WL;         // direct loads of a wave and stage
    constexpr int LDS = NS * STAGE;
    using OutT = std::conditional_t<OT == NM_DT_F32, float, uint16_t>;
    static_assert(XL >= 1 && WL >= 1 && TM % (RPL * NW) == 0 && TN % (RPL * NW) == 0 && TM <= NW * 64 && TN <= NW * 64 && LDS + 3 * NW * 256 <= 160 * 1024, "tile");
    __shared__ __attribute__((aligned(1024))) char S[LDS];
    __shared__ __attribute__((aligned(16))) float tile_xs[NW * 64], tile_ws[NW * 64], tile_add[NW * 64];       // scales and bias of the tile that leaves

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN, hi = lane >> 5, l32 = lane & 31;
    const int n = (int)((p.a.K + I8_K - 1) / I8_K);                               // stages of a tile
    const int tiles = p.tiles_m * p.tiles_n;
    auto place = [&](int tile, int64_t &m0, int64_t &n0) {
        int tm, tn;
        tile_of_workgroup(tile, p.tiles_m, p.tiles_n, tm, tn);
        m0 = (int64_t)__builtin_amdgcn_readfirstlane(tm) * TM;
        n0 = (int64_t)__builtin_amdgcn_readfirstlane(tn) * TN;
    };

    f32x16 acc[AM][AN];
#pragma unroll
    for (int a = 0; a < AM; ++a)
#pragma unroll
        for (int b = 0; b < AN; ++b) acc_zero(acc[a][b]);

    // ---- direct loads: load d of a wave covers 1 KB of the stage's image at (wave * XL + d) KB, resp. (wave * WL + d) KB behind the x tile.  Rows past
    // the end are clamped to the last one, their results are not stored; the buffer of w ends with the last row's last chunk of 16 bytes.
    const int r_load = lane >> 3, pos = lane & 7;
    uint32_t x_src[XL], w_src[WL];
    auto key_of = [](int row) { return (row >> 1) & 7; };
    auto chunk_of = [&](int row) { return pos ^ key_of(row); };
    // the tile and stage whose loads are being issued
    int f_tile = blockIdx.x, f_stage = 0;
    const char *xp, *wp;
    int64_t x_left, w_left;                                                      // bytes from xp and wp to the end of x and w
    auto enter_tile = [&]() {
        int64_t m0, n0;
        place(f_tile, m0, n0);
        const int rows_x = (int)min(p.a.M - 1 - m0, (int64_t)TM), rows_w = (int)min(p.a.N - 1 - n0, (int64_t)TN);
#pragma unroll
        for (int d = 0; d < XL; ++d) {
            const int row = (wave * XL + d) * RPL + r_load;
            x_src[d] = (uint32_t)min(row, rows_x) * (uint32_t)p.a.ldx + (uint32_t)chunk_of(row) * 16u;
        }
#pragma unroll
        for (int d = 0; d < WL; ++d) {
            const int row = (wave * WL + d) * RPL + r_load;
            w_src[d] = (uint32_t)min(row, rows_w) * (uint32_t)p.a.ldw + (uint32_t)chunk_of(row) * 16u;
        }
        xp = (const char *)(p.a.x + m0 * p.a.ldx);
        wp = (const char *)(p.a.w + n0 * p.a.ldw);
        x_left = (p.a.M - 1 - m0) * p.a.ldx + (p.a.x_zeros ? (int64_t)n * I8_K : (p.a.K + 15) / 16 * 16);
        w_left = (p.a.N - 1 - n0) * p.a.ldw + (p.a.K + 15) / 16 * 16;
    };
    enter_tile();
    auto next_stage = [&]() {
        xp += I8_K; wp += I8_K; x_left -= I8_K; w_left -= I8_K;
        if (++f_stage == n) {
            f_stage = 0;
            f_tile += gridDim.x;
            if (f_tile < tiles) enter_tile();
        }
    };
    auto rsrc = [&](const char *base, int64_t bytes) {
        return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, f_tile < tiles ? (int)max(min(bytes, (int64_t)0x7fffffff), (int64_t)0) : 0, 0x00020000);
    };
    auto fetch_one = [&](auto k_c, int buf) {
        constexpr int K = decltype(k_c)::value;
        char *stage = S + buf * STAGE;
        if constexpr (K < XL) load16_to_lds(rsrc(xp, x_left), stage + (wave * XL + K) * 1024, x_src[K], 0);
        else                  load16_to_lds(rsrc(wp, w_left), stage + X_BYTES + (wave * WL + K - XL) * 1024, w_src[K - XL], 0);
    };

    // zeros behind K in the chunks of x that a wave has loaded for the last stage
    const int k_last = p.a.x_zeros ? I8_K : (int)(p.a.K - (int64_t)(n - 1) * I8_K);
    auto clear_tail = [&](int buf) {
        for (int d = 0; d < XL; ++d) {
            const int left = k_last - chunk_of((wave * XL + d) * RPL + r_load) * 16;       // bytes of the lane's chunk that count
            if (left < 16) {
                u32x4 *at = (u32x4 *)(S + buf * STAGE + (wave * XL + d) * 1024 + lane * 16), v = *at;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] &= left >= 4 * j + 4 ? 0xffffffffu : left <= 4 * j ? 0u : (1u << (8 * (left - 4 * j))) - 1u;
                *at = v;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };

    // ---- LDS reads
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr_t)S;
    const uint32_t rd = lds0 + (uint32_t)(l32 * I8_K + (hi ^ key_of(l32)) * 16);   // a row's chunk of MFMA step 0; that of step kk is chunk 2 kk + hi: bits 5 and 6 turned
    const uint32_t x_base = (uint32_t)(wm * AM * 32 * I8_K), w_base = (uint32_t)(X_BYTES + wn * AN * 32 * I8_K);
    u32x4 xf[2][AM], wf[2][AN];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int a = 0; a < AM; ++a) xf[s][a] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int b = 0; b < AN; ++b) wf[s][b] = u32x4{0, 0, 0, 0};
    }
    constexpr int READS = AM + AN;
    static_assert(READS <= 15, "counter of LDS reads");
    auto read = [&](auto kk_c, int buf) {                                        // fragments of MFMA step kk, into set kk % 2
        constexpr int kk = decltype(kk_c)::value, set = kk % 2;
        const uint32_t at = (rd ^ (32u * kk)) + (uint32_t)(buf * STAGE), xa = at + x_base, wa = at + w_base;
        static_for<AM>([&](auto a_c) { constexpr int a = decltype(a_c)::value; lds_refill_b128<a * 32 * I8_K>(xf[set][a], xa); });
        static_for<AN>([&](auto b_c) { constexpr int b = decltype(b_c)::value; lds_refill_b128<b * 32 * I8_K>(wf[set][b], wa); });
    };
    // The fragments on their way are in their registers.  Stands wherever compiled code lies between a read and the wait for it, which at a loop's head
    // moves fragments to other registers (and would move what was there before); the empty statements keep the registers theirs until then.
    auto reads_landed = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int a = 0; a < AM; ++a) asm volatile("" : : "v"(xf[s][a]));
#pragma unroll
            for (int b = 0; b < AN; ++b) asm volatile("" : : "v"(wf[s][b]));
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // the same of the accumulators and the matrix pipeline
    auto sums_settled = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
        for (int a = 0; a < AM; ++a)
#pragma unroll
            for (int b = 0; b < AN; ++b) acc_settled(acc[a][b]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // MFMA step kk; the loads [lo, hi) of a stage are spread behind its MFMAs
    auto step = [&](auto kk_c, auto lo_c, auto hi_c, int buf) {
        constexpr int set = decltype(kk_c)::value % 2, lo = decltype(lo_c)::value, n_l = decltype(hi_c)::value - lo, NM = AM * AN;
        static_for<NM>([&](auto i_c) {
            constexpr int i = decltype(i_c)::value, a = i / AN, b = i % AN;
            if constexpr (OT == NM_DT_F32) mfma_i8_32x32x32(acc[a][b], xf[set][a], wf[set][b]);
            else                           mfma_i8_32x32x32(acc[a][b], wf[set][b], xf[set][a]);
            static_for<LPS>([&](auto k_c) {
                constexpr int k = decltype(k_c)::value;
                if constexpr (k >= lo && k < lo + n_l && (k - lo) * NM / n_l == i) fetch_one(k_c, buf);
            });
        });
    };
    using std::integral_constant;
    using I0 = integral_constant<int, 0>; using I1 = integral_constant<int, 1>; using I2 = integral_constant<int, 2>; using I3 = integral_constant<int, 3>;

    for (int s = 0; s < NS; ++s) {
        static_for<LPS>([&](auto k_c) { fetch_one(k_c, s); });
        next_stage();
    }
    wait_vmcnt<(NS - 1) * LPS>();
    if (n == 1 && k_last < I8_K) clear_tail(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(I0{}, 0);
    read(I1{}, 0);
    int buf = 0, s = 0, tile = blockIdx.x;                                       // the stage that is multiplied: its buffer, its number in its tile
    // Scales and bias of the tile: every thread takes one of each, wanted or not, in the tile's last stage, ahead of the wait for the loads there
    float my_xs = 0.f, my_ws = 0.f;
    uint32_t my_add = 0;                                                         // as it is stored: what is made of a load waits for it
    auto take_scales = [&]() {
        int64_t m0, n0;
        place(tile, m0, n0);
        int t = tid;
        asm volatile("" : "+v"(t));                                              // (computed here, tile by tile)
        const int64_t f = min(n0 + min(t, TN - 1), p.a.N - 1);
        my_xs = p.a.xs[min(m0 + min(t, TM - 1), p.a.M - 1)];
        my_ws = p.a.ws[f];
        if (p.a.bias) my_add = p.a.bias_dt == NM_DT_F32 ? ((const uint32_t *)p.a.bias)[f] : ((const uint16_t *)p.a.bias)[f];
    };
    // a stage's first half; behind it every read has landed, so that the loop below closes with none on its way
    auto open = [&]() {
        const int next = buf == NS - 1 ? 0 : buf + 1;
        if (s == n - 1) take_scales();
        asm volatile("s_waitcnt lgkmcnt(%0)" : : "n"(READS) : "memory");
        step(I0{}, I0{}, I0{}, 0);
        read(I2{}, buf);
        asm volatile("s_waitcnt lgkmcnt(%0)" : : "n"(READS) : "memory");
        step(I1{}, I0{}, I0{}, 0);
        read(I3{}, buf);
        // the next stage (of this tile or the next) has landed, and every wave has read all of this one.  (Loads are counted down in the order they
        // were issued, and the stores of the tile before with them.  At a tile's first stage those are younger than the loads that are
        // waited for, so that more has to have landed than is needed; from then on they are older.)
        wait_vmcnt<(NS - 2) * LPS>();
        reads_landed();
        if (k_last < I8_K && (s + 1 == n ? 0 : s + 1) == n - 1) clear_tail(next);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    open();
    for (;;) {
        const int next = buf == NS - 1 ? 0 : buf + 1;
        step(I2{}, I0{}, integral_constant<int, LPS / 2>{}, buf);
        read(I0{}, next);
        step(I3{}, integral_constant<int, LPS / 2>{}, integral_constant<int, LPS>{}, buf);
        read(I1{}, next);
        next_stage();
        buf = next;
        if (++s == n) {
            // The tile leaves while the next one's first stages are on their way.  The matrix pipeline has to be done with it first, and the reads of the
            // next tile's first fragments with their registers.
            s = 0;
            int64_t m0, n0;
            place(tile, m0, n0);
            reads_landed();
            sums_settled();
            // (what follows from these is computed here, tile by tile: left to itself the compiler keeps it in registers through the stages, which have none left)
            int l32 = lane & 31, hi = lane >> 5, tid = wave * 64 + lane;
            asm volatile("" : "+v"(l32), "+v"(hi), "+v"(tid));
            tile_xs[tid] = my_xs; tile_ws[tid] = my_ws; tile_add[tid] = __uint_as_float(p.a.bias_dt == NM_DT_BF16 ? my_add << 16 : my_add);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            const int rows = (int)min(p.a.M - m0, (int64_t)TM), cols = (int)min(p.a.N - n0, (int64_t)TN);
            char *y0 = (char *)((OutT *)p.a.y + m0 * p.a.ldy + n0);
            const float least = p.a.relu ? 0.f : -__builtin_inff();
            if constexpr (OT == NM_DT_F32) {
                // a lane holds the tokens 8 g + 4 hi .. + 3 of feature l32 of each block.  What is not there is sent out of the buffer's range, which drops it: branches
                // here cost the accumulators their registers.
                const auto y_buffer = __builtin_amdgcn_make_buffer_rsrc((void *)y0, 0, 0x7fffffff, 0x00020000);
                const uint32_t row_bytes = (uint32_t)p.a.ldy * 4u;
#pragma unroll
                for (int b = 0; b < AN; ++b) {
                    const int f = (wn * AN + b) * 32 + l32;
                    const float ws = tile_ws[f], add = tile_add[f];
#pragma unroll
                    for (int a = 0; a < AM; ++a) {
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const int row = (wm * AM + a) * 32 + 8 * g + 4 * hi;
                            const float4 xs = *(const float4 *)&tile_xs[row];
                            const float x4[4] = {xs.x, xs.y, xs.z, xs.w};
                            const uint32_t at = (uint32_t)row * row_bytes + (uint32_t)f * 4u;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                float v = sum_of(acc[a][b][4 * g + j]) * (x4[j] * ws) + add;
                                v = v <= least ? least : v;                          // (a NaN stays one)
                                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), y_buffer, row + j < rows && f < cols ? (int)(at + (uint32_t)j * row_bytes) : -1, 0, 0);
                            }
                            __builtin_amdgcn_sched_barrier(0);
                        }
                        acc_clear(acc[a][b]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            } else {
                // A lane holds four features of every eight of a token.  The halves of the wave exchange, so that it holds eight in a row, and their quarters then, so that four
                // lanes hold the 64 bytes that a block has of a token; the neighbouring blocks' follow at once.  (Stores of 32 bytes of a token: 16384 x 1024 -> 4096
                // 99 us, blocks apart 132.)
                const int q = tid & 63, chunk = (q >> 4 & 1) * 2 + (q >> 5), l16 = q & 15;
#pragma unroll
                for (int a = 0; a < AM; ++a) {
                    const int row = (wm * AM + a) * 32 + l16;
                    const float xs = tile_xs[(wm * AM + a) * 32 + l32];
                    const uint32_t at_row = (uint32_t)row * (uint32_t)p.a.ldy * 2u, half = (uint32_t)p.a.ldy * 32u;
#pragma unroll
                    for (int b = 0; b < AN; ++b) {
                        u32x4 r[2];
#pragma unroll
                        for (int g = 0; g < 4; g += 2) {
                            uint32_t w[2][2];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const int f0 = (wn * AN + b) * 32 + 8 * (g + i) + 4 * hi;
                                const float4 ws = *(const float4 *)&tile_ws[f0], add = *(const float4 *)&tile_add[f0];
                                const float w4[4] = {ws.x, ws.y, ws.z, ws.w}, b4[4] = {add.x, add.y, add.z, add.w};
                                float v[4];
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const float t = sum_of(acc[a][b][4 * (g + i) + j]) * (xs * w4[j]) + b4[j];
                                    v[j] = t <= least ? least : t;                   // (a NaN stays one)
                                }
                                w[i][0] = pack_bf16_rne(v[0], v[1]);
                                w[i][1] = pack_bf16_rne(v[2], v[3]);
                            }
                            const auto lo = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false), up = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
                            r[g / 2] = u32x4{lo[0], up[0], lo[1], up[1]};
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const auto both = __builtin_amdgcn_permlane16_swap(r[0][i], r[1][i], false, false);
                            r[0][i] = both[0];
                            r[1][i] = both[1];
                        }
                        const int f = (wn * AN + b) * 32 + 8 * chunk;
                        if (row < rows) store_features<WHOLE>(y0 + at_row + (uint32_t)f * 2u, cols - f, r[0]);
                        if (row + 16 < rows) store_features<WHOLE>(y0 + at_row + half + (uint32_t)f * 2u, cols - f, r[1]);
                        acc_clear(acc[a][b]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
            sums_settled();                                                          // (of the zeros)
            tile += gridDim.x;
            // the next tile's first fragments again, so that their registers are the epilogue's
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int a = 0; a < AM; ++a) xf[k][a] = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int b = 0; b < AN; ++b) wf[k][b] = u32x4{0, 0, 0, 0};
            }
            read(I0{}, buf);
            read(I1{}, buf);
        }
        if (tile >= tiles) break;
        open();
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");                  // what ran ahead
}

}  // namespace

// The tile whose time a model puts lowest: rounds of one or two tiles to a CU (`per_cu`), a round's stages in us at one tile to a CU (`alone`) and with every place
// taken (`shared`), and what a round costs besides (`round`, and `round_f32` where the results are binary32).  Fitted to sweeps of all five over products of 65 to
// 16384 tokens whose operands were in the caches; what the model takes is 0.3 % from the best.  (us, 64 x 64 / 128 x 64 / 128 x 128 two to a CU / one / 256 x 256:
// 512 x 1024 -> 1024 7.5 / 8.4 / 10.0 / 10.0 / 18.5, 2048 x 2048 -> 2048 22.9 / 17.2 / 16.7 / 16.3 / 29.2, 2048 x 1024 -> 4096 26.2 / 19.4 / 16.4 / 18.5 /
// 21.5, 4096 x 4096 -> 4096 136 / 99 / 77 / 87 / 65, 16384 x 1024 -> 4096 166 / 127 / 99 / 115 / 82.)
// Few tokens or features go to gemm_i8_few.hip where its own model's time is the lower one; 4.1 + 1.6 times is what this one's become with weights that
// come from memory.
hipError_t launch_gemm_i8(const I8Arg &a, hipStream_t st)
{
    if (a.M == 0 || a.N == 0) return hipSuccess;
    I8Tiles p{a, 0, 0};
    struct Tile { int tm, tn, per_cu; double alone, shared, round, round_f32; };
    constexpr Tile tiles[5] = {{64, 64, 2, 0.20, 0.45, 0.58, 0.62}, {128, 64, 2, 0.23, 0.59, 0.99, 0.65}, {128, 128, 2, 0.58, 0.78, 1.51, 2.05}, {128, 128, 1, 0.41, 0.51, 1.13, 0.69},
                               {256, 256, 1, 1.00, 1.13, 3.4, 12.5}};
    const double stages = (double)((a.K + I8_K - 1) / I8_K);
    int best = 0;
    double least = 1e300;
    for (int i = 0; i < 5; ++i) {
        const Tile &t = tiles[i];
        if (i > 0 && a.M <= 64) continue;                                        // (half of the rows would be nobody's: 16 x 8192 -> 28672 50 us against 54 to 103)
        const int64_t n = ((a.M + t.tm - 1) / t.tm) * ((a.N + t.tn - 1) / t.tn), whole = (int64_t)t.per_cu * NM_CUS, left = n % whole;
        const double round = a.y_dt == NM_DT_F32 ? t.round_f32 : t.round;
        const double part = t.per_cu == 1 ? t.alone + (t.shared - t.alone) * (double)left / NM_CUS : left <= NM_CUS ? t.alone : t.shared;
        const double cost = (double)(n / whole) * (stages * t.shared + round) + (left ? stages * part + round : 0.0);
        if (cost < least) { least = cost; best = i; }
    }
    if (gemm_i8_few_plan(a.M, a.N, a.K).us < 4.1 + 1.6 * least) return launch_gemm_i8_few(a, nullptr, 0, 0, st);
    const int64_t tm = (a.M + tiles[best].tm - 1) / tiles[best].tm, tn = (a.N + tiles[best].tn - 1) / tiles[best].tn, n_tiles = tm * tn;
    if (n_tiles > 0x7fffffffll - 1024) return hipErrorInvalidConfiguration;
    p.tiles_m = (int)tm;
    p.tiles_n = (int)tn;
    const int64_t wgs = std::min<int64_t>(n_tiles, (int64_t)tiles[best].per_cu * NM_CUS);
#define NM_I8_W(WM, WN, AM, AN, NS, OT, WHOLE) hipLaunchKernelGGL((gemm_i8_kernel<WM, WN, AM, AN, NS, OT, WHOLE>), dim3((unsigned)wgs), dim3(WM * WN * 64), 0, st, p)
#define NM_I8(WM, WN, AM, AN, NS)                                                             \
    do {                                                                                          \
        if (a.y_dt == NM_DT_F32) NM_I8_W(WM, WN, AM, AN, NS, NM_DT_F32, false);               \
        else if (a.N % 8 == 0) NM_I8_W(WM, WN, AM, AN, NS, NM_DT_BF16, true);                 \
        else NM_I8_W(WM, WN, AM, AN, NS, NM_DT_BF16, false);                                  \
    } while (0)
    switch (best) {
    case 0: NM_I8(2, 2, 1, 1, 4); break;
    case 1: NM_I8(2, 2, 2, 1, 3); break;
    case 2: NM_I8(2, 2, 2, 2, 2); break;
    case 3: NM_I8(2, 4, 2, 1, 4); break;
    default: NM_I8(2, 4, 4, 2, 2); break;
    }
#undef NM_I8
#undef NM_I8_W
    return hipGetLastError();
}

}  // namespace nm
