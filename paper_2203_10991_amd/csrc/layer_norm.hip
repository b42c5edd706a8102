// Layer norm over the rows of x [R x C], and its gradients.
//     y = (x - mean) r w + b, r = 1 / sqrt(var + eps)
//     with h = (x - mean) r and u = g w:  dx = r (u - mean(u) - h mean(u h))      dw = sum over the rows of g h      db = sum of g
// A row is held in registers, 8 N elements to a thread, T threads to a row, so that it is read once; a workgroup goes through its rows with w, b and the next row's elements
// in registers (LEAN, for rows beyond 16384: registers hold the row and half of the sums; w and b are read again, sums of dw wait in LDS).  Mean and sum of squared deviations: in two steps within a wave, and between the waves of a row by the formula for joining two samples (one exchange).
// Sums of dw and db stay with the threads of a column; what a workgroup has goes to the workspace, and a second launch adds the workgroups' parts up in a fixed order.
// Bound: HBM.  32768 rows of 8192 in bf16 206 us forward (5.2 TB/s) and 314 + 8 for the gradients (5.1), 16384 of 1024 13.5 and 20 + 4 (5.0); a copy of 4.3 GB reaches 4.6.  Few rows: a launch, 2.5 us for one of 1024.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "gemm_plan.h"           // NM_CUS
#include "nm_internal.h"
#include "row_vec.h"

namespace nm {

namespace {

constexpr int NORM_T = 256;      // threads of a workgroup, or of a row if that has more

template <int LANES = 64> __device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// where piece n of thread t's elements lies: the last piece of a row ends with the row, `skip` of its elements are the piece's before it; left: elements that are there
struct Piece { int at, skip, left; };
template <int T> __device__ __forceinline__ Piece piece_of(int n, int t, int C)
{
    const int e = (n * T + t) * EW;
    Piece p;
    p.at = C >= EW ? min(e, C - EW) : 0;
    p.skip = min(e - p.at, EW);
    p.left = min(C, EW);
    if (C < EW && e >= C) p.skip = EW;
    return p;
}
template <int DT> __device__ __forceinline__ Raw<DT> load_piece(const void *row, const Piece &p, int C)
{
    return C >= EW ? load_raw<DT>(row, p.at) : load_raw<DT, true>(row, p.at, p.left);
}
template <int WT, int T> __device__ __forceinline__ void load_weights(float (&w)[EW], const void *from, int n, int t, int C, float missing)
{
    if (!from) {
#pragma unroll
        for (int i = 0; i < EW; ++i) w[i] = missing;
    } else {
        const Raw<WT> r = load_piece<WT>(from, piece_of<T>(n, t, C), C);
#pragma unroll
        for (int i = 0; i < EW; ++i) w[i] = element(r, i);
    }
}
template <int DT> __device__ __forceinline__ const void *row_from(const void *p, int64_t row, int64_t ld) { return (const char *)p + row * ld * (DT == NM_DT_BF16 ? 2 : 4); }

template <int DT, int WT, int T, int N, bool LEAN>
__global__ __launch_bounds__(T < NORM_T ? NORM_T : T) void layer_norm_kernel(const NormArg p)
{
    constexpr int THREADS = T < NORM_T ? NORM_T : T, ROWS = THREADS / T, WAVES = T > 64 ? T / 64 : 1, LANES = T < 64 ? T : 64;
    __shared__ float join[2][WAVES > 1 ? WAVES : 1][3];
    const int t = (int)threadIdx.x % T, C = (int)p.C;
    float w[LEAN ? 1 : N][EW], b[LEAN ? 1 : N][EW];
    if constexpr (!LEAN)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            load_weights<WT, T>(w[n], p.w, n, t, C, 1.0f);
            load_weights<WT, T>(b[n], p.b, n, t, C, 0.0f);
        }
    int mine = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Piece q = piece_of<T>(n, t, C);
        mine += max(0, q.left - q.skip);
    }
    const float count = WAVES > 1 ? wave_sum((float)mine) : (float)C, divisor = count > 0.0f ? count : 1.0f;
    int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / T;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    Raw<DT> next[N];
    if (!LEAN && row < p.R)
#pragma unroll
        for (int n = 0; n < N; ++n) next[n] = load_piece<DT>(row_from<DT>(p.x, row, p.ldx), piece_of<T>(n, t, C), C);
    // (rows of a workgroup with several waves to a row end together)
    for (int odd = 0; row < p.R; row += step, odd ^= 1) {
        if constexpr (LEAN)
#pragma unroll
            for (int n = 0; n < N; ++n) next[n] = load_piece<DT>(row_from<DT>(p.x, row, p.ldx), piece_of<T>(n, t, C), C);
        float x[N][EW];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < EW; ++i) x[n][i] = element(next[n], i);
        if (!LEAN && row + step < p.R)
#pragma unroll
            for (int n = 0; n < N; ++n) next[n] = load_piece<DT>(row_from<DT>(p.x, row + step, p.ldx), piece_of<T>(n, t, C), C);
        float sum = 0.0f, sq = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Piece q = piece_of<T>(n, t, C);
#pragma unroll
            for (int i = 0; i < EW; ++i)
                if (i >= q.skip && i < q.left) sum += x[n][i];
        }
        float mean = wave_sum<LANES>(sum) / divisor;                              // (a quotient: the mean of equal elements is theirs)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Piece q = piece_of<T>(n, t, C);
#pragma unroll
            for (int i = 0; i < EW; ++i)
                if (i >= q.skip && i < q.left) { const float d = x[n][i] - mean; sq += d * d; }
        }
        sq = wave_sum<LANES>(sq);
        if constexpr (WAVES > 1) {
            if ((t & 63) == 0) { join[odd][t >> 6][0] = count; join[odd][t >> 6][1] = mean; join[odd][t >> 6][2] = sq; }
            __syncthreads();
            float total = 0.0f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) total += join[odd][k][0] * join[odd][k][1];
            mean = total / (float)C;
            sq = 0.0f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) { const float d = join[odd][k][1] - mean; sq += join[odd][k][2] + join[odd][k][0] * d * d; }
        }
        const float r = 1.0f / sqrtf(sq / (float)C + p.eps);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Piece q = piece_of<T>(n, t, C);
            if (q.skip >= EW) continue;
            if constexpr (LEAN) {
                load_weights<WT, T>(w[0], p.w, n, t, C, 1.0f);
                load_weights<WT, T>(b[0], p.b, n, t, C, 0.0f);
            }
            float y[EW];
#pragma unroll
            for (int i = 0; i < EW; ++i) y[i] = __builtin_fmaf((x[n][i] - mean) * r, w[LEAN ? 0 : n][i], b[LEAN ? 0 : n][i]);
            store_row<DT>((void *)row_from<DT>(p.y, row, p.ldy), q.at, q.skip, q.left, y);
        }
        if (t == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = r;
        }
    }
}

template <int DT, int WT, int T, int N, bool LEAN>
__global__ __launch_bounds__(T < NORM_T ? NORM_T : T) void layer_norm_grad_kernel(const NormGradArg p)
{
    constexpr int THREADS = T < NORM_T ? NORM_T : T, ROWS = THREADS / T, WAVES = T > 64 ? T / 64 : 1, LANES = T < 64 ? T : 64;
    __shared__ float join[2][WAVES > 1 ? WAVES : 1][2];
    __shared__ float sums[ROWS > 1 ? ROWS - 1 : 1][ROWS > 1 ? T * EW : 1];
    __shared__ float dw_lds[LEAN ? N * EW * T : 1];
    const int t = (int)threadIdx.x % T, group = (int)threadIdx.x / T, C = (int)p.C;
    float w[LEAN ? 1 : N][EW], dw[LEAN ? 1 : N][EW], db[N][EW];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if constexpr (!LEAN) load_weights<WT, T>(w[n], p.w, n, t, C, 1.0f);
#pragma unroll
        for (int i = 0; i < EW; ++i) {
            db[n][i] = 0.0f;
            if constexpr (LEAN) dw_lds[(n * EW + i) * T + t] = 0.0f;
            else dw[n][i] = 0.0f;
        }
    }
    int64_t row = (int64_t)blockIdx.x * ROWS + group;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    Raw<DT> nx[N], ng[N];
    float nmean = 0.0f, nr = 0.0f;
    auto load = [&](int64_t at) {
        nmean = p.mean[at];
        nr = p.rstd[at];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            nx[n] = load_piece<DT>(row_from<DT>(p.x, at, p.ldx), piece_of<T>(n, t, C), C);
            ng[n] = load_piece<DT>(row_from<DT>(p.g, at, p.ldg), piece_of<T>(n, t, C), C);
        }
    };
    if (!LEAN && row < p.R) load(row);
    for (int odd = 0; row < p.R; row += step, odd ^= 1) {
        if constexpr (LEAN) load(row);
        const float mean = nmean, r = nr;
        Raw<DT> x[N], g[N];
#pragma unroll
        for (int n = 0; n < N; ++n) { x[n] = nx[n]; g[n] = ng[n]; }
        if (!LEAN && row + step < p.R) load(row + step);
        float su = 0.0f, suh = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Piece q = piece_of<T>(n, t, C);
            if constexpr (LEAN) load_weights<WT, T>(w[0], p.w, n, t, C, 1.0f);
#pragma unroll
            for (int i = 0; i < EW; ++i)
                if (i >= q.skip && i < q.left) {
                    const float h = (element(x[n], i) - mean) * r, gi = element(g[n], i), u = gi * w[LEAN ? 0 : n][i];
                    if constexpr (LEAN) dw_lds[(n * EW + i) * T + t] += gi * h;
                    else dw[n][i] += gi * h;
                    db[n][i] += gi;
                    su += u;
                    suh += u * h;
                }
        }
        su = wave_sum<LANES>(su);
        suh = wave_sum<LANES>(suh);
        if constexpr (WAVES > 1) {
            if ((t & 63) == 0) { join[odd][t >> 6][0] = su; join[odd][t >> 6][1] = suh; }
            __syncthreads();
            su = suh = 0.0f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) { su += join[odd][k][0]; suh += join[odd][k][1]; }
        }
        su /= (float)C;
        suh /= (float)C;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Piece q = piece_of<T>(n, t, C);
            if (q.skip >= EW) continue;
            if constexpr (LEAN) load_weights<WT, T>(w[0], p.w, n, t, C, 1.0f);
            float y[EW];
#pragma unroll
            for (int i = 0; i < EW; ++i) y[i] = (element(g[n], i) * w[LEAN ? 0 : n][i] - su - (element(x[n], i) - mean) * r * suh) * r;
            store_row<DT>((void *)row_from<DT>(p.dx, row, p.lddx), q.at, q.skip, q.left, y);
        }
    }
    if (!p.part) return;
    // the sums of the workgroup's groups of threads together, and to the workspace: [workgroup][dw, db][C]
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float d[EW];
#pragma unroll
            for (int i = 0; i < EW; ++i) {
                if (which) d[i] = db[n][i];
                else if constexpr (LEAN) d[i] = dw_lds[(n * EW + i) * T + t];
                else d[i] = dw[n][i];
            }
            if constexpr (ROWS > 1) {
                __syncthreads();
                if (group > 0)
#pragma unroll
                    for (int i = 0; i < EW; ++i) sums[group - 1][i * T + t] = d[i];
                __syncthreads();
                if (group > 0) continue;
                for (int k = 0; k < ROWS - 1; ++k)
#pragma unroll
                    for (int i = 0; i < EW; ++i) d[i] += sums[k][i * T + t];
            }
            const Piece q = piece_of<T>(n, t, C);
            if (q.skip < EW) store_row<NM_DT_F32>(p.part, ((int64_t)blockIdx.x * 2 + which) * C + q.at, q.skip, q.left, d);
        }
}

// column sums of the parts [parts][2 C]: 32 columns to a workgroup, 32 groups of threads with every 32nd part
template <int WT> __global__ __launch_bounds__(1024) void layer_norm_sum_kernel(const float *part, int parts, int C, void *dw, void *db)
{
    __shared__ float sums[32][33];
    const int c = (int)blockIdx.x * 32 + (threadIdx.x & 31), k = (int)threadIdx.x >> 5;
    float s = 0.0f;
    if (c < 2 * C)
#pragma unroll 8
        for (int j = k; j < parts; j += 32) s += part[(int64_t)j * 2 * C + c];
    sums[k][threadIdx.x & 31] = s;
    __syncthreads();
    if (k != 0 || c >= 2 * C) return;
    for (int j = 1; j < 32; ++j) s += sums[j][threadIdx.x];
    void *to = c < C ? dw : db;
    const int at = c < C ? c : c - C;
    if (!to) return;
    if constexpr (WT == NM_DT_F32) ((float *)to)[at] = s;
    else ((uint16_t *)to)[at] = (uint16_t)pack_bf16_rne(s, s);
}

template <int T, int N, bool LEAN = false> struct Shape { static constexpr int t = T, n = N, threads = T < NORM_T ? NORM_T : T, rows = threads / T; static constexpr bool lean = LEAN; };
// Threads to a row and pieces to a thread: part of a wave up to 256 elements, a wave up to 1024.  200000 rows of 64 in bf16: 60 us with a wave to a row, 12 with 8 threads.  LEAN: the
// gradients of binary32 rows of 8193 to 16384 elements (4096 x 16384: 251 us with 512 threads and 94 spills, 196 lean; in bf16 101 and 128).  Gradients of wider rows spill 32 to 74 registers
// of the 128 that 1024 threads have: 2048 x 32768 in bf16 169 us, 3.2 TB/s.
template <bool LEAN, typename F> auto with_shape(int64_t C, F &&f)
{
    if (C <= 64) return f(Shape<8, 1>{});
    if (C <= 128) return f(Shape<16, 1>{});
    if (C <= 256) return f(Shape<32, 1>{});
    if (C <= 512) return f(Shape<64, 1>{});
    if (C <= 1024) return f(Shape<64, 2>{});
    if (C <= 2048) return f(Shape<256, 1>{});
    if (C <= 4096) return f(Shape<256, 2>{});
    if (C <= 8192) return f(Shape<256, 4>{});
    if (C <= 16384) return f(std::conditional_t<LEAN, Shape<1024, 2, true>, Shape<512, 4>>{});
    return f(Shape<1024, 4, true>{});
}
// (a workgroup's sums are 8 C bytes out and in again: 512 rows of 16384 in 512 workgroups take 37 us, in 256 25)
inline int64_t grad_workgroups(int64_t R, int64_t C)
{
    const int64_t rows = with_shape<false>(C, [](auto s) { return (int64_t)decltype(s)::rows; }), wgs = (R + rows - 1) / rows;
    return std::min<int64_t>(wgs, (C > 16384 || wgs < 4 * NM_CUS ? 1 : 2) * NM_CUS);
}

}  // namespace

hipError_t launch_layer_norm(const NormArg &a, hipStream_t st)
{
    if (a.R <= 0) return hipSuccess;
    return with_shape<false>(a.C, [&](auto s) {
        typedef decltype(s) S;
        const unsigned wgs = (unsigned)std::min<int64_t>((a.R + S::rows - 1) / S::rows, 5 * NM_CUS);
        const dim3 threads(S::threads);
        if (a.x_dt == NM_DT_BF16) {
            if (a.w_dt == NM_DT_BF16) layer_norm_kernel<NM_DT_BF16, NM_DT_BF16, S::t, S::n, S::lean><<<wgs, threads, 0, st>>>(a);
            else layer_norm_kernel<NM_DT_BF16, NM_DT_F32, S::t, S::n, S::lean><<<wgs, threads, 0, st>>>(a);
        } else if (a.w_dt == NM_DT_BF16) layer_norm_kernel<NM_DT_F32, NM_DT_BF16, S::t, S::n, S::lean><<<wgs, threads, 0, st>>>(a);
        else layer_norm_kernel<NM_DT_F32, NM_DT_F32, S::t, S::n, S::lean><<<wgs, threads, 0, st>>>(a);
        return hipGetLastError();
    });
}

size_t layer_norm_grad_workspace(int64_t R, int64_t C) { return (size_t)grad_workgroups(R, C) * 2 * C * 4; }

hipError_t launch_layer_norm_grad(const NormGradArg &a, hipStream_t st)
{
    const int64_t wgs = grad_workgroups(a.R, a.C);
    hipError_t e = hipSuccess;
    if (wgs > 0 && a.x_dt == NM_DT_BF16)
        e = with_shape<false>(a.C, [&](auto s) {
            typedef decltype(s) S;
            if (a.w_dt == NM_DT_BF16) layer_norm_grad_kernel<NM_DT_BF16, NM_DT_BF16, S::t, S::n, S::lean><<<(unsigned)wgs, S::threads, 0, st>>>(a);
            else layer_norm_grad_kernel<NM_DT_BF16, NM_DT_F32, S::t, S::n, S::lean><<<(unsigned)wgs, S::threads, 0, st>>>(a);
            return hipGetLastError();
        });
    else if (wgs > 0)
        e = with_shape<true>(a.C, [&](auto s) {
            typedef decltype(s) S;
            if (a.w_dt == NM_DT_BF16) layer_norm_grad_kernel<NM_DT_F32, NM_DT_BF16, S::t, S::n, S::lean><<<(unsigned)wgs, S::threads, 0, st>>>(a);
            else layer_norm_grad_kernel<NM_DT_F32, NM_DT_F32, S::t, S::n, S::lean><<<(unsigned)wgs, S::threads, 0, st>>>(a);
            return hipGetLastError();
        });
    if (e != hipSuccess || !a.part) return e;
    const unsigned sums = (unsigned)((2 * a.C + 31) / 32);
    if (a.w_dt == NM_DT_BF16) layer_norm_sum_kernel<NM_DT_BF16><<<sums, 1024, 0, st>>>(a.part, (int)wgs, (int)a.C, a.dw, a.db);
    else layer_norm_sum_kernel<NM_DT_F32><<<sums, 1024, 0, st>>>(a.part, (int)wgs, (int)a.C, a.dw, a.db);
    return hipGetLastError();
}

}  // namespace nm
