// Embedding: rows of a table by token, scaled, and the table's gradient.
//     out[n] = scale E[id_n]                     dE[v] = scale * sum over the tokens n with id_n = v of g[n], in the order of n
// The gradient's tokens are sorted by id, stably, and each row's sum runs over its tokens in their order in binary32: the result does not depend on the
// launch, and a row that half of the tokens share costs no more than as many rows with a token each.
//   sort    up to RANK_MOST tokens, one launch: the rank of a token is the number of tokens whose (id, position) is smaller, which 64 x 4 threads count
//           for 64 tokens from LDS.  Beyond, radix passes of at most 9 bits, a counting launch and a moving one each.
//           Workgroups behind those of the first launch fill the gradient with zeros meanwhile.
//   sum     a workgroup takes CHUNK consecutive tokens of the sorted list and a slab of columns.  Rows whose tokens all lie inside are written; the sums of
//           a row that began in an earlier chunk, or runs on into the next one, go to the workspace.
//   join    those rows: the chunk where a row begins adds up its parts, chunk after chunk.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "nm_internal.h"
#include "prune_common.h"        // Row, pack_bf16_rne

namespace nm {

namespace {

__device__ __forceinline__ int64_t id_at(const void *ids, bool wide, int64_t n)
{
    return wide ? ((const int64_t *)ids)[n] : (int64_t)((const int32_t *)ids)[n];
}

// W elements of a row as binary32, and back.  VEC: W elements fill 16 bytes of the wider of the two types, on a boundary of their size.
template <int DT, int W, bool VEC> __device__ __forceinline__ void load_row(const void *p, int64_t at, int left, float (&v)[W])
{
    if constexpr (VEC && DT == NM_DT_F32) {
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            const float4 x = *(const float4 *)((const float *)p + at + i);
            v[i] = x.x; v[i + 1] = x.y; v[i + 2] = x.z; v[i + 3] = x.w;
        }
    } else if constexpr (VEC && W == 8) {
        const uint4 x = *(const uint4 *)((const uint16_t *)p + at);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = Row<NM_DT_BF16>::get(x, i);
    } else if constexpr (VEC) {
        const uint2 x = *(const uint2 *)((const uint16_t *)p + at);
        v[0] = __uint_as_float(x.x << 16); v[1] = __uint_as_float(x.x & 0xffff0000u); v[2] = __uint_as_float(x.y << 16); v[3] = __uint_as_float(x.y & 0xffff0000u);
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            v[i] = 0.f;
            if (i < left) v[i] = DT == NM_DT_F32 ? ((const float *)p)[at + i] : __uint_as_float((uint32_t)((const uint16_t *)p)[at + i] << 16);
        }
    }
}
template <int DT, int W, bool VEC> __device__ __forceinline__ void store_row(void *p, int64_t at, int left, const float (&v)[W])
{
    if constexpr (VEC && DT == NM_DT_F32) {
#pragma unroll
        for (int i = 0; i < W; i += 4) *(float4 *)((float *)p + at + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else if constexpr (VEC && W == 8) {
        *(uint4 *)((uint16_t *)p + at) = make_uint4(pack_bf16_rne(v[0], v[1]), pack_bf16_rne(v[2], v[3]), pack_bf16_rne(v[4], v[5]), pack_bf16_rne(v[6], v[7]));
    } else if constexpr (VEC) {
        *(uint2 *)((uint16_t *)p + at) = make_uint2(pack_bf16_rne(v[0], v[1]), pack_bf16_rne(v[2], v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < left) {
                if constexpr (DT == NM_DT_F32) ((float *)p)[at + i] = v[i];
                else                           ((uint16_t *)p)[at + i] = (uint16_t)pack_bf16_rne(v[i], v[i]);
            }
    }
}

constexpr int EW = 8;            // elements of a row that a thread takes at a time: 16 bytes of bf16, 32 of binary32

// ---- lookup: 2^shift threads to a row
template <int TT, int OT, bool VEC>
__global__ __launch_bounds__(256) void embed_kernel(const void *table, int64_t V, int64_t D, int64_t ldt, const void *ids, bool wide, int64_t N, float scale,
                                                    void *out, int64_t ldo, int shift)
{
    const int64_t n = (int64_t)blockIdx.x * (256 >> shift) + (threadIdx.x >> shift);
    if (n >= N) return;
    const int64_t id = id_at(ids, wide, n);
    const bool there = id >= 0 && id < V;                            // (a token outside the table: a row of NaN, nothing is read)
    const int64_t step = (int64_t)EW << shift;
    for (int64_t c = (int64_t)(threadIdx.x & ((1 << shift) - 1)) * EW; c < D; c += step) {
        const int left = (int)min(D - c, (int64_t)EW);
        float v[EW];
        if (there) {
            if (VEC && left == EW) load_row<TT, EW, true>(table, id * ldt + c, left, v); else load_row<TT, EW, false>(table, id * ldt + c, left, v);
#pragma unroll
            for (int i = 0; i < EW; ++i) v[i] *= scale;
        } else
#pragma unroll
            for (int i = 0; i < EW; ++i) v[i] = __uint_as_float(0x7fc00000u);
        if (VEC && left == EW) store_row<OT, EW, true>(out, n * ldo + c, left, v); else store_row<OT, EW, false>(out, n * ldo + c, left, v);
    }
}

// ---- the gradient's sort
constexpr int64_t RANK_MOST = 8192;
constexpr int RADIX_BITS = 9, RADIX_BINS = 1 << RADIX_BITS, KEYS = 2048;     // keys of a workgroup in a radix pass: KEYS or a multiple

struct Fill { char *at; int64_t rows, row_bytes, stride_bytes; };            // rows that become zeros; rows == 0: none
// rows are taken as one run of bytes where they are contiguous
__device__ void fill_zeros(const Fill &f, int64_t wg, int64_t wgs)
{
    const int64_t tid = wg * blockDim.x + threadIdx.x, all = wgs * blockDim.x;
    if (f.row_bytes == f.stride_bytes && ((uintptr_t)f.at & 15) == 0) {
        const int64_t bytes = f.rows * f.row_bytes, n = bytes / 16;
        const uint4 z = make_uint4(0, 0, 0, 0);
        for (int64_t i = tid; i < n; i += all) ((uint4 *)f.at)[i] = z;
        for (int64_t i = n * 16 + 2 * tid; i < bytes; i += 2 * all) *(uint16_t *)(f.at + i) = 0;
    } else {
        for (int64_t r = wg; r < f.rows; r += wgs)
            for (int64_t i = 2 * threadIdx.x; i < f.row_bytes; i += 2 * blockDim.x) *(uint16_t *)(f.at + r * f.stride_bytes + i) = 0;
    }
}

// the key of a token: its id, or V where it counts for nothing
__device__ __forceinline__ uint32_t key_of(const void *ids, bool wide, int64_t n, int64_t V, int64_t padding)
{
    const int64_t id = id_at(ids, wide, n);
    return id < 0 || id >= V || id == padding ? (uint32_t)V : (uint32_t)id;
}

// rank by counting: N <= RANK_MOST tokens, 13 bits of position behind the id's
__global__ __launch_bounds__(256) void embed_rank_kernel(const void *ids, bool wide, int N, int64_t V, int64_t padding, int sort_wgs, uint32_t *keys, uint32_t *perm, Fill f)
{
    if ((int)blockIdx.x >= sort_wgs) { fill_zeros(f, (int)blockIdx.x - sort_wgs, (int)gridDim.x - sort_wgs); return; }
    extern __shared__ __attribute__((aligned(16))) uint2 all[];              // (position, key) of each token
    __shared__ int rank[64];
    const int tid = threadIdx.x, lane = tid & 63, part = tid >> 6;
    const int padded = (N + 7) & ~7;
    for (int n = tid; n < padded; n += 256) all[n] = n < N ? make_uint2((uint32_t)n, key_of(ids, wide, n, V, padding)) : make_uint2(0xffffffffu, 0xffffffffu);
    if (tid < 64) rank[tid] = 0;
    __syncthreads();
    const int mine = (int)blockIdx.x * 64 + lane;
    if (mine < N) {
        const uint2 me = all[mine];
        const uint64_t key = (uint64_t)me.y << 32 | me.x;
        int below = 0;
        for (int i = part * 2; i < padded; i += 8) {                         // two entries a read
            const uint4 v = *(const uint4 *)&all[i];
            below += ((uint64_t)v.y << 32 | v.x) < key;
            below += ((uint64_t)v.w << 32 | v.z) < key;
        }
        atomicAdd(&rank[lane], below);
    }
    __syncthreads();
    if (tid < 64 && mine < N) {
        const uint2 me = all[mine];
        keys[rank[lane]] = me.y;
        perm[rank[lane]] = me.x;
    }
}

// A radix pass: a workgroup takes `per_wg` consecutive keys (a multiple of 256: a quarter to each wave).  counts: [bins][workgroups]
struct Radix { const void *ids; bool wide; int64_t N, V, padding; const uint32_t *keys_in, *perm_in; uint32_t *keys_out, *perm_out, *counts; int shift, bins, wgs, per_wg; };
__device__ __forceinline__ uint32_t radix_key(const Radix &r, int64_t n)
{
    return r.keys_in ? r.keys_in[n] : key_of(r.ids, r.wide, n, r.V, r.padding);
}

__global__ __launch_bounds__(256) void embed_count_kernel(Radix r, Fill f)
{
    if ((int)blockIdx.x >= r.wgs) { fill_zeros(f, (int)blockIdx.x - r.wgs, (int)gridDim.x - r.wgs); return; }
    __shared__ uint32_t count[RADIX_BINS];
    for (int b = threadIdx.x; b < r.bins; b += 256) count[b] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * r.per_wg, to = min(from + r.per_wg, r.N);
    for (int64_t n = from + threadIdx.x; n < to; n += 256) atomicAdd(&count[radix_key(r, n) >> r.shift & (r.bins - 1)], 1u);
    __syncthreads();
    for (int b = threadIdx.x; b < r.bins; b += 256) r.counts[(int64_t)b * r.wgs + blockIdx.x] = count[b];
}

__global__ __launch_bounds__(256) void embed_move_kernel(Radix r)
{
    __shared__ uint32_t at[4][RADIX_BINS];                                   // where a wave's next key of a bin goes
    __shared__ uint32_t wave_sum[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, me = (int)blockIdx.x;
    // keys of smaller bins anywhere, and of a bin in earlier workgroups: two bins to a thread
    uint32_t total[2], before[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int b = 2 * tid + j;
        total[j] = before[j] = 0;
        if (b < r.bins)
            for (int w = 0; w < r.wgs; ++w) {
                const uint32_t c = r.counts[(int64_t)b * r.wgs + w];
                total[j] += c;
                if (w < me) before[j] += c;
            }
    }
    uint32_t sum = total[0] + total[1], scan = sum;
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t v = __shfl_up(scan, d);
        if (lane >= d) scan += v;
    }
    if (lane == 63) wave_sum[wave] = scan;
    for (int b = tid; b < 4 * RADIX_BINS; b += 256) (&at[0][0])[b] = 0;
    __syncthreads();
    uint32_t base = scan - sum;
    for (int w = 0; w < wave; ++w) base += wave_sum[w];
    // keys of a bin in each wave's quarter
    const int64_t per_wave = r.per_wg / 4, from = (int64_t)me * r.per_wg + wave * per_wave, to = min(from + per_wave, r.N);
    for (int64_t n = from + lane; n < to; n += 64) atomicAdd(&at[wave][radix_key(r, n) >> r.shift & (r.bins - 1)], 1u);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int b = 2 * tid + j;
        if (b < r.bins) {
            uint32_t next = base + (j ? total[0] : 0u) + before[j];
            for (int w = 0; w < 4; ++w) { const uint32_t c = at[w][b]; at[w][b] = next; next += c; }
        }
    }
    __syncthreads();
    // 64 keys at a time in their order: a key's place is its bin's next one, behind the lower lanes with the same bin
    for (int64_t first = from; first < to; first += 64) {
        const int64_t n = first + lane;
        const bool there = n < to;
        const uint32_t key = there ? radix_key(r, n) : 0, perm = there ? (r.perm_in ? r.perm_in[n] : (uint32_t)n) : 0;
        const uint32_t bin = key >> r.shift & (r.bins - 1);
        uint64_t same = __ballot(there);
        for (int bit = 0; (1 << bit) < r.bins; ++bit) {
            const bool set = bin >> bit & 1;
            const uint64_t with = __ballot(set);
            same &= set ? with : ~with;
        }
        const int ahead = __popcll(same & ((1ull << lane) - 1));
        // (volatile: lanes of a wave read each other's counters)
        volatile uint32_t *next = &at[wave][bin];
        uint32_t place = 0;
        if (there) place = *next;
        __builtin_amdgcn_wave_barrier();
        if (there && ahead == 0) *next = place + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (there) { r.keys_out[place + ahead] = key; r.perm_out[place + ahead] = perm; }
    }
}

// ---- sums
struct Sums {
    const void *g;
    int64_t ldg, D, ldo;
    int N, chunk, chunks;
    uint32_t V;
    const uint32_t *keys, *perm;
    void *out;
    float *part;                 // [chunks][2][part_ld]: the sums of the row that began before the chunk, and of the one that runs on behind it
    int64_t part_ld;
    float scale;
    int accumulate;
};

template <int OT, bool VEC> __device__ __forceinline__ void write_sum(const Sums &s, uint32_t row, int64_t c, int left, float (&v)[EW])
{
    const int64_t at = (int64_t)row * s.ldo + c;
#pragma unroll
    for (int i = 0; i < EW; ++i) v[i] *= s.scale;
    const bool vec = VEC && left == EW;
    if (s.accumulate) {
        float old[EW];
        if (vec) load_row<OT, EW, true>(s.out, at, left, old); else load_row<OT, EW, false>(s.out, at, left, old);
#pragma unroll
        for (int i = 0; i < EW; ++i) v[i] += old[i];
    }
    if (vec) store_row<OT, EW, true>(s.out, at, left, v); else store_row<OT, EW, false>(s.out, at, left, v);
}

template <int GT, int OT, bool VEC>
__global__ __launch_bounds__(256) void embed_sum_kernel(Sums s)
{
    const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * EW;
    if (c >= s.D) return;
    const int left = (int)min(s.D - c, (int64_t)EW);
    const int from = (int)blockIdx.x * s.chunk, to = min(from + s.chunk, s.N);
    const uint32_t before = from > 0 ? s.keys[from - 1] : 0xffffffffu, behind = to < s.N ? s.keys[to] : 0xffffffffu;
    float acc[EW];
#pragma unroll
    for (int j = 0; j < EW; ++j) acc[j] = 0.f;
    uint32_t row = s.keys[from];
    bool began = row != before;                                              // whether this row's tokens begin in this chunk
    auto leave = [&](bool runs_on) {
        if (row >= s.V) return;                                              // (tokens that count for nothing)
        if (began && !runs_on) write_sum<OT, VEC>(s, row, c, left, acc);
        else {
            float *to_part = s.part + ((int64_t)blockIdx.x * 2 + (began ? 1 : 0)) * s.part_ld + c;
            *(float4 *)to_part = make_float4(acc[0], acc[1], acc[2], acc[3]);
            *(float4 *)(to_part + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
        }
    };
    constexpr int AHEAD = GT == NM_DT_F32 ? 4 : 8;
    for (int i = from; i < to; i += AHEAD) {
        float v[AHEAD][EW];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int k = min(i + j, to - 1);
            const int64_t at = (int64_t)s.perm[k] * s.ldg + c;
            if (VEC && left == EW) load_row<GT, EW, true>(s.g, at, left, v[j]); else load_row<GT, EW, false>(s.g, at, left, v[j]);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (i + j < to) {
                const uint32_t key = s.keys[i + j];
                if (key != row) {
                    leave(false);
                    row = key;
                    began = true;
#pragma unroll
                    for (int e = 0; e < EW; ++e) acc[e] = 0.f;
                }
#pragma unroll
                for (int e = 0; e < EW; ++e) acc[e] += v[j][e];
            }
    }
    leave(row == behind);
}

// a row that runs over several chunks, where it begins: its parts, chunk after chunk
template <int OT, bool VEC>
__global__ __launch_bounds__(256) void embed_join_kernel(Sums s)
{
    const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * EW;
    const int chunk = (int)blockIdx.x, from = chunk * s.chunk, to = from + s.chunk;
    if (to >= s.N) return;                                                   // the last chunk: nothing runs on
    const uint32_t row = s.keys[to];
    if (row >= s.V || s.keys[to - 1] != row || (from > 0 && s.keys[from] == row && s.keys[from - 1] == row)) return;
    if (c >= s.D) return;
    const int left = (int)min(s.D - c, (int64_t)EW);
    // the last chunk that has some of the row
    int lo = chunk + 1, hi = s.chunks - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s.keys[mid * s.chunk] == row) lo = mid; else hi = mid - 1;
    }
    float acc[EW];
    load_row<NM_DT_F32, EW, true>(s.part, ((int64_t)chunk * 2 + 1) * s.part_ld + c, EW, acc);
    for (int k = chunk + 1; k <= lo; ++k) {
        float v[EW];
        load_row<NM_DT_F32, EW, true>(s.part, (int64_t)k * 2 * s.part_ld + c, EW, v);
#pragma unroll
        for (int e = 0; e < EW; ++e) acc[e] += v[e];
    }
    write_sum<OT, VEC>(s, row, c, left, acc);
}

int bits_of(int64_t v) { int b = 0; while (v >> b) ++b; return b; }

struct GradPlan { int64_t keys, perm, counts, part, part_ld, bytes; int chunk, chunks, per_wg, wgs, passes, digit; };
GradPlan plan_grad(int64_t N, int64_t V, int64_t D)
{
    GradPlan p{};
    auto up = [](int64_t b) { return (b + 255) / 256 * 256; };
    p.chunk = 16;
    p.chunks = (int)((N + p.chunk - 1) / p.chunk);
    p.part_ld = (D + EW - 1) / EW * EW;
    const int bits = bits_of(V);                                             // keys are 0 .. V
    p.passes = N <= RANK_MOST ? 0 : (bits + RADIX_BITS - 1) / RADIX_BITS;
    p.digit = p.passes ? (bits + p.passes - 1) / p.passes : 0;
    p.per_wg = (int)((N / 256 + KEYS) / KEYS * KEYS);                        // at most 256 workgroups
    p.wgs = (int)((N + p.per_wg - 1) / p.per_wg);
    p.keys = 0;
    p.perm = p.keys + 2 * up(N * 4);
    p.counts = p.perm + 2 * up(N * 4);
    p.part = p.counts + up((int64_t)RADIX_BINS * p.wgs * 4);
    p.bytes = p.part + up((int64_t)p.chunks * 2 * p.part_ld * 4);
    return p;
}

}  // namespace

hipError_t launch_embed(int table_dt, int out_dt, const void *table, int64_t V, int64_t D, int64_t ldt, const void *ids, bool wide, int64_t N, float scale, void *out,
                        int64_t ldo, hipStream_t st)
{
    if (N == 0 || D == 0) return hipSuccess;
    int shift = 0;
    while (shift < 8 && ((int64_t)EW << shift) < D) ++shift;
    const int64_t te = table_dt == NM_DT_F32 ? 4 : 2, oe = out_dt == NM_DT_F32 ? 4 : 2;
    const bool vec = (uintptr_t)table % 16 == 0 && (uintptr_t)out % 16 == 0 && ldt * te % 16 == 0 && ldo * oe % 16 == 0;
    const int64_t wgs = (N + (256 >> shift) - 1) / (256 >> shift);
    if (wgs > 0x7fffffff) return hipErrorInvalidConfiguration;
#define NM_EMBED(TT, OT)                                                                                                                                   \
    do {                                                                                                                                                   \
        if (vec) hipLaunchKernelGGL((embed_kernel<TT, OT, true>), dim3((unsigned)wgs), dim3(256), 0, st, table, V, D, ldt, ids, wide, N, scale, out, ldo, shift); \
        else hipLaunchKernelGGL((embed_kernel<TT, OT, false>), dim3((unsigned)wgs), dim3(256), 0, st, table, V, D, ldt, ids, wide, N, scale, out, ldo, shift);    \
    } while (0)
    if (table_dt == NM_DT_F32) { if (out_dt == NM_DT_F32) NM_EMBED(NM_DT_F32, NM_DT_F32); else NM_EMBED(NM_DT_F32, NM_DT_BF16); }
    else                       { if (out_dt == NM_DT_F32) NM_EMBED(NM_DT_BF16, NM_DT_F32); else NM_EMBED(NM_DT_BF16, NM_DT_BF16); }
#undef NM_EMBED
    return hipGetLastError();
}

size_t embed_grad_workspace(int64_t N, int64_t V, int64_t D) { return N > 0 ? (size_t)plan_grad(N, V, D).bytes : 0; }

hipError_t launch_embed_grad(int g_dt, int out_dt, const void *g, int64_t ldg, const void *ids, bool wide, int64_t N, int64_t V, int64_t D, float scale,
                             int64_t padding, bool accumulate, void *out, int64_t ldo, void *workspace, hipStream_t st)
{
    const int64_t oe = out_dt == NM_DT_F32 ? 4 : 2, ge = g_dt == NM_DT_F32 ? 4 : 2;
    const Fill fill{(char *)out, accumulate ? 0 : V, D * oe, ldo * oe};
    const int fill_wgs = accumulate ? 0 : (int)std::min<int64_t>((V * D * oe + 16383) / 16384, 2048);
    const GradPlan p = plan_grad(std::max<int64_t>(N, 1), V, D);
    char *w = (char *)workspace;
    uint32_t *keys[2], *perm[2];
    const int64_t half = (N * 4 + 255) / 256 * 256;
    for (int i = 0; i < 2; ++i) { keys[i] = (uint32_t *)(w + p.keys + i * half); perm[i] = (uint32_t *)(w + p.perm + i * half); }
    int now = 0;
    if (p.passes == 0) {
        const int sort_wgs = (int)((N + 63) / 64);
        if (sort_wgs + fill_wgs == 0) return hipSuccess;
        hipLaunchKernelGGL(embed_rank_kernel, dim3((unsigned)(sort_wgs + fill_wgs)), dim3(256), (size_t)(N + 7) / 8 * 64, st, ids, wide, (int)N, V, padding, sort_wgs, keys[0], perm[0], fill);
    } else {
        for (int k = 0; k < p.passes; ++k) {
            const Radix r{ids, wide, N, V, padding, k ? keys[now] : nullptr, k ? perm[now] : nullptr, keys[k ? 1 - now : 0], perm[k ? 1 - now : 0], (uint32_t *)(w + p.counts),
                          k * p.digit, 1 << p.digit, p.wgs, p.per_wg};
            if (k) now = 1 - now;
            hipLaunchKernelGGL(embed_count_kernel, dim3((unsigned)(p.wgs + (k ? 0 : fill_wgs))), dim3(256), 0, st, r, fill);
            hipLaunchKernelGGL(embed_move_kernel, dim3((unsigned)p.wgs), dim3(256), 0, st, r);
        }
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (N == 0) return hipSuccess;
    const Sums s{g, ldg, D, ldo, (int)N, p.chunk, p.chunks, (uint32_t)V, keys[now], perm[now], out, (float *)(w + p.part), p.part_ld, scale, accumulate};
    const bool vec = (uintptr_t)g % 16 == 0 && (uintptr_t)out % 16 == 0 && ldg * ge % 16 == 0 && ldo * oe % 16 == 0;
    const int64_t columns = (D + EW - 1) / EW;
    const int threads = (int)std::min<int64_t>((columns + 63) / 64 * 64, 256);
    const dim3 grid((unsigned)p.chunks, (unsigned)((columns + threads - 1) / threads));
#define NM_SUM(GT, OT, VEC)                                                                                  \
    do {                                                                                                     \
        hipLaunchKernelGGL((embed_sum_kernel<GT, OT, VEC>), grid, dim3(threads), 0, st, s);                   \
        hipLaunchKernelGGL((embed_join_kernel<OT, VEC>), grid, dim3(threads), 0, st, s);                      \
    } while (0)
#define NM_SUM_V(GT, OT) do { if (vec) NM_SUM(GT, OT, true); else NM_SUM(GT, OT, false); } while (0)
    if (g_dt == NM_DT_F32) { if (out_dt == NM_DT_F32) NM_SUM_V(NM_DT_F32, NM_DT_F32); else NM_SUM_V(NM_DT_F32, NM_DT_BF16); }
    else                   { if (out_dt == NM_DT_F32) NM_SUM_V(NM_DT_BF16, NM_DT_F32); else NM_SUM_V(NM_DT_BF16, NM_DT_BF16); }
#undef NM_SUM_V
#undef NM_SUM
    return hipGetLastError();
}

}  // namespace nm
