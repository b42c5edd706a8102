// Embedding: rows of a table by token, scaled, and the table's gradient.
//     out[n] = scale E[id_n]                     dE[v] = scale * sum over the tokens n with id_n = v of g[n]
// The gradient's tokens are sorted by id, stably.  A row's sum is binary32, in an order that follows from the arguments alone, so that the same call gives the same bits: up to
// LIGHT tokens in their order, more of them in parts by place in the sorted list, each in order, and the parts in 16 groups, each in order (the one-launch form: quarters of
// the row's tokens, each in order).
// Up to FEW_MOST tokens take one launch (embed_few_kernel), more of them:
//   sort    up to RANK_MOST tokens, one launch: the rank of a token is the number of tokens whose (id, position) is smaller, which 16 waves count
//           for 64 tokens from LDS.  Up to MERGE_MOST, two: chunks of 256 tokens sorted that way, and merged.  Beyond, radix passes of at most 9 bits, a counting
//           launch and a moving one each.  Workgroups behind those of the first launch fill the gradient with zeros meanwhile.
//   sum     a workgroup takes CHUNK consecutive tokens of the sorted list and a slab of columns.  A row with at most LIGHT tokens is summed, and written, where
//           it begins; of a longer one each chunk leaves its part in the workspace.
//   join    those rows: a workgroup for 512 columns of a row adds up its parts in 16 groups.  Tokens that count for nothing stand last and are no row.
// Bound: HBM.  32768 tokens of 120001 x 4096 in bf16: lookup 69 us (441 MB moved, 6.4 TB/s), sort and zeros 145 + 13 (983 MB, 6.8 TB/s), sums 112 (359 MB; the
// zeros that still wait to be written back are in their way: 69 with zeros that bypass the caches, which take 224 instead of 145), join 14.  16384 tokens of 50001 x
// 1024 with a binary32 gradient: 14.3, 26 + 5, 18, 5.2: half of that is launches and latency.  Sorts in us: rank 256 / 1024 / 4096 tokens 2.6 / 5.1 / 9.5; chunks and
// merge 4097 / 16384 / 32768 6.3 + 4 / 6.4 + 5 / 6.4 + 12.8 (4096 by rank and two launches saved beats it); radix 32769 / 65536 2 x 19 / 2 x 23.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "nm_internal.h"
#include "grid_row.h"
#include "gemm_plan.h"           // NM_CUS
#include "prune_common.h"        // Row
#include "row_vec.h"

namespace nm {

namespace {

// Tokens: 32 or 64 bits wide, read as words of 32 without a branch (a branch for each load would have it waited for before the next one is sent)
struct Ids { const uint32_t *at; int words; };
// the token at n where it lies in 0 .. V - 1, otherwise V (below 2^32)
__device__ __forceinline__ uint32_t token_at(const Ids &ids, int64_t n, int64_t V)
{
    const uint32_t lo = ids.at[n * ids.words], hi = ids.at[n * ids.words + ids.words - 1];
    return (ids.words == 2 ? hi == 0 : (int32_t)lo >= 0) && lo < (uint64_t)V ? lo : (uint32_t)V;
}

// ---- lookup: 2^shift threads to a row
template <int TT, int OT, bool NARROW>
__global__ __launch_bounds__(256) void embed_kernel(const void *table, int64_t V, int64_t D, int64_t ldt, Ids ids, int64_t N, float scale, void *out, int64_t ldo, int shift)
{
    const int64_t n = (int64_t)grid_place(blockIdx.x, blockIdx.y) * (256 >> shift) + (threadIdx.x >> shift);
    if (n >= N) return;
    const uint32_t lo = ids.at[n * ids.words], hi = ids.at[n * ids.words + ids.words - 1];
    const int64_t id = ids.words == 2 ? (int64_t)((uint64_t)hi << 32 | lo) : (int32_t)lo;
    const bool there = id >= 0 && id < V;                            // (a token outside the table: a row of NaN, nothing is read)
    const int64_t step = (int64_t)EW << shift;
    for (int64_t c0 = (int64_t)(threadIdx.x & ((1 << shift) - 1)) * EW; c0 < D; c0 += step) {
        const int64_t c = NARROW ? c0 : min(c0, D - EW);             // (the row's last elements are written twice, with the same values)
        const int left = NARROW ? (int)D : EW;
        float v[EW];
        if (there) {
            const Raw<TT> r = load_raw<TT, NARROW>(table, id * ldt + c, left);
#pragma unroll
            for (int i = 0; i < EW; ++i) v[i] = element(r, i) * scale;
        } else
#pragma unroll
            for (int i = 0; i < EW; ++i) v[i] = __uint_as_float(0x7fc00000u);
        store_row<OT>(out, n * ldo + c, 0, left, v);
    }
}

// ---- the gradient's sort
constexpr int FEW_MOST = 512, RANK_MOST = 4096, MERGE_MOST = 32768;
constexpr int RADIX_BITS = 9, RADIX_BINS = 1 << RADIX_BITS, KEYS = 2048;     // keys of a workgroup in a radix pass: KEYS or a multiple

struct Fill { char *at; int64_t rows, row_bytes, stride_bytes; };            // rows that become zeros; rows == 0: none
// Rows are taken as one run of bytes where they are contiguous, FILL of them to a workgroup: 983 MB take 144 us (6.8 TB/s) in workgroups of their own, 190 us dealt in
// turn to the threads of 2048.
constexpr int FILL = 16384;
template <int THREADS> __device__ __forceinline__ void fill_zeros(const Fill &f, int64_t wg, int64_t wgs)
{
    if (f.row_bytes == f.stride_bytes && ((uintptr_t)f.at & 15) == 0) {
        const int64_t bytes = f.rows * f.row_bytes, n = bytes / 16;
        const uint4 z = make_uint4(0, 0, 0, 0);
        for (int64_t i = wg * (FILL / 16) + threadIdx.x; i < n; i += wgs * (FILL / 16))
#pragma unroll
            for (int j = 0; j < FILL / 16; j += THREADS)
                if (i + j < n) ((uint4 *)f.at)[i + j] = z;
        if (wg == 0)
            for (int64_t i = n * 16 + 2 * threadIdx.x; i < bytes; i += 2 * THREADS) *(uint16_t *)(f.at + i) = 0;
    } else {
        for (int64_t r = wg; r < f.rows; r += wgs)
            for (int64_t i = 2 * threadIdx.x; i < f.row_bytes; i += 2 * THREADS) *(uint16_t *)(f.at + r * f.stride_bytes + i) = 0;
    }
}

// the key of a token: its id, or V where it counts for nothing
__device__ __forceinline__ uint32_t key_of(const Ids &ids, int64_t n, int64_t V, int64_t padding)
{
    const uint32_t id = token_at(ids, n, V);
    return (int64_t)id == padding ? (uint32_t)V : id;
}

// Rank by counting: a wave counts for 64 tokens through a sixteenth of the list.  Keys in order of their tokens compare by key alone: of the tokens before a token those
// with its key count too.
__global__ __launch_bounds__(1024) void embed_rank_kernel(Ids ids, int N, int64_t V, int64_t padding, int sort_wgs, uint32_t *keys, uint32_t *perm, uint32_t *heavy, Fill f)
{
    if (heavy && blockIdx.x == 0 && threadIdx.x == 0) *heavy = 0;
    if ((int)blockIdx.x >= sort_wgs) { fill_zeros<1024>(f, (int)blockIdx.x - sort_wgs, (int)gridDim.x - sort_wgs); return; }
    __shared__ __attribute__((aligned(16))) uint32_t all[RANK_MOST];
    __shared__ int rank[64];
    const int tid = threadIdx.x, lane = tid & 63, part = __builtin_amdgcn_readfirstlane(tid >> 6), first = (int)blockIdx.x * 64, mine = first + lane;
    const int each = ((N + 15) / 16 + 15) & ~15, from = part * each, to = min(from + each, (N + 15) & ~15);
    for (int n = tid; n < RANK_MOST && n < N + 16; n += 1024) all[n] = n < N ? key_of(ids, n, V, padding) : 0xffffffffu;
    if (tid < 64) rank[tid] = 0;
    __syncthreads();
    const uint32_t me = all[min(mine, N - 1)];
    int below = 0;
    auto count = [&](int lo, int hi, uint32_t limit) {                       // keys below `limit` at places lo .. hi - 1, multiples of 16
#pragma unroll 2
        for (int i = lo; i < hi; i += 16)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const uint4 v = *(const uint4 *)&all[i + j];
                below += (v.x < limit) + (v.y < limit) + (v.z < limit) + (v.w < limit);
            }
    };
    // (first is a multiple of 64, and each part of 16: a part lies before the 64 tokens, behind them, or among them in groups of 16)
    const int a = min(max(first, from), to), b = min(max(first + 64, from), to);
    count(from, a, me + 1);
    for (int i = a; i < b; ++i) below += all[i] < me || (all[i] == me && i < mine);
    count(b, to, me);
    atomicAdd(&rank[lane], below);
    __syncthreads();
    if (tid < 64 && mine < N) { keys[rank[lane]] = me; perm[rank[lane]] = (uint32_t)mine; }
}

// A radix pass: a workgroup takes `per_wg` consecutive keys (a multiple of 256: a quarter to each wave).  counts: [bins][workgroups]
struct Radix { Ids ids; int64_t N, V, padding; const uint32_t *keys_in, *perm_in; uint32_t *keys_out, *perm_out, *counts; int shift, bins, wgs, per_wg; };
__device__ __forceinline__ uint32_t radix_key(const Radix &r, int64_t n)
{
    return r.keys_in ? r.keys_in[n] : key_of(r.ids, n, r.V, r.padding);
}

__global__ __launch_bounds__(256) void embed_count_kernel(Radix r, uint32_t *heavy, Fill f)
{
    if (heavy && blockIdx.x == 0 && threadIdx.x == 0) *heavy = 0;
    if ((int)blockIdx.x >= r.wgs) { fill_zeros<256>(f, (int)blockIdx.x - r.wgs, (int)gridDim.x - r.wgs); return; }
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

// Chunks of 256 tokens sorted each by a workgroup, a token's rank in its chunk by counting; then a token's place is its rank plus, from each other chunk, the
// number of keys below its own, which a search in eight steps finds (of earlier chunks the equal ones count too).  The search runs in LDS, which holds all
// keys: 64 tokens to a workgroup, each of its 16 waves searches every sixteenth chunk.
constexpr int SORTED = 256;
__global__ __launch_bounds__(SORTED) void embed_chunk_kernel(Ids ids, int N, int64_t V, int64_t padding, int sort_wgs, uint32_t *keys, uint32_t *perm, uint32_t *heavy, Fill f)
{
    if (heavy && blockIdx.x == 0 && threadIdx.x == 0) *heavy = 0;
    if ((int)blockIdx.x >= sort_wgs) { fill_zeros<256>(f, (int)blockIdx.x - sort_wgs, (int)gridDim.x - sort_wgs); return; }
    __shared__ __attribute__((aligned(16))) uint32_t all[SORTED];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = (int)blockIdx.x * SORTED + tid;
    const uint32_t me = n < N ? key_of(ids, n, V, padding) : 0xffffffffu;
    all[tid] = me;
    __syncthreads();
    int rank = 0;
    auto count = [&](int lo, int hi, uint32_t limit) {
#pragma unroll 4
        for (int i = lo; i < hi; i += 4) {
            const uint4 v = *(const uint4 *)&all[i];
            rank += (v.x < limit) + (v.y < limit) + (v.z < limit) + (v.w < limit);
        }
    };
    count(0, wave * 64, me + 1);                                             // (of what lies behind the list's end none is asked: 0xffffffff + 1 is 0)
#pragma unroll 4
    for (int i = 0; i < 64; ++i) {
        const uint32_t other = all[wave * 64 + i];
        rank += other < me || (other == me && wave * 64 + i < tid);
    }
    count(wave * 64 + 64, SORTED, me);
    if (n < N) {
        const int at = (int)blockIdx.x * SORTED + rank;
        keys[at] = me;
        perm[at] = (uint32_t)n;
    }
}
__global__ __launch_bounds__(1024) void embed_merge_kernel(const uint32_t *keys_in, const uint32_t *perm_in, int N, int chunks, int rounds, uint32_t *keys, uint32_t *perm)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t sorted[];       // [chunk][SORTED]
    __shared__ int place[64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int i = 4 * tid; i < chunks * SORTED; i += 4096) {
        uint4 v = make_uint4(0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu);
        if (i + 4 <= N) v = *(const uint4 *)(keys_in + i);
        else {
            if (i < N) v.x = keys_in[i];
            if (i + 1 < N) v.y = keys_in[i + 1];
            if (i + 2 < N) v.z = keys_in[i + 2];
        }
        *(uint4 *)&sorted[i] = v;
    }
    for (int first = (int)blockIdx.x * 64 * rounds, end = min(first + 64 * rounds, N); first < end; first += 64) {
        const int mine = min(first + lane, N - 1), own = first / SORTED;
        __syncthreads();                                                     // (the round before is done with place)
        if (tid < 64) place[tid] = first + tid - own * SORTED;
        __syncthreads();
        const uint32_t me = sorted[mine];
        int below = 0;
#pragma unroll 4
        for (int c = wave; c < chunks; c += 16) {
            const uint32_t *list = sorted + c * SORTED, limit = me + (c < own ? 1 : 0);
            int at = 0;
#pragma unroll
            for (int step = SORTED / 2; step; step >>= 1) at += list[at + step - 1] < limit ? step : 0;
            at += list[at] < limit;                                          // (at is SORTED - 1 at most)
            below += c == own ? 0 : at;
        }
        atomicAdd(&place[lane], below);
        __syncthreads();
        if (tid < 64 && first + tid < N) { keys[place[tid]] = me; perm[place[tid]] = perm_in[mine]; }
    }
}

// ---- sums
constexpr int CHUNK = 16;        // tokens of a workgroup
constexpr int LIGHT = 48;        // tokens of a row that one workgroup sums, wherever they lie: it sees 64 places from its chunk on
struct Sums {
    const void *g;
    int64_t ldg, D, ldo;
    int N, chunks;
    uint32_t V;
    const uint32_t *keys, *perm;
    void *out;
    float *part;                 // [chunks][2][part_ld]: the sums of the row that began before the chunk, and of the one that runs on behind it
    int64_t part_ld;
    uint32_t *heavy;             // how many rows have more than LIGHT tokens, and the chunks where they begin
    float scale;
    int accumulate;
    int later;                   // the columns behind those of another launch, which has counted the long rows
};

template <int OT, bool NARROW> __device__ __forceinline__ void write_sum(const Sums &s, uint32_t row, int64_t c, int skip, float (&v)[EW])
{
    const int64_t at = (int64_t)row * s.ldo + c;
    const int left = NARROW ? (int)s.D : EW;
#pragma unroll
    for (int i = 0; i < EW; ++i) v[i] *= s.scale;
    if (s.accumulate) {
        const Raw<OT> old = load_raw<OT, NARROW>(s.out, at, left);
#pragma unroll
        for (int i = 0; i < EW; ++i) v[i] += element(old, i);
    }
    store_row<OT>(s.out, at, skip, left, v);
}

// What a chunk has to do, from the 64 keys before it (lane i: place from - 64 + i) and the 64 from its first on.  A row with at most LIGHT tokens belongs to the
// chunk where it begins; a longer one leaves the sum of its tokens in each chunk in the workspace.
struct Share {
    int begin, end;              // places to sum, from the chunk's first on
    bool head, tail;             // the first of their rows began earlier, the last one runs on behind the chunk: both longer than LIGHT
};
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int k) { return (uint32_t)__builtin_amdgcn_readlane((int)v, k); }
__device__ __forceinline__ Share share_of(uint32_t before, uint32_t here, int n, uint32_t V)
{
    Share s{0, n, false, false};
    const uint32_t first = lane_of(here, 0);
    const uint64_t differ = ~__ballot(here == first), differ_before = ~__ballot(before == first);
    const int after = differ ? __builtin_ctzll(differ) : 64, earlier = differ_before ? __builtin_clzll(differ_before) : 64;
    if (earlier > 0) {
        if (earlier + after <= LIGHT) s.begin = min(after, n);
        else s.head = true;
    }
    const uint32_t last = lane_of(here, n - 1);
    if (last >= V) return s;                                                 // (tokens that count for nothing are no row: none to join, nothing behind the chunk to sum)
    const uint64_t runs = __ballot(here == last) >> (n - 1);                 // from the chunk's last place on
    const int behind = (~runs ? __builtin_ctzll(~runs) : 64) - 1;            // places of the last row behind the chunk
    if (n == CHUNK && behind > 0 && !(last == first && after > n - 1 && earlier > 0)) {      // (a row that began earlier is not this chunk's)
        const uint64_t back = ~(__ballot(here == last) << (63 - (n - 1)));   // from the chunk's last place backwards
        const int begun = n - min(n, back ? __builtin_clzll(back) : 64);     // where the last row begins
        const int length = n - begun + behind;
        if (length <= LIGHT) s.end = n + behind;
        else s.tail = true;
    }
    return s;
}

template <int GT, int OT, bool NARROW>
__global__ __launch_bounds__(256) void embed_sum_kernel(Sums s)
{
    const int64_t c0 = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * EW, c = NARROW ? c0 : min(c0, s.D - EW);
    const int skip = (int)(c0 - c);
    const uint32_t chunk = grid_place(blockIdx.x, blockIdx.z);
    if (chunk >= (uint32_t)s.chunks) return;
    const int from = (int)chunk * CHUNK, n = min(CHUNK, s.N - from), lane = threadIdx.x & 63;
    uint32_t before = 0xffffffffu, here = 0xfffffffeu, place = 0;
    if (from - 64 + lane >= 0) before = s.keys[from - 64 + lane];
    if (from + lane < s.N) { here = s.keys[from + lane]; place = s.perm[from + lane]; }
    if (lane_of(here, 0) >= s.V) return;                                     // (tokens that count for nothing, the last of the list)
    const Share share = share_of(before, here, n, s.V);
    if (share.tail && !s.later && blockIdx.y == 0 && threadIdx.x == 0) s.heavy[1 + atomicAdd(s.heavy, 1u)] = chunk;       // (in any order: each row is joined by itself)
    if (c0 >= s.D || share.begin >= share.end) return;
    float acc[EW];
#pragma unroll
    for (int e = 0; e < EW; ++e) acc[e] = 0.f;
    uint32_t row = lane_of(here, share.begin);
    bool head = share.head;
    auto leave = [&](bool tail) {
        if (row < s.V) {
            if (!head && !tail) write_sum<OT, NARROW>(s, row, c, skip, acc);
            else {
                float *to_part = s.part + ((int64_t)chunk * 2 + (head ? 0 : 1)) * s.part_ld + c0;
                *(float4 *)to_part = make_float4(acc[0], acc[1], acc[2], acc[3]);
                *(float4 *)(to_part + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
            }
        }
        head = false;
#pragma unroll
        for (int e = 0; e < EW; ++e) acc[e] = 0.f;
    };
    constexpr int AHEAD = GT == NM_DT_F32 ? 4 : 8;                           // rows on their way
    for (int k = share.begin; k < share.end; k += AHEAD) {
        Raw<GT> v[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)                                      // (past the end the last token's again)
            v[j] = load_raw<GT, NARROW>(s.g, (int64_t)lane_of(place, min(k + j, share.end - 1)) * s.ldg + c, NARROW ? (int)s.D : EW);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (k + j < share.end) {
                const uint32_t key = lane_of(here, k + j);
                if (key != row) { leave(false); row = key; }
#pragma unroll
                for (int e = 0; e < EW; ++e) acc[e] += element(v[j], e);
            }
    }
    leave(share.tail);
}

// The rows with more than LIGHT tokens: their parts in 16 groups, each chunk after chunk, and the groups in order
constexpr int GROUPS = 16;
constexpr int64_t SLAB = 65535ll * 64 * EW;  // columns of a launch: a workgroup of the join takes 64 EW of them
template <int OT, bool NARROW>
__global__ __launch_bounds__(64 * GROUPS) void embed_join_kernel(Sums s)
{
    __shared__ float sums[GROUPS - 1][EW][64];
    const int lane = threadIdx.x & 63, group = threadIdx.x >> 6, count = (int)s.heavy[0];
    const int64_t c0 = ((int64_t)blockIdx.y * 64 + lane) * EW, c = NARROW ? c0 : min(c0, s.D - EW);
    const bool there = c0 < s.D;
    for (int k = (int)blockIdx.x; k < count; k += (int)gridDim.x) {
        const int chunk = (int)s.heavy[1 + k];
        const uint32_t row = s.keys[(chunk + 1) * CHUNK];
        // the last chunk that has some of the row, by 64 probes at a time
        int lo = chunk + 1, hi = s.chunks - 1;
        while (lo < hi) {
            const int step = (hi - lo + 63) / 64;
            const uint64_t others = ~__ballot(s.keys[min(lo + step * (lane + 1), hi) * CHUNK] == row);
            const int same = others ? __builtin_ctzll(others) : 64;
            const int to = min(lo + step * same, hi);
            hi = same < 64 ? min(lo + step * (same + 1), hi) - 1 : hi;
            lo = to;
            if (same == 64) break;
            hi = max(hi, lo);
        }
        const int parts = lo - chunk + 1, each = (parts + GROUPS - 1) / GROUPS, first = min(group * each, parts), last = min(first + each, parts);
        float acc[EW];
#pragma unroll
        for (int e = 0; e < EW; ++e) acc[e] = 0.f;
        if (there)
            for (int i = first; i < last; i += 4) {
                Raw<NM_DT_F32> v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int p = min(i + j, last - 1);                      // part 0: what the row has in the chunk where it begins
                    v[j] = load_raw<NM_DT_F32>(s.part, ((int64_t)(chunk + p) * 2 + (p == 0 ? 1 : 0)) * s.part_ld + c0);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (i + j < last)
#pragma unroll
                        for (int e = 0; e < EW; ++e) acc[e] += element(v[j], e);
            }
        if (group > 0)
#pragma unroll
            for (int e = 0; e < EW; ++e) sums[group - 1][e][lane] = acc[e];
        __syncthreads();
        if (group == 0 && there) {
#pragma unroll
            for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
                for (int e = 0; e < EW; ++e) acc[e] += sums[g][e][lane];
            write_sum<OT, NARROW>(s, row, c, (int)(c0 - c), acc);
        }
        __syncthreads();
    }
}

// ---- up to FEW_MOST tokens: one launch, without a sorted list.  A workgroup to a token reads all ids; the first token with an id sums the rows of all that have it.  The
// workgroups behind them fill with zeros the rows that no token has: each marks which of its rows those are.
// (us, this way / sorted, rank, sum and join kernels: 14 tokens of 3070 x 97 9.3 / 15.3, 199 of 11855 x 135 9.1 / 14.7, 21 of 50605 x 789, 80 MB of gradient, 14.3 / 21.6, 200 of
// 120001 x 4096 165 / 168; 256 tokens that share one row of 4096 12.5 / 14.5 in bf16, 17.5 / 14.5 in binary32.)
constexpr int FEW_WG = 256;
constexpr int FEW_WGS = 2048;    // all at once on the chip: with more than 256 tokens the way to take while its workgroups are no more than these (300 of 5000 x 512
                                 // 8.3 / 12.9 us; 450 of 56382 x 2161, 17000 workgroups that read all ids each, 172 / 40)
// PER: ids that a thread looks at, next to each other
template <int GT, int OT, int PER>
__global__ __launch_bounds__(FEW_WG) void embed_few_kernel(Ids ids, int64_t V, int64_t padding, Sums s, int rows_per_wg, int shift)
{
    constexpr int WAVES = FEW_WG / 64;
    __shared__ uint32_t list[FEW_WG * PER], taken[FILL / (2 * EW)];
    __shared__ int counts[WAVES];
    __shared__ uint32_t wanted;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = (int)blockIdx.x;
    uint32_t key[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int at = tid * PER + j;
        key[j] = key_of(ids, min(at, s.N - 1), V, padding);
        if (at >= s.N) key[j] = (uint32_t)V;
    }
    if (n >= s.N) {
        if (blockIdx.y) return;
        const int64_t r0 = (int64_t)(n - s.N) * rows_per_wg;
        const int rows = (int)min(V - r0, (int64_t)rows_per_wg);
        for (int r = tid; r < rows; r += FEW_WG) taken[r] = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if ((int64_t)key[j] >= r0 && (int64_t)key[j] < r0 + rows) taken[(int64_t)key[j] - r0] = 1;
        __syncthreads();
        const float zeros[EW] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int r = tid >> shift; r < rows; r += FEW_WG >> shift)
            if (!taken[r])
                for (int64_t c = (int64_t)(tid & ((1 << shift) - 1)) * EW; c < s.D; c += (int64_t)EW << shift) store_row<OT>(s.out, (r0 + r) * s.ldo + min(c, s.D - EW), 0, EW, zeros);
        return;
    }
    if (n / PER == tid)
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (n % PER == j) wanted = key[j];
    __syncthreads();
    const uint32_t row = wanted;
    uint64_t in_wave[PER];
    int mine = 0, before = 0;
    bool earlier = false;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const bool same = key[j] == row;
        in_wave[j] = __ballot(same);
        mine += __popcll(in_wave[j]);
        before += __popcll(in_wave[j] & ((1ull << lane) - 1));
        earlier |= same && tid * PER + j < n;
    }
    if (lane == 0) counts[wave] = mine;
    if (__syncthreads_or(earlier) || row == (uint32_t)V) return;                 // (an earlier token's, or nobody's)
    int total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { before += w < wave ? counts[w] : 0; total += counts[w]; }
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (key[j] == row) list[before++] = (uint32_t)(tid * PER + j);
    __syncthreads();
    // a wave takes 512 columns; of more than AHEAD rows a quarter, and the quarters are added in their order
    constexpr int AHEAD = GT == NM_DT_F32 ? 8 : 16;                          // rows on their way
    const int64_t c0 = ((int64_t)blockIdx.y * 64 + lane) * EW, c = min(c0, s.D - EW);
    const int each = total > AHEAD ? (total + WAVES - 1) / WAVES : total, from = min(wave * each, total), to = min(from + each, total);
    float acc[EW] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int k = from; k < to; k += AHEAD) {
        Raw<GT> v[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (k + j < to) v[j] = load_raw<GT>(s.g, (int64_t)list[k + j] * s.ldg + c);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (k + j < to)
#pragma unroll
                for (int e = 0; e < EW; ++e) acc[e] += element(v[j], e);
    }
    if (total > AHEAD) {
        __shared__ float parts[WAVES - 1][EW][64];
        if (wave > 0)
#pragma unroll
            for (int e = 0; e < EW; ++e) parts[wave - 1][e][lane] = acc[e];
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES - 1; ++w)
#pragma unroll
            for (int e = 0; e < EW; ++e) acc[e] += parts[w][e][lane];
    }
    if (wave == 0 && c0 < s.D) write_sum<OT, false>(s, row, c, (int)(c0 - c), acc);
}

int bits_of(int64_t v) { int b = 0; while (v >> b) ++b; return b; }

struct GradPlan { int64_t keys, perm, counts, heavy, part, part_ld, bytes; int chunks, per_wg, wgs, passes, digit; };
GradPlan plan_grad(int64_t N, int64_t V, int64_t D)
{
    GradPlan p{};
    auto up = [](int64_t b) { return (b + 255) / 256 * 256; };
    p.chunks = (int)((N + CHUNK - 1) / CHUNK);
    p.part_ld = (D + EW - 1) / EW * EW;
    const int bits = bits_of(V);                                             // keys are 0 .. V
    p.passes = N <= RANK_MOST ? 0 : (bits + RADIX_BITS - 1) / RADIX_BITS;
    p.digit = p.passes ? (bits + p.passes - 1) / p.passes : 0;
    p.per_wg = (int)((N / 256 + KEYS) / KEYS * KEYS);                        // at most 256 workgroups
    p.wgs = (int)((N + p.per_wg - 1) / p.per_wg);
    p.keys = 0;
    p.perm = p.keys + 2 * up(N * 4);
    p.counts = p.perm + 2 * up(N * 4);
    p.heavy = p.counts + up((int64_t)RADIX_BINS * p.wgs * 4);
    p.part = p.heavy + up((N / LIGHT + 2) * 4);
    p.bytes = p.part + up((int64_t)p.chunks * 2 * p.part_ld * 4);
    return p;
}

}  // namespace

hipError_t launch_embed(int table_dt, int out_dt, const void *table, int64_t V, int64_t D, int64_t ldt, const void *ids, bool wide, int64_t N, float scale, void *out,
                        int64_t ldo, hipStream_t st)
{
    if (N == 0 || D == 0) return hipSuccess;
    const Ids tokens{(const uint32_t *)ids, wide ? 2 : 1};
    int shift = 0;
    while (shift < 8 && ((int64_t)EW << shift) < D) ++shift;
    const int64_t wgs = (N + (256 >> shift) - 1) / (256 >> shift);
    if (wgs > 0x7fffffff) return hipErrorInvalidConfiguration;
#define NM_EMBED(TT, OT)                                                                                                                                          \
    do {                                                                                                                                                          \
        if (D < EW) hipLaunchKernelGGL((embed_kernel<TT, OT, true>), dim3(grid_row(wgs), grid_rows(wgs)), dim3(256), 0, st, table, V, D, ldt, tokens, N, scale, out, ldo, shift);  \
        else hipLaunchKernelGGL((embed_kernel<TT, OT, false>), dim3(grid_row(wgs), grid_rows(wgs)), dim3(256), 0, st, table, V, D, ldt, tokens, N, scale, out, ldo, shift);        \
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
    const int64_t oe = out_dt == NM_DT_F32 ? 4 : 2;
    const Fill fill{(char *)out, accumulate ? 0 : V, D * oe, ldo * oe};
    const int fill_wgs = accumulate ? 0 : (int)std::min<int64_t>((V * D * oe + FILL - 1) / FILL, 1 << GRID_ROW_BITS);
    const GradPlan p = plan_grad(std::max<int64_t>(N, 1), V, D);
    const Ids tokens{(const uint32_t *)ids, wide ? 2 : 1};
    char *w = (char *)workspace;
    uint32_t *keys[2], *perm[2];
    const int64_t half = (N * 4 + 255) / 256 * 256;
    for (int i = 0; i < 2; ++i) { keys[i] = (uint32_t *)(w + p.keys + i * half); perm[i] = (uint32_t *)(w + p.perm + i * half); }
    uint32_t *heavy = N ? (uint32_t *)(w + p.heavy) : nullptr;               // (without tokens there is no workspace)
    if (N > 0 && N <= FEW_MOST && D >= EW && D <= 65535 * 64) {
        const int rows = (int)std::max<int64_t>(FILL / (D * oe), 1);
        int shift = 0;
        while (shift < 8 && ((int64_t)EW << shift) < D) ++shift;
        const int64_t wgs = N + (accumulate ? 0 : (V + rows - 1) / rows);
        const Sums s{g, ldg, D, ldo, (int)N, 0, (uint32_t)V, nullptr, nullptr, out, nullptr, 0, nullptr, scale, accumulate, 0};
#define NM_FEW_P(GT, OT, PER) hipLaunchKernelGGL((embed_few_kernel<GT, OT, PER>), dim3((unsigned)wgs, (unsigned)((D + 64 * EW - 1) / (64 * EW))), dim3(FEW_WG), 0, st, tokens, V, padding, s, rows, shift)
#define NM_FEW(GT, OT) do { if (N <= FEW_WG) NM_FEW_P(GT, OT, 1); else NM_FEW_P(GT, OT, 2); } while (0)
        if (N <= FEW_WG ? wgs * FEW_WG < (int64_t)1 << 32 : wgs + N * ((D - 1) / (64 * EW)) <= FEW_WGS) {
            if (g_dt == NM_DT_F32) { if (out_dt == NM_DT_F32) NM_FEW(NM_DT_F32, NM_DT_F32); else NM_FEW(NM_DT_F32, NM_DT_BF16); }
            else                   { if (out_dt == NM_DT_F32) NM_FEW(NM_DT_BF16, NM_DT_F32); else NM_FEW(NM_DT_BF16, NM_DT_BF16); }
            return hipGetLastError();
        }
#undef NM_FEW_P
#undef NM_FEW
    }
    int now = 0;
    if (p.passes == 0) {
        const int sort_wgs = (int)((N + 63) / 64);
        if (sort_wgs + fill_wgs == 0) return hipSuccess;
        hipLaunchKernelGGL(embed_rank_kernel, dim3((unsigned)(sort_wgs + fill_wgs)), dim3(1024), 0, st, tokens, (int)N, V, padding, sort_wgs, keys[0], perm[0], heavy, fill);
    } else if (N <= MERGE_MOST) {
        const int chunks = (int)((N + SORTED - 1) / SORTED);
        now = 1;
        hipLaunchKernelGGL(embed_chunk_kernel, dim3((unsigned)(chunks + fill_wgs)), dim3(SORTED), 0, st, tokens, (int)N, V, padding, chunks, keys[0], perm[0], heavy, fill);
        const int groups = (int)((N + 63) / 64), rounds = (groups + NM_CUS - 1) / NM_CUS;       // (a CU holds one workgroup's keys)
        hipLaunchKernelGGL(embed_merge_kernel, dim3((unsigned)((groups + rounds - 1) / rounds)), dim3(1024), (size_t)chunks * SORTED * 4, st, keys[0], perm[0], (int)N, chunks, rounds, keys[1],
                           perm[1]);
    } else {
        for (int k = 0; k < p.passes; ++k) {
            const Radix r{tokens, N, V, padding, k ? keys[now] : nullptr, k ? perm[now] : nullptr, keys[k ? 1 - now : 0], perm[k ? 1 - now : 0], (uint32_t *)(w + p.counts),
                          k * p.digit, 1 << p.digit, p.wgs, p.per_wg};
            if (k) now = 1 - now;
            hipLaunchKernelGGL(embed_count_kernel, dim3((unsigned)(p.wgs + (k ? 0 : fill_wgs))), dim3(256), 0, st, r, heavy, fill);
            hipLaunchKernelGGL(embed_move_kernel, dim3((unsigned)p.wgs), dim3(256), 0, st, r);
        }
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (N == 0) return hipSuccess;
#define NM_SUM_N(GT, OT, NARROW)                                                                 \
    do {                                                                                         \
        hipLaunchKernelGGL((embed_sum_kernel<GT, OT, NARROW>), grid, dim3(threads), 0, st, s);   \
        hipLaunchKernelGGL((embed_join_kernel<OT, NARROW>), join, dim3(64 * GROUPS), 0, st, s);  \
    } while (0)
#define NM_SUM(GT, OT) do { if (width < EW) NM_SUM_N(GT, OT, true); else NM_SUM_N(GT, OT, false); } while (0)
    // (a dimension of a grid but the first has at most 65535 workgroups: wider rows in slabs)
    const int64_t ge = g_dt == NM_DT_F32 ? 4 : 2;
    for (int64_t from = 0; from < D; from += SLAB) {
        const int64_t width = std::min(D - from, SLAB), columns = (width + EW - 1) / EW;
        const Sums s{(const char *)g + from * ge, ldg, width, ldo, (int)N, p.chunks, (uint32_t)V, keys[now], perm[now], (char *)out + from * oe, (float *)(w + p.part) + from, p.part_ld, heavy,
                     scale, accumulate, from > 0};
        const int threads = (int)std::min<int64_t>((columns + 63) / 64 * 64, 256);
        const dim3 grid(grid_row(p.chunks), (unsigned)((columns + threads - 1) / threads), grid_rows(p.chunks)), join((unsigned)std::min<int64_t>(N / LIGHT + 1, 64), (unsigned)((columns + 63) / 64));
        if (g_dt == NM_DT_F32) { if (out_dt == NM_DT_F32) NM_SUM(NM_DT_F32, NM_DT_F32); else NM_SUM(NM_DT_F32, NM_DT_BF16); }
        else                   { if (out_dt == NM_DT_F32) NM_SUM(NM_DT_BF16, NM_DT_F32); else NM_SUM(NM_DT_BF16, NM_DT_BF16); }
    }
#undef NM_SUM
#undef NM_SUM_N
    return hipGetLastError();
}

}  // namespace nm
