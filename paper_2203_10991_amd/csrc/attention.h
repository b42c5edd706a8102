// What the attention kernels share: arguments, tiles in LDS, matrix fragments.
//
// Heads of queries come in groups of `group` that share a head of keys and values.  The queries of a group are the rows of one matrix: row r is query r / group of the
// group's head r % group, so that shared heads need no sum over workgroups, a tile of rows spans few queries (little of a causal tile is empty), and one new token of a
// group fills a tile.  Row r sees the keys below seen(r): all of the sequence's, or where causal those up to the query's own place, the last query seeing the last key.
//
// Every product is D[m][n] += A[m][k] B[k][n] in 32 x 32 blocks, the operand that a wave keeps in registers as B: its lane l is column l % 32 for the whole kernel, and
// softmax statistics of a column are one number of a lane.  Lane l holds of A and B eight values of k, of D the rows 8 (i / 4) + 4 (l / 32) + i % 4.  The values of k may
// be taken in any order that A and B share: with slot (l / 32, j) as k = 8 (j / 4) + 4 (l / 32) + j % 4, eight values of a D block are, rounded, a B fragment as they lie.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "nm_internal.h"
#include "prune_common.h"        // pack_bf16_rne

namespace nm {

namespace attn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// rows of D = 32 BLOCKS or fewer elements in LDS, each in a power of two of 16-byte chunks; chunk c of row r lies at c ^ turn(r): 16 rows' same chunk, and the four
// rows x four chunks that a transposing read takes with 32 lanes, lie in 256 bytes of different banks
template <int DT, int BLOCKS> struct Tile {
    static constexpr int ES = DT == NM_DT_BF16 ? 2 : 4;
    static constexpr int CHUNKS = (BLOCKS == 3 ? 4 : BLOCKS) * 32 * ES / 16;       // of a row
    static constexpr int USED = BLOCKS * 32 * ES / 16;                             // that are read
    static constexpr int ROW = CHUNKS * 16;
    static constexpr int EC = 16 / ES;                                             // elements of a chunk
    static __device__ __forceinline__ int turn(int r)
    {
        const int low = r >> 2 & 3;
        if constexpr (CHUNKS >= 16) return (r & 3) << 2 | low;
        else if constexpr (CHUNKS == 8) return (r >> 1 & 1) << 2 | low;
        else return low;
    }
    static __device__ __forceinline__ int at(int r, int c) { return r * ROW + ((c ^ turn(r)) << 4); }
};

template <int DT> struct Frag;
template <> struct Frag<NM_DT_BF16> { bf16x8 v; };
template <> struct Frag<NM_DT_F32> { f32x8 v; };

__device__ __forceinline__ void mma(f32x16 &d, const Frag<NM_DT_BF16> &a, const Frag<NM_DT_BF16> &b) { d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, d, 0, 0, 0); }
__device__ __forceinline__ void mma(f32x16 &d, const Frag<NM_DT_F32> &a, const Frag<NM_DT_F32> &b)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) d = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], d, 0, 0, 0);
}

// Where a lane's fragments lie in LDS: the turns of rows and chunks are exclusive-ors, so the address of row r + r', chunk c + c' is the lane's own (r, c) with
// (c' ^ turn(r')) << 4 turned in, plus r' rows, as long as no bits meet.  Two registers and an exclusive-or before a read then take the place of a register for every
// read, which the kernels do not have: held in registers, addresses of 128-element heads made 27 to 45 spills in the dk dv kernel, whose reloads wait for the tiles on
// their way (2 x 8192 tokens, 64 heads over 8: 8.1 to 12.8 ms).
typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(const lds_char *)p; }
template <typename T> __device__ __forceinline__ T lds_read(uint32_t at) { return *(const __attribute__((address_space(3))) T *)(uintptr_t)at; }

template <int DT, int BLOCKS> struct Lane {
    typedef Tile<DT, BLOCKS> L;
    uint32_t row, col;               // relative to a tile
    __device__ __forceinline__ Lane(int lane)
    {
        const int hi = lane >> 5, e = lane & 31;
        row = (uint32_t)L::at(e, DT == NM_DT_BF16 ? hi : 2 * hi);
        // bf16: 16 lanes bring 4 rows x 16 elements, 8 bytes each, and get an element's 4 rows each
        if constexpr (DT == NM_DT_BF16) col = (uint32_t)(L::at(4 * hi + (lane >> 2 & 3), (lane >> 4 & 1) * 2 + (lane >> 1 & 1)) + (lane & 1) * 8);
        else col = (uint32_t)(L::at(4 * hi, e >> 2) + (e & 3) * 4);
    }
    static __device__ __forceinline__ uint32_t moved(uint32_t at, int r, int c) { return (at ^ (uint32_t)((c ^ L::turn(r)) << 4)) + (uint32_t)(r * L::ROW); }
    // the addresses in a tile, as the compiler shall not know them from the last tile's
    __device__ __forceinline__ uint32_t rows_of(uint32_t tile) const { uint32_t at = tile + row; asm volatile("" : "+v"(at)); return at; }
    __device__ __forceinline__ uint32_t columns_of(uint32_t tile) const { uint32_t at = tile + col; asm volatile("" : "+v"(at)); return at; }

    // A fragment of rows r0 .. r0 + 31 (r0 a multiple of 32) and elements 16 kk .. 16 kk + 15 (here k in its plain order); from: rows_of(tile)
    static __device__ __forceinline__ Frag<DT> rows(uint32_t from, int r0, int kk)
    {
        Frag<DT> f;
        if constexpr (DT == NM_DT_BF16) f.v = lds_read<bf16x8>(moved(from, r0, 2 * kk));
        else {
            const f32x4 a = lds_read<f32x4>(moved(from, r0, 4 * kk)), b = lds_read<f32x4>(moved(from, r0, 4 * kk + 1));
#pragma unroll
            for (int j = 0; j < 4; ++j) { f.v[j] = a[j]; f.v[4 + j] = b[j]; }
        }
        return f;
    }
    // A fragment of the transposed tile: elements 32 b .. 32 b + 31 as its rows, the tile's rows r0 .. r0 + 15 (r0 a multiple of 16) as k in the slots' order
    static __device__ __forceinline__ Frag<DT> columns(uint32_t from, int r0, int b)
    {
        Frag<DT> f;
        if constexpr (DT == NM_DT_BF16) {
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)moved(from, r0, 4 * b));
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)moved(from, r0 + 8, 4 * b));
            f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f.v[j] = lds_read<float>(moved(from, r0 + 8 * (j >> 2) + (j & 3), 8 * b));
        }
        return f;
    }
};

// eight values of a D block as a B fragment.  bf16: probabilities and their gradients are rounded to the operands' own type for the second product, to nearest; sums of
// probabilities take them before that
template <int DT> __device__ __forceinline__ Frag<DT> as_fragment(const f32x16 &d, int first)
{
    Frag<DT> f;
    if constexpr (DT == NM_DT_BF16) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack_bf16_rne(d[first + 2 * j], d[first + 2 * j + 1]);
        f.v = __builtin_bit_cast(bf16x8, w);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f.v[j] = d[first + j];
    }
    return f;
}

__device__ __forceinline__ int row_of(int i, int hi) { return 8 * (i >> 2) + 4 * hi + (i & 3); }        // of a D block
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ int query_of(int r, const AttnArg &p) { return (int)((uint64_t)(uint32_t)r * p.group_mul >> p.group_shift); }

// where a workgroup works, and the sequence's lengths
struct Sequence {
    int b, h, nq, nk;
    __device__ __forceinline__ Sequence(const AttnArg &p, int bh)
    {
        b = (int)((uint32_t)bh / (uint32_t)p.Hk); h = bh - b * p.Hk;
        // (lengths outside the tensors count as the nearest inside)
        nq = p.q_lens ? min(max(p.q_lens[b], 0), p.Tq) : p.Tq;
        nk = p.k_lens ? min(max(p.k_lens[b], 0), p.Tk) : p.Tk;
    }
    // keys that query i sees; not below 0
    __device__ __forceinline__ int seen(const AttnArg &p, int i) const { return p.causal ? max(0, min(nk, i + 1 + nk - nq)) : nk; }
};
// Workgroups go round-robin to the XCDs; each XCD takes a run of the list, so that the workgroups that read the same keys and values share an L2.
__device__ __forceinline__ uint32_t place_of(uint32_t id, uint32_t n)
{
    const uint32_t x = id % 8;
    return x * (n / 8) + min(x, n % 8) + id / 8;
}

// the first of part k of n parts of some tiles (2^26 at most)
__device__ __forceinline__ int part_of(int tiles, int k, int n) { return n == 1 ? k * tiles : k * (tiles / n) + min(k, tiles % n); }

__device__ __forceinline__ const char *row_at(const void *p, const AttnStride &s, int64_t b, int64_t t, int64_t h, int es) { return (const char *)p + (b * s.b + t * s.t + h * s.h) * es; }

// a row's B fragments: lane l has row `from` (its own), elements 16 kk + 8 (l / 32) ..; what lies behind D, and rows that are not there, are zeros
template <int DT, int BLOCKS> __device__ __forceinline__ void load_fragments(Frag<DT> (&f)[2 * BLOCKS], const char *from, bool there, int D, int lane)
{
    const int hi = lane >> 5;
#pragma unroll
    for (int kk = 0; kk < 2 * BLOCKS; ++kk) {
        const int e = 16 * kk + 8 * hi;
        const bool ok = there && e < D;
        const char *at = from + (ok ? e : 0) * Tile<DT, BLOCKS>::ES;
        if constexpr (DT == NM_DT_BF16) {
            u32x4 w = *(const u32x4 *)at;
            if (!ok) w = u32x4{0, 0, 0, 0};
            f[kk].v = __builtin_bit_cast(bf16x8, w);
        } else {
            f32x4 a = *(const f32x4 *)at, b = *(const f32x4 *)(at + 16);
            if (!ok) a = b = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) { f[kk].v[j] = a[j]; f[kk].v[4 + j] = b[j]; }
        }
    }
}

// ROWS rows of a tile on their way from memory to LDS through the registers of THREADS threads.  Rows behind `rows` and chunks behind D become zeros (a masked key's
// probability is zero, and zero times what a padded row may hold would not be).
template <int DT, int BLOCKS, int ROWS, int THREADS> struct Stage {
    typedef Tile<DT, BLOCKS> L;
    static constexpr int PIECES = ROWS * L::USED, N = (PIECES + THREADS - 1) / THREADS;
    u32x4 v[N];
    // at(row): the row's address; rows `from` .. rows - 1 of the tile are there, rows > 0.  What is not there is read from a row that is, and left out by store: a choice
    // made here would wait for the loads.
    template <typename At> __device__ __forceinline__ void load(const At &at, int rows, int D)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int piece = (int)threadIdx.x + n * THREADS, r = piece / L::USED, c = piece % L::USED;
            v[n] = *(const u32x4 *)(at(min(r, rows - 1)) + (c * L::EC < D ? c : 0) * 16);
        }
    }
    __device__ __forceinline__ void store(char *tile, int rows, int D, int from = 0) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int piece = (int)threadIdx.x + n * THREADS, r = piece / L::USED, c = piece % L::USED;
            const bool ok = r < rows && r >= from && c * L::EC < D;
            const u32x4 w = {ok ? v[n][0] : 0u, ok ? v[n][1] : 0u, ok ? v[n][2] : 0u, ok ? v[n][3] : 0u};
            if (PIECES % THREADS == 0 || piece < PIECES) *(u32x4 *)(tile + L::at(r, c)) = w;
        }
    }
};

// a column of D blocks (an output row of D elements) times `by`, to memory
template <int DT, int BLOCKS> __device__ __forceinline__ void store_column(char *to, const f32x16 (&d)[BLOCKS], float by, int D, int lane)
{
    const int hi = lane >> 5;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int e = 32 * b + 8 * (i >> 2) + 4 * hi;
            if (e >= D) continue;
            if constexpr (DT == NM_DT_BF16) *(u32x2 *)(to + e * 2) = u32x2{pack_bf16_rne(d[b][i] * by, d[b][i + 1] * by), pack_bf16_rne(d[b][i + 2] * by, d[b][i + 3] * by)};
            else *(f32x4 *)(to + e * 4) = f32x4{d[b][i] * by, d[b][i + 1] * by, d[b][i + 2] * by, d[b][i + 3] * by};
        }
}

}  // namespace attn

}  // namespace nm
