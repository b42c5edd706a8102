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

#include "gemm_plan.h"           // NM_CUS
#include "nm_internal.h"
#include "prune_common.h"        // pack_bf16_rne

namespace nm {

namespace attn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// Binary32 operands go through the bf16 instructions as three terms, x = x1 + x2 + x3, the first two rounded to nearest, the third what is left, which is exact: |x2| <= 2^-8, |x3| <= 2^-17
// of x's power of two.  A product takes the six products of terms down to 2^-16 of the first; x2 y3 + x3 y2 + x3 y3, which it leaves out, is 2^-24 of it at most, of either sign (cut off instead
// of rounded, the terms have x's sign and up to two and four times the size: what is left out is then up to 2^-21, always of the product's sign, and adds up over a sum.  Rounding costs
// nothing at 2 x 4096 tokens of 8 heads of 64, 1 to 2 % at 8 x 197 of 12, 3 to 4 % with heads of 32).  The binary32 instructions have a sixteenth of the bf16 ones' rate, six products an eighth of work to sixteen.  An infinity becomes NaN.
template <int DT> constexpr int TERMS = DT == NM_DT_BF16 ? 1 : 3;

// rows of D = 32 BLOCKS or fewer elements in LDS as bf16 (binary32: three tiles of terms), each in a power of two of 16-byte chunks; chunk c of row r lies at c ^ turn(r):
// 16 rows' same chunk, and the four rows x four chunks that a transposing read takes with 32 lanes, lie in 256 bytes of different banks
template <int BLOCKS> struct Tile {
    static constexpr int CHUNKS = (BLOCKS == 3 ? 4 : BLOCKS) * 4;                  // of a row
    static constexpr int ROW = CHUNKS * 16;
    static __device__ __forceinline__ int turn(int r)
    {
        const int low = r >> 2 & 3;
        if constexpr (CHUNKS == 16) return (r & 3) << 2 | low;
        else if constexpr (CHUNKS == 8) return (r >> 1 & 1) << 2 | low;
        else return low;
    }
    static __device__ __forceinline__ int at(int r, int c) { return r * ROW + ((c ^ turn(r)) << 4); }
};

template <int DT> struct Frag { bf16x8 v[TERMS<DT>]; };

__device__ __forceinline__ void mma(f32x16 &d, const bf16x8 &a, const bf16x8 &b) { d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, d, 0, 0, 0); }
template <int DT> __device__ __forceinline__ void mma(f32x16 &d, const Frag<DT> &a, const Frag<DT> &b)
{
    if constexpr (DT == NM_DT_F32) {
        mma(d, a.v[2], b.v[0]);
        mma(d, a.v[0], b.v[2]);
        mma(d, a.v[1], b.v[1]);
        mma(d, a.v[1], b.v[0]);
        mma(d, a.v[0], b.v[1]);
    }
    mma(d, a.v[0], b.v[0]);
}

// the upper halves of two words in one
__device__ __forceinline__ uint32_t upper(float lo, float hi) { return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u); }
// the terms of two values: word k holds term k of both.  WHOLE: up to the largest binary32 numbers (what would round to an infinity becomes the largest bf16 number, with a second
// term as large as a step of it), for the tensors' own values; without it from 2^128 - 2^119 on NaN, for probabilities and their gradients
template <bool WHOLE> __device__ __forceinline__ void terms_of(float x, float y, uint32_t (&w)[3])
{
    constexpr float MOST = 3.38953139e38f;
    w[0] = WHOLE ? pack_bf16_rne(__builtin_amdgcn_fmed3f(x, -MOST, MOST), __builtin_amdgcn_fmed3f(y, -MOST, MOST)) : pack_bf16_rne(x, y);
    const float rx = x - __uint_as_float(w[0] << 16), ry = y - __uint_as_float(w[0] & 0xffff0000u);
    w[1] = pack_bf16_rne(rx, ry);
    w[2] = upper(rx - __uint_as_float(w[1] << 16), ry - __uint_as_float(w[1] & 0xffff0000u));
}

// Where a lane's fragments lie in LDS: the turns of rows and chunks are exclusive-ors, so the address of row r + r', chunk c + c' is the lane's own (r, c) with
// (c' ^ turn(r')) << 4 turned in, plus r' rows, as long as no bits meet: tiles start at multiples of a row.  Two registers and an exclusive-or before a read then take the place of a register for every
// read, which the kernels do not have: held in registers, addresses of 128-element heads made 27 to 45 spills in the dk dv kernel, whose reloads wait for the tiles on
// their way (2 x 8192 tokens, 64 heads over 8: 8.1 to 12.8 ms).
typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(const lds_char *)p; }
template <typename T> __device__ __forceinline__ T lds_read(uint32_t at) { return *(const __attribute__((address_space(3))) T *)(uintptr_t)at; }

// ROWS: of a tile
template <int DT, int BLOCKS, int ROWS> struct Lane {
    typedef Tile<BLOCKS> L;
    static constexpr uint32_t TERM = ROWS * L::ROW, BYTES = TERMS<DT> * TERM;      // from a term's tile to the next one's, and of all of them
    // a tile starts with a row: `moved` turns bits of whole addresses, which are a row's own only then
    static constexpr uint32_t ALIGN = L::ROW;
    static_assert(TERM % ALIGN == 0 && BYTES % ALIGN == 0 && (ALIGN & (ALIGN - 1)) == 0 && ALIGN == 16 * L::CHUNKS, "tiles one behind the other start with a row each");
    uint32_t row, col;               // relative to a tile
    __device__ __forceinline__ Lane(int lane)
    {
        const int hi = lane >> 5;
        row = (uint32_t)L::at(lane & 31, hi);
        // 16 lanes bring 4 rows x 16 elements, 8 bytes each, and get an element's 4 rows each
        col = (uint32_t)(L::at(4 * hi + (lane >> 2 & 3), (lane >> 4 & 1) * 2 + (lane >> 1 & 1)) + (lane & 1) * 8);
    }
    static __device__ __forceinline__ uint32_t moved(uint32_t at, int r, int c) { return (at ^ (uint32_t)((c ^ L::turn(r)) << 4)) + (uint32_t)(r * L::ROW); }
    // the addresses in a tile, as the compiler shall not know them from the last tile's
    __device__ __forceinline__ uint32_t rows_of(uint32_t tile) const { uint32_t at = tile + row; asm volatile("" : "+v"(at)); return at; }
    __device__ __forceinline__ uint32_t columns_of(uint32_t tile) const { uint32_t at = tile + col; asm volatile("" : "+v"(at)); return at; }

    // A fragment of rows r0 .. r0 + 31 (r0 a multiple of 32) and elements 16 kk .. 16 kk + 15 (here k in its plain order); from: rows_of(tile)
    static __device__ __forceinline__ Frag<DT> rows(uint32_t from, int r0, int kk)
    {
        Frag<DT> f;
#pragma unroll
        for (int n = 0; n < TERMS<DT>; ++n) f.v[n] = lds_read<bf16x8>(moved(from, r0, 2 * kk) + n * TERM);
        return f;
    }
    // A fragment of the transposed tile: elements 32 b .. 32 b + 31 as its rows, the tile's rows r0 .. r0 + 15 (r0 a multiple of 16) as k in the slots' order
    static __device__ __forceinline__ Frag<DT> columns(uint32_t from, int r0, int b)
    {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        Frag<DT> f;
#pragma unroll
        for (int n = 0; n < TERMS<DT>; ++n) {
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(moved(from, r0, 4 * b) + n * TERM));
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(moved(from, r0 + 8, 4 * b) + n * TERM));
            f.v[n] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        return f;
    }
};

// eight values of a D block as a B fragment.  bf16: probabilities and their gradients are rounded to the operands' own type for the second product, to nearest; sums of
// probabilities take them before that
template <int DT, bool WHOLE = false> __device__ __forceinline__ Frag<DT> as_fragment(const f32x16 &d, int first)
{
    u32x4 w[TERMS<DT>];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (DT == NM_DT_BF16) w[0][j] = pack_bf16_rne(d[first + 2 * j], d[first + 2 * j + 1]);
        else {
            uint32_t t[3];
            terms_of<WHOLE>(d[first + 2 * j], d[first + 2 * j + 1], t);
#pragma unroll
            for (int n = 0; n < 3; ++n) w[n][j] = t[n];
        }
    }
    Frag<DT> f;
#pragma unroll
    for (int n = 0; n < TERMS<DT>; ++n) f.v[n] = __builtin_bit_cast(bf16x8, w[n]);
    return f;
}

// eight values less what that rounding made of them
template <int DT> __device__ __forceinline__ void take_rounded(f32x16 &d, int first, const Frag<DT> &f)
{
    const u32x4 w = __builtin_bit_cast(u32x4, f.v[0]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        d[first + 2 * j] -= __builtin_bit_cast(float, w[j] << 16);
        d[first + 2 * j + 1] -= __builtin_bit_cast(float, w[j] & 0xffff0000u);
    }
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
// Workgroups go round-robin to the XCDs; here each XCD takes 32 (its CUs) in a row of the list at a time, which mostly read the same keys and values and share its L2.  A
// head's tiles stand in the list by falling work, and sequences differ in length, so runs of 32 go to the XCDs forth and back (one long run to each left XCDs with the short
// sequences of a batch idle).  Where a CU holds two workgroups at once, its XCD's second 32 go in reverse, so that each CU starts with a long and a short one; where heads
// have few tiles, every other 32, since 32 are then whole heads and a CU would get the same tile of each.  2 x 4096 tokens, 8 heads of 64 in binary32, causal, all
// workgroups at once: forward 560 us without, 233 with; 32 x 512 tokens, 16 heads of 64: dk dv 95 and 81 us.  Where a CU holds one, the list as it is: whoever is
// done takes the longest that is left (2 x 8192 tokens, 64 heads of 128 over 8: dk dv 4.6 ms, in reverse 6.5).
__device__ __forceinline__ uint32_t place_of(uint32_t id, uint32_t n, bool every_other, bool two)
{
    const uint32_t x = id % 8, i = id / 8, round = i / 32, at = i % 32;
    if (round >= n / 256) return id;
    const bool reverse = every_other ? round & 1 : two && round == 1;
    return (round * 8 + (round & 1 ? 7 - x : x)) * 32 + (reverse ? 31 - at : at);
}
// a workgroup's head of keys, its tile in the order of falling work, and its part of it; the tiles of `mix` heads stand in the list together
struct Place {
    uint32_t bh;
    int tile, split;
    __device__ __forceinline__ Place(const AttnArg &p, int tiles, int splits, bool two)
    {
        const uint32_t at = place_of(blockIdx.x, gridDim.x, p.mix > 1 || tiles <= 16, two), whole = splits == 1 ? at : at / (uint32_t)splits;
        split = (int)(at - whole * splits);
        const uint32_t set = whole / (uint32_t)(tiles * p.mix), in = whole - set * tiles * p.mix, heads = min((uint32_t)p.mix, (uint32_t)(p.B * p.Hk) - set * p.mix);
        tile = (int)(in / heads);
        bh = set * p.mix + in - tile * heads;
    }
};
// How many heads that is.  Where the list is a few rounds long, all of them, so that the longest tiles of every head start first: forward / gradients, 6 x up to 1333 tokens, 12 heads of 80 over
// 1: 47 / 147 us a head at a time, 36 / 129 so; 4 x 2048, 16 heads of 64: 73 / 221 and 63 / 175; 12 x 1200, 12 heads of 40: 60 / 165 and 51 / 137; 8 x 1000, 16 heads of 64 over 4, lengths from
// half: 28.2 / 101 and 29.9 / 102.  Where it is longer, a head at a time (all: 2 x 8192, 64 heads of 128 over 8 2764 and 2865 us), but with lengths and many tiles to a head eight: empty tiles of short
// sequences come at the same place of every head's, which is the same XCD's (8 x up to 8192, 32 heads of 128 over 8 4900 / 13000 and 3490 / 11200; 4 x up to 4096 583 / 1840 and 522 / 1570;
// with 32 tiles to a head, 16 x up to 4096, 16 heads of 64, eight heads at a time are 674 / 1695 against 533 / 1490: runs of 32 no longer share keys).
inline int mix_of(const AttnArg &a, int64_t heads, int64_t tiles)
{
    if (!a.causal || tiles <= 8) return 1;
    if (heads * tiles <= 6 * NM_CUS) return (int)heads;
    return (a.q_lens || a.k_lens) && tiles >= 64 ? 8 : 1;
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
        if constexpr (DT == NM_DT_BF16) {
            u32x4 w = *(const u32x4 *)(from + (ok ? e : 0) * 2);
            if (!ok) w = u32x4{0, 0, 0, 0};
            f[kk].v[0] = __builtin_bit_cast(bf16x8, w);
        } else {
            const char *at = from + (ok ? e : 0) * 4;
            f32x4 a = *(const f32x4 *)at, b = *(const f32x4 *)(at + 16);
            if (!ok) a = b = f32x4{0, 0, 0, 0};
            f32x16 x;
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[j] = a[j]; x[4 + j] = b[j]; }
            f[kk] = as_fragment<DT, true>(x, 0);
        }
    }
}
// What rounding took from a bf16 o: word w of a row holds elements 2 w and 2 w + 1, and stands with word w of all rows, which lie as in lse.  (A cut of lse and of these planes
// beside each other is then what the cut tensors' call would leave.  32 rows of one head write, or read, 128 bytes in a run, those of a group shorter ones: 6 x up to 1333 tokens, 12 heads of 80 over
// 1, forward 40.5 us with a row's words in a run and 43.4 so, dq 53.5 and 55.2; 32 x 512, 16 heads of 64, 50 and 50, 73 and 65.)  at: the row's first word, null: none
struct Rest { uint32_t *at; int64_t apart; };
__device__ __forceinline__ Rest rest_at(const AttnArg &p, int64_t row) { return Rest{p.rest ? (uint32_t *)p.rest + row : nullptr, (int64_t)p.B * p.Hq * p.Tq}; }

// The product of a row x with y + rest, element by element, added up over this lane's elements.  f: x's fragments, zeros behind D (and where the row is not there; what y holds
// then does not count).  bf16: all loads first, none behind a choice: a row's words lie in as many places as it has pairs, and waiting for some of them before the next are on
// their way took dq of 32 x 512 tokens, 16 heads of 64, from 73 to 84 us
template <int DT, int BLOCKS> __device__ __forceinline__ float row_product(const Frag<DT> (&f)[2 * BLOCKS], const char *x, const char *y, const Rest &rest, int D, int lane)
{
    const int hi = lane >> 5;
    float sum = 0.0f;
    if constexpr (DT == NM_DT_BF16) {
        u32x4 o[2 * BLOCKS], d[2 * BLOCKS];
#pragma unroll
        for (int kk = 0; kk < 2 * BLOCKS; ++kk) {
            const int e = 16 * kk + 8 * hi;
            o[kk] = *(const u32x4 *)(y + (e < D ? e : 0) * 2);
        }
        if (rest.at) {
#pragma unroll
            for (int kk = 0; kk < 2 * BLOCKS; ++kk) {
                const int e = 16 * kk + 8 * hi;
                const uint32_t *from = rest.at + (e < D ? e / 2 : 0) * rest.apart;
#pragma unroll
                for (int j = 0; j < 4; ++j) d[kk][j] = from[j * rest.apart];
            }
        } else {
#pragma unroll
            for (int kk = 0; kk < 2 * BLOCKS; ++kk) d[kk] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int kk = 0; kk < 2 * BLOCKS; ++kk) {
            const bf16x8 a = f[kk].v[0], b = __builtin_bit_cast(bf16x8, o[kk]), c = __builtin_bit_cast(bf16x8, d[kk]);
            if (16 * kk + 8 * hi < D) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = __builtin_fmaf((float)a[j], (float)b[j], sum);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = __builtin_fmaf((float)a[j], (float)c[j], sum);
            }
        }
    } else {
#pragma unroll
        for (int kk = 0; kk < 2 * BLOCKS; ++kk) {
            const int e = 16 * kk + 8 * hi;
            if (e >= D) continue;
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                const f32x4 a = *(const f32x4 *)(x + (e + h) * 4), b = *(const f32x4 *)(y + (e + h) * 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum = __builtin_fmaf(a[j], b[j], sum);
            }
        }
    }
    return sum;
}

// ROWS rows of a tile on their way from memory to LDS through the registers of THREADS threads, 16 bytes at a time.  Rows behind `rows` and elements behind D become zeros (a
// masked key's probability is zero, and zero times what a padded row may hold would not be).
template <int DT, int BLOCKS, int ROWS, int THREADS> struct Stage {
    typedef Tile<BLOCKS> L;
    static constexpr int EC = DT == NM_DT_BF16 ? 8 : 4, USED = 32 * BLOCKS / EC;   // elements of a piece, pieces of a row
    static constexpr int PIECES = ROWS * USED, N = (PIECES + THREADS - 1) / THREADS;
    u32x4 v[N];
    // at(row): the row's address; `rows` > 0 of the tile's are there.  What is not there is read from a row that is, and left out by store: a choice made here would
    // wait for the loads.
    template <typename At> __device__ __forceinline__ void load(const At &at, int rows, int D)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int piece = (int)threadIdx.x + n * THREADS, r = piece / USED, c = piece % USED;
            v[n] = *(const u32x4 *)(at(min(r, rows - 1)) + (c * EC < D ? c : 0) * 16);
        }
    }
    // rows `from` .. rows - 1 are there
    __device__ __forceinline__ void store(char *tile, int rows, int D, int from = 0) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int piece = (int)threadIdx.x + n * THREADS, r = piece / USED, c = piece % USED;
            const bool ok = r < rows && r >= from && c * EC < D;
            const u32x4 w = {ok ? v[n][0] : 0u, ok ? v[n][1] : 0u, ok ? v[n][2] : 0u, ok ? v[n][3] : 0u};
            if (PIECES % THREADS != 0 && piece >= PIECES) continue;
            if constexpr (DT == NM_DT_BF16) *(u32x4 *)(tile + L::at(r, c)) = w;
            else {
                uint32_t lo[3], hi[3];
                terms_of<true>(__uint_as_float(w[0]), __uint_as_float(w[1]), lo);
                terms_of<true>(__uint_as_float(w[2]), __uint_as_float(w[3]), hi);
#pragma unroll
                for (int k = 0; k < 3; ++k) *(u32x2 *)(tile + k * ROWS * L::ROW + L::at(r, c >> 1) + (c & 1) * 8) = u32x2{lo[k], hi[k]};
            }
        }
    }
};

// four elements of a row, and (bf16) what rounding took from them
template <int DT> __device__ __forceinline__ void store_four(char *to, const Rest &rest, int e, const f32x4 &x)
{
    if constexpr (DT == NM_DT_BF16) {
        const u32x2 w = {pack_bf16_rne(x[0], x[1]), pack_bf16_rne(x[2], x[3])};
        *(u32x2 *)(to + e * 2) = w;
        if (rest.at) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
                rest.at[(e / 2 + j) * rest.apart] = pack_bf16_rne(x[2 * j] - __uint_as_float(w[j] << 16), x[2 * j + 1] - __uint_as_float(w[j] & 0xffff0000u));
        }
    } else *(f32x4 *)(to + e * 4) = x;
}
// Two words of both halves of a wave: the lower half keeps its first and gets the other's first behind it, the upper half keeps its second and gets the other's second in front
__device__ __forceinline__ void join_halves(uint32_t &first, uint32_t &second)
{
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(first, second, false, false));
    first = r[0];
    second = r[1];
}
// a column of D blocks (an output row of D elements) times `by`, to memory.  A lane holds 4 of every 8 elements of its row and lane + 32 the others; in bf16 they exchange
// every other 4, so that each writes 16 bytes.
template <int DT, int BLOCKS> __device__ __forceinline__ void store_column(char *to, const f32x16 (&d)[BLOCKS], float by, int D, int lane, const Rest &rest = Rest{nullptr, 0})
{
    const int hi = lane >> 5;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        if constexpr (DT == NM_DT_BF16) {
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                const int e = 32 * b + 2 * i + 8 * hi;
                float x[8];
                uint32_t w[4], r[4];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = d[b][i + j] * by;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    w[j] = pack_bf16_rne(x[2 * j], x[2 * j + 1]);
                    r[j] = pack_bf16_rne(x[2 * j] - __uint_as_float(w[j] << 16), x[2 * j + 1] - __uint_as_float(w[j] & 0xffff0000u));
                }
                join_halves(w[0], w[2]);
                join_halves(w[1], w[3]);
                if (e < D) *(u32x4 *)(to + e * 2) = u32x4{w[0], w[1], w[2], w[3]};
                if (rest.at) {                                           // (as they lie: 4 elements from the first eight, 4 from the second)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (32 * b + 2 * i + 4 * (j & 2) < D) rest.at[(16 * b + i + 4 * (j >> 1) + 2 * hi + (j & 1)) * rest.apart] = r[j];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int e = 32 * b + 8 * (i >> 2) + 4 * hi;
                if (e < D) *(f32x4 *)(to + e * 4) = f32x4{d[b][i] * by, d[b][i + 1] * by, d[b][i + 2] * by, d[b][i + 3] * by};
            }
        }
    }
}

// the sum of a fragment's values as they are rounded
__device__ __forceinline__ float sum_of(const Frag<NM_DT_BF16> &f, float sum)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
    const bf16x2 *p = (const bf16x2 *)&f.v[0];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = __builtin_amdgcn_fdot2_f32_bf16(p[j], one, sum, false);
    return sum;
}

}  // namespace attn

}  // namespace nm
