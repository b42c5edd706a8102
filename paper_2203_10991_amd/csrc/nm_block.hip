// C ABI of the operators between a transformer block's linear layers: layer norm, rotary positions, attention.  Host-side argument validation and dispatch, as in nm_abi.hip.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/nm_mvue.h"
#include "nm_internal.h"

namespace nm {
int abi_fail(int code, const char *message);
void abi_clear();
}  // namespace nm

namespace {

int fail(int code, const char *fmt, ...)
{
    char text[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof text, fmt, ap);
    va_end(ap);
    return nm::abi_fail(code, text);
}
int launched(const char *fn, hipError_t e)
{
    if (e != hipSuccess) return fail(NM_ERR_LAUNCH, "%s: HIP launch failed: %s", fn, hipGetErrorString(e));
    nm::abi_clear();
    return NM_OK;
}
inline bool is_float(int dt) { return dt == NM_F32 || dt == NM_BF16; }
inline int64_t esize(int dt) { return dt == NM_BF16 ? 2 : 4; }
inline bool aligned(const void *p, int64_t to) { return (uintptr_t)p % (uintptr_t)to == 0; }

// What a call reads or writes: bytes lo .. hi - 1, and in them runs of `run` bytes that come again every step[0] bytes, all of those every step[1], and so on (steps rise; a
// step that appears less often than would fit counts as if it went on)
struct Range { uintptr_t lo, hi; int64_t run; int dims; int64_t step[3], span[4]; };      // span[i]: from the first to the last byte of what steps below i make
inline Range range_of(const void *p, int64_t bytes) { const int64_t n = p && bytes > 0 ? bytes : 0; return Range{(uintptr_t)p, (uintptr_t)p + (uintptr_t)n, n, 0, {}, {n}}; }
// n[i] times s[i] bytes apart
inline Range range_of(const void *p, int64_t run, const int64_t (&n)[3], const int64_t (&s)[3])
{
    Range r = range_of(p, run);
    int64_t count[3];
    for (int i = 0; i < 3; ++i) {
        if (n[i] < 2 || s[i] == 0) continue;
        int at = r.dims++;
        for (; at > 0 && r.step[at - 1] > s[i]; --at) { r.step[at] = r.step[at - 1]; count[at] = count[at - 1]; }
        r.step[at] = s[i];
        count[at] = n[i];
    }
    for (int i = 0; i < r.dims; ++i) r.span[i + 1] = r.span[i] + (count[i] - 1) * r.step[i];
    r.hi = r.lo + (uintptr_t)r.span[r.dims];
    return r;
}
// do the lower n steps of a, from byte x on, and the lower m steps of b, from byte y on, meet?  Only where both come in the same outermost step, which holds what lies within it, is that looked
// at more closely than from the first to the last byte: of a's repetitions at k step and b's at y - x + k step, one and its next can meet.
inline bool meet(const Range &a, int n, int64_t x, const Range &b, int m, int64_t y)
{
    if (x + a.span[n] <= y || y + b.span[m] <= x) return false;
    if (n == 0 || m == 0 || a.step[n - 1] != b.step[m - 1] || a.span[n - 1] > a.step[n - 1] || b.span[m - 1] > b.step[m - 1]) return true;
    const int64_t step = a.step[n - 1], off = ((y - x) % step + step) % step;
    return meet(a, n - 1, 0, b, m - 1, off) || meet(a, n - 1, step, b, m - 1, off);
}
inline bool overlap(const Range &a, const Range &b)
{
    if (a.lo >= b.hi || b.lo >= a.hi || a.lo == a.hi || b.lo == b.hi) return false;
    return a.lo < b.lo ? meet(a, a.dims, 0, b, b.dims, (int64_t)(b.lo - a.lo)) : meet(a, a.dims, (int64_t)(a.lo - b.lo), b, b.dims, 0);
}

constexpr int64_t LIM = (int64_t)1 << 56, STRIDE_MOST = (int64_t)1 << 40, SIZE_MOST = 0x7fffffff;
inline bool too_big(int64_t rows, int64_t stride) { return rows > LIM || stride > LIM || (rows > 0 && stride > 0 && rows > LIM / stride); }

// a matrix [R x C] of dt: sizes, stride, base
int check_matrix(const char *fn, const char *what, const void *p, int64_t R, int64_t C, int64_t ld, int dt)
{
    if (R < 0 || C < 0 || too_big(R, C) || too_big(R, ld)) return fail(NM_ERR_SHAPE, "%s: %s has sizes %lld x %lld, row stride %lld", fn, what, (long long)R, (long long)C, (long long)ld);
    if (R == 0 || C == 0) return NM_OK;
    if (!p) return fail(NM_ERR_NULL, "%s: %s is NULL", fn, what);
    if (R > 1 && ld < C) return fail(NM_ERR_SHAPE, "%s: row stride %lld of %s is smaller than %lld", fn, (long long)ld, what, (long long)C);
    if (!aligned(p, esize(dt))) return fail(NM_ERR_ALIGN, "%s: %s is not on its elements' boundary", fn, what);
    return NM_OK;
}
inline Range matrix_range(const void *p, int64_t R, int64_t C, int64_t ld, int dt)
{
    if (R < 1 || C < 1) return range_of(nullptr, 0);
    return range_of(p, C * esize(dt), {R, 1, 1}, {R > 1 ? ld * esize(dt) : 0, 0, 0});
}

constexpr int64_t NORM_MOST = 32768;
int check_norm(const char *fn, int64_t R, int64_t C, int x_dtype, int w_dtype)
{
    if (!is_float(x_dtype) || !is_float(w_dtype)) return fail(NM_ERR_DTYPE, "%s: tensors are NM_F32 (0) or NM_BF16 (1), got %d and %d", fn, x_dtype, w_dtype);
    if (R < 0 || C < 1 || C > NORM_MOST) return fail(NM_ERR_SHAPE, "%s: %lld rows of %lld (1 to 32768)", fn, (long long)R, (long long)C);
    return NM_OK;
}

// heads [B][T][H][D] of dt: strides, base
int check_heads(const char *fn, const char *what, const nm_heads *p, int64_t B, int64_t T, int64_t H, int64_t D, int dt, int64_t to, bool written)
{
    if (!p) return fail(NM_ERR_NULL, "%s: %s is NULL", fn, what);
    const int64_t n[3] = {B, T, H}, s[3] = {p->batch, p->token, p->head};
    int64_t span = D;
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (s[i] < 0 || s[i] > STRIDE_MOST || too_big(n[i], s[i]))) return fail(NM_ERR_SHAPE, "%s: strides %lld, %lld, %lld of %s", fn, (long long)s[0], (long long)s[1], (long long)s[2], what);
    if (B == 0 || T == 0 || H == 0) return NM_OK;
    if (!p->data) return fail(NM_ERR_NULL, "%s: %s is NULL", fn, what);
    if (!aligned(p->data, to)) return fail(NM_ERR_ALIGN, "%s: %s is not on a boundary of %lld bytes", fn, what, (long long)to);
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && s[i] * esize(dt) % to) return fail(NM_ERR_ALIGN, "%s: rows of %s are not on boundaries of %lld bytes", fn, what, (long long)to);
    if (!written) return NM_OK;
    // no element twice: each stride leaves room for what lies within it
    bool used[3] = {n[0] < 2, n[1] < 2, n[2] < 2};
    for (int k = 0; k < 3; ++k) {
        int least = -1;
        for (int i = 0; i < 3; ++i)
            if (!used[i] && (least < 0 || s[i] < s[least])) least = i;
        if (least < 0) break;
        if (s[least] < span) return fail(NM_ERR_SHAPE, "%s: elements of %s share memory (strides %lld, %lld, %lld)", fn, what, (long long)s[0], (long long)s[1], (long long)s[2]);
        span += (n[least] - 1) * s[least];
        used[least] = true;
    }
    return NM_OK;
}
inline Range heads_range(const nm_heads *p, int64_t B, int64_t T, int64_t H, int64_t D, int dt)
{
    if (B < 1 || T < 1 || H < 1 || D < 1) return range_of(nullptr, 0);
    const int64_t e = esize(dt);
    return range_of(p->data, D * e, {B, T, H}, {B > 1 ? p->batch * e : 0, T > 1 ? p->token * e : 0, H > 1 ? p->head * e : 0});
}
inline nm::AttnStride strides_of(const nm_heads *p, int64_t B, int64_t T, int64_t H) { return nm::AttnStride{B > 1 ? p->batch : 0, T > 1 ? p->token : 0, H > 1 ? p->head : 0}; }

// what the two attention calls have in common
int check_attention(const char *fn, nm::AttnArg &a, const nm_heads *q, const nm_heads *k, const nm_heads *v, int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hk, int64_t D, int dtype,
                    int causal, float scale, const int32_t *q_lens, const int32_t *k_lens)
{
    if (!is_float(dtype)) return fail(NM_ERR_DTYPE, "%s: tensors are NM_F32 (0) or NM_BF16 (1), got %d", fn, dtype);
    if (B < 0 || Tq < 0 || Tk < 0 || Hq < 0 || Hk < 0 || B > SIZE_MOST || Hq > SIZE_MOST || Tk > SIZE_MOST - 256) return fail(NM_ERR_SHAPE, "%s: B=%lld Tq=%lld Tk=%lld Hq=%lld Hk=%lld", fn, (long long)B, (long long)Tq, (long long)Tk, (long long)Hq, (long long)Hk);
    if (Hk == 0 ? Hq != 0 : Hq < Hk || Hq % Hk != 0) return fail(NM_ERR_SHAPE, "%s: %lld heads of queries are no multiple of %lld heads of keys", fn, (long long)Hq, (long long)Hk);
    if (D < 8 || D > 128 || D % 8) return fail(NM_ERR_SHAPE, "%s: heads of %lld elements (a multiple of 8 up to 128)", fn, (long long)D);
    const int64_t group = Hk ? Hq / Hk : 1;
    if (Tq > (SIZE_MOST - 256) / (group ? group : 1) || too_big(B * Hq, Tq * D * 4) || too_big(B * Hk, Tk * D * 4)) return fail(NM_ERR_SHAPE, "%s: %lld queries of %lld heads to a head of keys", fn, (long long)Tq, (long long)group);
    if (!(scale > 0.0f) || !isfinite(scale)) return fail(NM_ERR_UNSUPPORTED, "%s: scale %g has to be positive and finite", fn, scale);
    if (!aligned(q_lens, 4) || !aligned(k_lens, 4)) return fail(NM_ERR_ALIGN, "%s: lengths are not on a 4-byte boundary", fn);
    if (int rc = check_heads(fn, "q", q, B, Tq, Hq, D, dtype, 16, false)) return rc;
    if (int rc = check_heads(fn, "k", k, B, Tk, Hk, D, dtype, 16, false)) return rc;
    if (int rc = check_heads(fn, "v", v, B, Tk, Hk, D, dtype, 16, false)) return rc;
    a = nm::AttnArg{};
    a.q = q->data; a.k = k->data; a.v = v->data;
    a.sq = strides_of(q, B, Tq, Hq); a.sk = strides_of(k, B, Tk, Hk); a.sv = strides_of(v, B, Tk, Hk);
    a.q_lens = q_lens; a.k_lens = k_lens;
    a.B = (int)B; a.Tq = (int)Tq; a.Tk = (int)Tk; a.Hq = (int)Hq; a.Hk = (int)Hk; a.D = (int)D; a.dt = dtype; a.causal = causal != 0;
    a.group = (int)group;
    int bits = 0;
    while (((int64_t)1 << bits) < group) ++bits;
    a.group_shift = 31 + bits;
    // r * ceil(2^(31 + bits) / group) >> (31 + bits) is r / group for every r below 2^31
    a.group_mul = group ? (uint32_t)((((uint64_t)1 << a.group_shift) + group - 1) / group) : 0;
    a.scale = scale;
    return NM_OK;
}
int check_sizes(const char *fn, const nm::AttnArg &a, size_t need, const void *workspace, size_t workspace_bytes)
{
    if (need && (!workspace || workspace_bytes < need)) return fail(NM_ERR_WORKSPACE, "%s: workspace of %zu bytes required, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
    if (need && !aligned(workspace, 16)) return fail(NM_ERR_ALIGN, "%s: workspace needs a 16-byte aligned base", fn);
    return NM_OK;
}
// the sizes alone, for the workspaces: group 0 where a call would be refused or do nothing
nm::AttnArg sizes_of(int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hk, int64_t D, int dtype)
{
    nm::AttnArg a;
    const nm_heads none{nullptr, 0, 0, 0};
    nm_heads some{(void *)16, 0, 0, 0};
    if (B < 1 || Tq < 1 || Hk < 1 || Tk < 0 || check_attention("nm_attention_workspace", a, &some, Tk ? &some : &none, Tk ? &some : &none, B, Tq, Tk, Hq, Hk, D, dtype, 0, 1.0f, nullptr, nullptr)) a.group = 0;
    return a;
}

}  // namespace

extern "C" {

int nm_layer_norm(const void *x, int64_t ldx, int x_dtype, const void *w, const void *b, int w_dtype, int64_t R, int64_t C, float eps, void *y, int64_t ldy, float *mean, float *rstd,
                  void *hip_stream)
{
    const char *fn = "nm_layer_norm";
    if (int rc = check_norm(fn, R, C, x_dtype, w_dtype)) return rc;
    if (!(eps >= 0.0f) || !isfinite(eps)) return fail(NM_ERR_UNSUPPORTED, "%s: eps %g must be finite and not negative", fn, eps);
    if (int rc = check_matrix(fn, "x", x, R, C, ldx, x_dtype)) return rc;
    if (int rc = check_matrix(fn, "y", y, R, C, ldy, x_dtype)) return rc;
    if (!aligned(w, esize(w_dtype)) || !aligned(b, esize(w_dtype)) || !aligned(mean, 4) || !aligned(rstd, 4)) return fail(NM_ERR_ALIGN, "%s: w, b, mean or rstd is not on its elements' boundary", fn);
    const Range out[3] = {matrix_range(y, R, C, ldy, x_dtype), range_of(mean, R * 4), range_of(rstd, R * 4)};
    const Range in[3] = {matrix_range(x, R, C, ldx, x_dtype), range_of(w, C * esize(w_dtype)), range_of(b, C * esize(w_dtype))};
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < 3; ++j)
            if (overlap(out[i], in[j]) || (j < i && overlap(out[i], out[j]))) return fail(NM_ERR_ALIAS, "%s: outputs must not overlap inputs or each other", fn);
    return launched(fn, nm::launch_layer_norm(nm::NormArg{x, w, b, y, mean, rstd, R, C, ldx, ldy, x_dtype, w_dtype, eps}, (hipStream_t)hip_stream));
}

size_t nm_layer_norm_grad_workspace(int64_t R, int64_t C) { return R < 1 || C < 1 || C > NORM_MOST ? 0 : nm::layer_norm_grad_workspace(R, C); }

int nm_layer_norm_grad(const void *g, int64_t ldg, const void *x, int64_t ldx, int x_dtype, const void *w, int w_dtype, const float *mean, const float *rstd, int64_t R, int64_t C,
                       void *dx, int64_t lddx, void *dw, void *db, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const char *fn = "nm_layer_norm_grad";
    if (int rc = check_norm(fn, R, C, x_dtype, w_dtype)) return rc;
    if (int rc = check_matrix(fn, "g", g, R, C, ldg, x_dtype)) return rc;
    if (int rc = check_matrix(fn, "x", x, R, C, ldx, x_dtype)) return rc;
    if (int rc = check_matrix(fn, "dx", dx, R, C, lddx, x_dtype)) return rc;
    if (R > 0 && (!mean || !rstd)) return fail(NM_ERR_NULL, "%s: mean and rstd must not be NULL", fn);
    if (!aligned(w, esize(w_dtype)) || !aligned(dw, esize(w_dtype)) || !aligned(db, esize(w_dtype)) || !aligned(mean, 4) || !aligned(rstd, 4))
        return fail(NM_ERR_ALIGN, "%s: w, dw, db, mean or rstd is not on its elements' boundary", fn);
    const size_t need = dw || db ? nm_layer_norm_grad_workspace(R, C) : 0;
    if (need && (!workspace || workspace_bytes < need)) return fail(NM_ERR_WORKSPACE, "%s: workspace of %zu bytes required, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
    if (need && !aligned(workspace, 16)) return fail(NM_ERR_ALIGN, "%s: workspace needs a 16-byte aligned base", fn);
    const Range out[4] = {matrix_range(dx, R, C, lddx, x_dtype), range_of(dw, C * esize(w_dtype)), range_of(db, C * esize(w_dtype)), range_of(workspace, (int64_t)need)};
    const Range in[5] = {matrix_range(g, R, C, ldg, x_dtype), matrix_range(x, R, C, ldx, x_dtype), range_of(w, C * esize(w_dtype)), range_of(mean, R * 4), range_of(rstd, R * 4)};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 5; ++j)
            if (overlap(out[i], in[j]) || (j < i && overlap(out[i], out[j]))) return fail(NM_ERR_ALIAS, "%s: outputs and the workspace must not overlap inputs or each other", fn);
    float *part = dw || db ? (float *)(workspace ? workspace : (void *)16) : nullptr;                     // (R = 0 needs no workspace: the sums are zeros)
    return launched(fn, nm::launch_layer_norm_grad(nm::NormGradArg{g, x, w, mean, rstd, dx, dw, db, R, C, ldg, ldx, lddx, x_dtype, w_dtype, part}, (hipStream_t)hip_stream));
}

int nm_rotary(const nm_heads *x, const nm_heads *y, int dtype, int64_t B, int64_t T, int64_t H, int64_t D, int64_t part, const double *freqs, const void *positions, int position_bits,
              int64_t position_stride, int interleaved, float scale, int inverse, void *hip_stream)
{
    const char *fn = "nm_rotary";
    if (!is_float(dtype)) return fail(NM_ERR_DTYPE, "%s: tensors are NM_F32 (0) or NM_BF16 (1), got %d", fn, dtype);
    if (position_bits != 32 && position_bits != 64) return fail(NM_ERR_DTYPE, "%s: positions are 32 or 64 bits wide, got %d", fn, position_bits);
    if (B < 0 || T < 0 || H < 0 || D < 2 || D > 1024 || B > SIZE_MOST || T > SIZE_MOST || H > SIZE_MOST || B * T > SIZE_MOST)
        return fail(NM_ERR_SHAPE, "%s: B=%lld T=%lld H=%lld D=%lld (D from 2 to 1024, below 2^31 tokens)", fn, (long long)B, (long long)T, (long long)H, (long long)D);
    if (part < 2 || part > D || part % 2) return fail(NM_ERR_SHAPE, "%s: %lld elements of a head of %lld turned: an even number from 2 on", fn, (long long)part, (long long)D);
    if (!isfinite(scale)) return fail(NM_ERR_UNSUPPORTED, "%s: scale must be finite", fn);
    if (int rc = check_heads(fn, "x", x, B, T, H, D, dtype, esize(dtype), false)) return rc;
    if (int rc = check_heads(fn, "y", y, B, T, H, D, dtype, esize(dtype), true)) return rc;
    if (B == 0 || T == 0 || H == 0) { nm::abi_clear(); return NM_OK; }
    if (!freqs) return fail(NM_ERR_NULL, "%s: freqs is NULL", fn);
    if (!aligned(freqs, 8) || !aligned(positions, position_bits / 8)) return fail(NM_ERR_ALIGN, "%s: freqs or positions are not on their elements' boundary", fn);
    if (positions && (position_stride < 0 || too_big(B, position_stride))) return fail(NM_ERR_SHAPE, "%s: positions of the sequences %lld apart", fn, (long long)position_stride);
    const nm::AttnStride sx = strides_of(x, B, T, H), sy = strides_of(y, B, T, H);
    const Range ry = heads_range(y, B, T, H, D, dtype), rf = range_of(freqs, part / 2 * 8), rp = range_of(positions, ((B - 1) * position_stride + T) * (position_bits / 8));
    const bool in_place = x->data == y->data && sx.b == sy.b && sx.t == sy.t && sx.h == sy.h;
    if (overlap(ry, rf) || overlap(ry, rp) || (!in_place && overlap(ry, heads_range(x, B, T, H, D, dtype))))
        return fail(NM_ERR_ALIAS, "%s: y must be x itself or overlap no input", fn);
    return launched(fn, nm::launch_rotary(nm::RotaryArg{x->data, y->data, sx, sy, freqs, positions, position_stride, B, T, (int)H, (int)D, (int)part, position_bits == 64, interleaved != 0, dtype,
                                                        scale, inverse ? -1.0f : 1.0f}, (hipStream_t)hip_stream));
}

size_t nm_attention_workspace(int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hk, int64_t D, int dtype)
{
    const nm::AttnArg a = sizes_of(B, Tq, Tk, Hq, Hk, D, dtype);
    nm::abi_clear();
    return a.group ? nm::attention_workspace(a) : 0;
}

int nm_attention(const nm_heads *q, const nm_heads *k, const nm_heads *v, const nm_heads *o, float *lse, void *rest, int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hk, int64_t D, int dtype,
                 int causal, float scale, const int32_t *q_lens, const int32_t *k_lens, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const char *fn = "nm_attention";
    nm::AttnArg a;
    if (int rc = check_attention(fn, a, q, k, v, B, Tq, Tk, Hq, Hk, D, dtype, causal, scale, q_lens, k_lens)) return rc;
    if (int rc = check_heads(fn, "o", o, B, Tq, Hq, D, dtype, 16, true)) return rc;
    if (!aligned(lse, 4) || !aligned(rest, 4)) return fail(NM_ERR_ALIGN, "%s: lse or rest is not on a 4-byte boundary", fn);
    if (B == 0 || Tq == 0 || Hq == 0) { nm::abi_clear(); return NM_OK; }
    const size_t need = nm::attention_workspace(a);
    if (int rc = check_sizes(fn, a, need, workspace, workspace_bytes)) return rc;
    if (dtype == NM_F32) rest = nullptr;
    const Range out[4] = {heads_range(o, B, Tq, Hq, D, dtype), range_of(lse, B * Hq * Tq * 4), range_of(workspace, (int64_t)need), range_of(rest, B * Hq * Tq * D * 2)};
    const Range in[5] = {heads_range(q, B, Tq, Hq, D, dtype), heads_range(k, B, Tk, Hk, D, dtype), heads_range(v, B, Tk, Hk, D, dtype), range_of(q_lens, B * 4), range_of(k_lens, B * 4)};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 5; ++j)
            if (overlap(out[i], in[j]) || (j < i && overlap(out[i], out[j]))) return fail(NM_ERR_ALIAS, "%s: outputs and the workspace must not overlap inputs or each other", fn);
    a.o = o->data;
    a.so = strides_of(o, B, Tq, Hq);
    a.lse = lse;
    a.rest = rest;
    return launched(fn, nm::launch_attention(a, workspace, (hipStream_t)hip_stream));
}

size_t nm_attention_grad_workspace(int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hk, int64_t D, int dtype)
{
    const nm::AttnArg a = sizes_of(B, Tq, Tk, Hq, Hk, D, dtype);
    nm::abi_clear();
    return a.group ? nm::attention_grad_workspace(a) : 0;
}

int nm_attention_grad(const nm_heads *g, const nm_heads *q, const nm_heads *k, const nm_heads *v, const nm_heads *o, const float *lse, const void *rest, int64_t B, int64_t Tq, int64_t Tk, int64_t Hq,
                      int64_t Hk, int64_t D, int dtype, int causal, float scale, const int32_t *q_lens, const int32_t *k_lens, const nm_heads *dq, const nm_heads *dk, const nm_heads *dv,
                      void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const char *fn = "nm_attention_grad";
    nm::AttnArg a;
    if (int rc = check_attention(fn, a, q, k, v, B, Tq, Tk, Hq, Hk, D, dtype, causal, scale, q_lens, k_lens)) return rc;
    if (int rc = check_heads(fn, "g", g, B, Tq, Hq, D, dtype, 16, false)) return rc;
    if (int rc = check_heads(fn, "o", o, B, Tq, Hq, D, dtype, 16, false)) return rc;
    if (int rc = check_heads(fn, "dq", dq, B, Tq, Hq, D, dtype, 16, true)) return rc;
    if (int rc = check_heads(fn, "dk", dk, B, Tk, Hk, D, dtype, 16, true)) return rc;
    if (int rc = check_heads(fn, "dv", dv, B, Tk, Hk, D, dtype, 16, true)) return rc;
    if (B == 0 || Hq == 0) { nm::abi_clear(); return NM_OK; }
    if (Tq > 0 && !lse) return fail(NM_ERR_NULL, "%s: lse is NULL", fn);
    if (!aligned(lse, 4) || !aligned(rest, 4)) return fail(NM_ERR_ALIGN, "%s: lse or rest is not on a 4-byte boundary", fn);
    if (dtype == NM_F32) rest = nullptr;
    const size_t need = Tq > 0 ? nm::attention_grad_workspace(a) : 0;
    if (int rc = check_sizes(fn, a, need, workspace, workspace_bytes)) return rc;
    const Range out[4] = {heads_range(dq, B, Tq, Hq, D, dtype), heads_range(dk, B, Tk, Hk, D, dtype), heads_range(dv, B, Tk, Hk, D, dtype), range_of(workspace, (int64_t)need)};
    const Range in[9] = {heads_range(q, B, Tq, Hq, D, dtype), heads_range(k, B, Tk, Hk, D, dtype), heads_range(v, B, Tk, Hk, D, dtype), heads_range(g, B, Tq, Hq, D, dtype),
                         heads_range(o, B, Tq, Hq, D, dtype), range_of(lse, B * Hq * Tq * 4), range_of(q_lens, B * 4), range_of(k_lens, B * 4), range_of(rest, B * Hq * Tq * D * 2)};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 9; ++j)
            if (overlap(out[i], in[j]) || (j < i && overlap(out[i], out[j]))) return fail(NM_ERR_ALIAS, "%s: outputs and the workspace must not overlap inputs or each other", fn);
    a.g = g->data; a.o = o->data; a.dq = dq->data; a.dk = dk->data; a.dv = dv->data;
    a.sg = strides_of(g, B, Tq, Hq); a.so = strides_of(o, B, Tq, Hq); a.sdq = strides_of(dq, B, Tq, Hq); a.sdk = strides_of(dk, B, Tk, Hk); a.sdv = strides_of(dv, B, Tk, Hk);
    a.lse = (float *)lse;
    a.rest = (void *)rest;
    return launched(fn, nm::launch_attention_grad(a, workspace, (hipStream_t)hip_stream));
}

}  // extern "C"
