// C ABI of the operators around the update phase: 8-bit integer products, embedding, AdamW.  Host-side argument validation and dispatch, as in nm_abi.hip.
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
struct Range { uintptr_t lo, hi; };
inline Range range_of(const void *p, int64_t bytes) { return Range{(uintptr_t)p, (uintptr_t)p + (uintptr_t)(p && bytes > 0 ? bytes : 0)}; }
inline bool overlap(const Range &a, const Range &b) { return a.lo < b.hi && b.lo < a.hi && a.lo != a.hi && b.lo != b.hi; }

// rows x stride elements must stay far below 2^63 bytes: every byte range below is formed without overflow
inline bool too_big(int64_t rows, int64_t stride)
{
    const int64_t lim = (int64_t)1 << 56;
    return rows > lim || stride > lim || (rows > 0 && stride > 0 && rows > lim / stride);
}
// a matrix [R x C] of dt: sizes, stride, base
int check_matrix(const char *fn, const char *what, const void *p, int64_t R, int64_t C, int64_t ld, int dt)
{
    if (!is_float(dt)) return fail(NM_ERR_DTYPE, "%s: %s is NM_F32 (0) or NM_BF16 (1), got %d", fn, what, dt);
    if (R < 0 || C < 0 || too_big(R, C) || too_big(R, ld)) return fail(NM_ERR_SHAPE, "%s: %s has sizes %lld x %lld, row stride %lld", fn, what, (long long)R, (long long)C, (long long)ld);
    if (R == 0 || C == 0) return NM_OK;
    if (!p) return fail(NM_ERR_NULL, "%s: %s is NULL", fn, what);
    if (R > 1 && ld < C) return fail(NM_ERR_SHAPE, "%s: row stride %lld of %s is smaller than %lld", fn, (long long)ld, what, (long long)C);
    if (!aligned(p, esize(dt))) return fail(NM_ERR_ALIGN, "%s: %s is not on its elements' boundary", fn, what);
    return NM_OK;
}
inline Range matrix_range(const void *p, int64_t R, int64_t C, int64_t ld, int dt) { return range_of(p, R > 0 && C > 0 ? ((R - 1) * ld + C) * esize(dt) : 0); }
int check_ids(const char *fn, const void *ids, int bits, int64_t N)
{
    if (bits != 32 && bits != 64) return fail(NM_ERR_DTYPE, "%s: ids are 32 or 64 bits wide, got %d", fn, bits);
    if (N < 0 || N > 0x7fffffff - 65536) return fail(NM_ERR_SHAPE, "%s: %lld tokens", fn, (long long)N);
    if (N && !ids) return fail(NM_ERR_NULL, "%s: ids is NULL", fn);
    if (N && !aligned(ids, bits / 8)) return fail(NM_ERR_ALIGN, "%s: ids are not on their elements' boundary", fn);
    return NM_OK;
}

constexpr int64_t I8_SIZE = (int64_t)1 << 30, I8_LD = (int64_t)1 << 21, I8_K_MOST = 131072;

// codes [R x C] of 8-bit integers with a scale for each row
int check_codes(const char *fn, const char *what, const int8_t *q, int64_t ld, const float *scale, int64_t R, int64_t C)
{
    if (R < 0 || C < 0 || R > I8_SIZE || C > I8_SIZE) return fail(NM_ERR_SHAPE, "%s: %s has sizes %lld x %lld", fn, what, (long long)R, (long long)C);
    if (ld < C || ld % 16 || ld > I8_LD) return fail(ld % 16 ? NM_ERR_ALIGN : NM_ERR_SHAPE, "%s: row stride %lld of %s has to be a multiple of 16 from %lld to 2^21", fn, (long long)ld, what, (long long)C);
    if (R == 0) return NM_OK;
    if (!q || !scale) return fail(NM_ERR_NULL, "%s: %s and its scales must not be NULL", fn, what);
    if (!aligned(q, 16) || !aligned(scale, 4)) return fail(NM_ERR_ALIGN, "%s: %s needs a 16-byte aligned base, its scales a 4-byte aligned one", fn, what);
    return NM_OK;
}
inline Range codes_range(const int8_t *q, int64_t ld, int64_t R) { return range_of(q, R * ld); }
// ... as an input: its last row may end with its last whole 16 bytes
inline Range codes_in(const int8_t *q, int64_t ld, int64_t R, int64_t C) { return range_of(q, R ? (R - 1) * ld + (C + 15) / 16 * 16 : 0); }
inline int64_t i8_row(int64_t I) { return (I + nm::I8_K - 1) / nm::I8_K * nm::I8_K; }

// what the two products have in common: w, bias and y
int check_product(const char *fn, const int8_t *wq, int64_t ldw, const float *ws, const void *bias, int bias_dtype, int64_t T, int64_t O, int64_t I, const void *y, int64_t ldy, int y_dtype)
{
    if (T < 0 || O < 0 || I < 1 || T > I8_SIZE || O > I8_SIZE || I > I8_K_MOST)
        return fail(NM_ERR_SHAPE, "%s: T=%lld O=%lld I=%lld (I from 1 to 131072: the sums are 32-bit integers)", fn, (long long)T, (long long)O, (long long)I);
    if (int rc = check_codes(fn, "w", wq, ldw, ws, O, I)) return rc;
    if (int rc = check_matrix(fn, "y", y, T, O, ldy, y_dtype)) return rc;
    if (ldy > I8_LD || O > I8_LD) return fail(NM_ERR_SHAPE, "%s: rows of y are at most 2^21 elements apart", fn);
    if (bias && !is_float(bias_dtype)) return fail(NM_ERR_DTYPE, "%s: bias is NM_F32 (0) or NM_BF16 (1), got %d", fn, bias_dtype);
    if (bias && !aligned(bias, esize(bias_dtype))) return fail(NM_ERR_ALIGN, "%s: bias is not on its elements' boundary", fn);
    const Range ry = matrix_range(y, T, O, ldy, y_dtype);
    if (overlap(ry, codes_in(wq, ldw, O, I)) || overlap(ry, range_of(ws, O * 4)) || overlap(ry, range_of(bias, O * esize(bias_dtype)))) return fail(NM_ERR_ALIAS, "%s: y must not overlap an input", fn);
    return NM_OK;
}

}  // namespace

extern "C" {

int nm_quant_i8(const void *x, int64_t R, int64_t C, int64_t ldx, int dtype, int8_t *q, int64_t ldq, float *scale, void *hip_stream)
{
    const char *fn = "nm_quant_i8";
    if (int rc = check_matrix(fn, "x", x, R, C, ldx, dtype)) return rc;
    if (int rc = check_codes(fn, "q", q, ldq, scale, R, C)) return rc;
    const Range rx = matrix_range(x, R, C, ldx, dtype), rq = codes_range(q, ldq, R), rs = range_of(scale, R * 4);
    if (overlap(rq, rx) || overlap(rs, rx) || overlap(rq, rs)) return fail(NM_ERR_ALIAS, "%s: q and scale must not overlap x or each other", fn);
    return launched(fn, nm::launch_quant_i8(dtype, x, R, C, ldx, q, ldq, scale, (hipStream_t)hip_stream));
}

size_t nm_quant_i8_t_workspace(int64_t R, int64_t C) { return R < 0 || C <= 0 || R > I8_SIZE || C > I8_LD ? 0 : (size_t)nm::quant_i8_slabs(R, C) * (size_t)C * 4; }

int nm_quant_i8_t(const void *x, int64_t R, int64_t C, int64_t ldx, int dtype, int8_t *q, int64_t ldq, float *scale, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const char *fn = "nm_quant_i8_t";
    if (int rc = check_matrix(fn, "x", x, R, C, ldx, dtype)) return rc;
    if (C > I8_LD) return fail(NM_ERR_SHAPE, "%s: %lld columns, 2^21 at most", fn, (long long)C);
    if (int rc = check_codes(fn, "q", q, ldq, scale, C, R)) return rc;
    const size_t need = nm_quant_i8_t_workspace(R, C);
    if (need && (!workspace || workspace_bytes < need)) return fail(NM_ERR_WORKSPACE, "%s: workspace of %zu bytes required, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
    if (need && !aligned(workspace, 16)) return fail(NM_ERR_ALIGN, "%s: workspace needs a 16-byte aligned base", fn);
    const Range rx = matrix_range(x, R, C, ldx, dtype), rq = codes_range(q, ldq, C), rs = range_of(scale, C * 4), rw = range_of(workspace, (int64_t)need);
    if (overlap(rq, rx) || overlap(rs, rx) || overlap(rq, rs) || overlap(rw, rx) || overlap(rw, rq) || overlap(rw, rs))
        return fail(NM_ERR_ALIAS, "%s: q, scale and the workspace must not overlap x or each other", fn);
    return launched(fn, nm::launch_quant_i8_t(dtype, x, R, C, ldx, q, ldq, scale, (uint32_t *)workspace, (hipStream_t)hip_stream));
}

int nm_gemm_i8(const int8_t *xq, int64_t ldx, const float *xs, const int8_t *wq, int64_t ldw, const float *ws, const void *bias, int bias_dtype, int64_t T, int64_t O,
               int64_t I, int relu, void *y, int64_t ldy, int y_dtype, void *hip_stream)
{
    const char *fn = "nm_gemm_i8";
    if (int rc = check_product(fn, wq, ldw, ws, bias, bias_dtype, T, O, I, y, ldy, y_dtype)) return rc;
    if (int rc = check_codes(fn, "x", xq, ldx, xs, T, I)) return rc;
    const Range ry = matrix_range(y, T, O, ldy, y_dtype);
    if (overlap(ry, codes_in(xq, ldx, T, I)) || overlap(ry, range_of(xs, T * 4))) return fail(NM_ERR_ALIAS, "%s: y must not overlap an input", fn);
    return launched(fn, nm::launch_gemm_i8(nm::I8Arg{xq, wq, xs, ws, bias, y, ldx, ldw, ldy, T, O, I, bias_dtype, y_dtype, relu, 0}, (hipStream_t)hip_stream));
}

size_t nm_linear_i8_workspace(int64_t T, int64_t I) { return T <= 0 || I < 1 || T > I8_SIZE || I > I8_K_MOST ? 0 : (size_t)T * (size_t)i8_row(I) + ((size_t)T * 4 + 15) / 16 * 16; }

int nm_linear_i8(const void *x, int64_t ldx, int x_dtype, const int8_t *wq, int64_t ldw, const float *ws, const void *bias, int bias_dtype, int64_t T, int64_t O, int64_t I,
                 int relu, void *y, int64_t ldy, int y_dtype, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const char *fn = "nm_linear_i8";
    if (int rc = check_product(fn, wq, ldw, ws, bias, bias_dtype, T, O, I, y, ldy, y_dtype)) return rc;
    if (int rc = check_matrix(fn, "x", x, T, I, ldx, x_dtype)) return rc;
    if (T == 0 || O == 0) { nm::abi_clear(); return NM_OK; }
    const size_t need = nm_linear_i8_workspace(T, I);
    if (!workspace || workspace_bytes < need) return fail(NM_ERR_WORKSPACE, "%s: workspace of %zu bytes required, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
    if (!aligned(workspace, 16)) return fail(NM_ERR_ALIGN, "%s: workspace needs a 16-byte aligned base", fn);
    const Range rx = matrix_range(x, T, I, ldx, x_dtype), ry = matrix_range(y, T, O, ldy, y_dtype), rw = range_of(workspace, (int64_t)need);
    if (overlap(ry, rx) || overlap(rw, rx) || overlap(rw, ry) || overlap(rw, codes_in(wq, ldw, O, I)) || overlap(rw, range_of(ws, O * 4)) || overlap(rw, range_of(bias, O * esize(bias_dtype))))
        return fail(NM_ERR_ALIAS, "%s: y and the workspace must not overlap an input or each other", fn);
    const int64_t row = i8_row(I);
    int8_t *q = (int8_t *)workspace;
    float *s = (float *)(q + T * row);
    hipStream_t st = (hipStream_t)hip_stream;
    const nm::I8Arg product{q, wq, s, ws, bias, y, row, ldw, ldy, T, O, I, bias_dtype, y_dtype, relu, 1};
    if (nm::gemm_i8_few_fused(T, I)) return launched(fn, nm::launch_gemm_i8_few(product, x, ldx, x_dtype, st));
    hipError_t e = nm::launch_quant_i8(x_dtype, x, T, I, ldx, q, row, s, st);
    if (e == hipSuccess) e = nm::launch_gemm_i8(product, st);
    return launched(fn, e);
}

int nm_embed(const void *table, int64_t V, int64_t D, int64_t ldt, int table_dtype, const void *ids, int id_bits, int64_t N, float scale, void *out, int64_t ldo,
             int out_dtype, void *hip_stream)
{
    const char *fn = "nm_embed";
    if (int rc = check_ids(fn, ids, id_bits, N)) return rc;
    if (int rc = check_matrix(fn, "table", table, V, D, ldt, table_dtype)) return rc;
    if (int rc = check_matrix(fn, "out", out, N, D, ldo, out_dtype)) return rc;
    const Range ro = matrix_range(out, N, D, ldo, out_dtype);
    if (overlap(ro, matrix_range(table, V, D, ldt, table_dtype)) || overlap(ro, range_of(ids, N * id_bits / 8))) return fail(NM_ERR_ALIAS, "%s: out must not overlap the table or the ids", fn);
    return launched(fn, nm::launch_embed(table_dtype, out_dtype, table, V, D, ldt, ids, id_bits == 64, N, scale, out, ldo, (hipStream_t)hip_stream));
}

size_t nm_embed_grad_workspace(int64_t N, int64_t V, int64_t D)
{
    if (N <= 0 || V < 0 || D <= 0 || N > 0x7fffffff - 65536 || V > 0x7ffffffe || D > ((int64_t)1 << 32)) return 0;
    return nm::embed_grad_workspace(N, V, D);
}

int nm_embed_grad(const void *g, int64_t ldg, int g_dtype, const void *ids, int id_bits, int64_t N, int64_t V, int64_t D, float scale, int64_t padding, int accumulate,
                  void *out, int64_t ldo, int out_dtype, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const char *fn = "nm_embed_grad";
    if (int rc = check_ids(fn, ids, id_bits, N)) return rc;
    if (V > 0x7ffffffe || D > ((int64_t)1 << 32)) return fail(NM_ERR_SHAPE, "%s: a table of %lld x %lld", fn, (long long)V, (long long)D);
    if (int rc = check_matrix(fn, "g", g, N, D, ldg, g_dtype)) return rc;
    if (int rc = check_matrix(fn, "out", out, V, D, ldo, out_dtype)) return rc;
    if (V == 0 || D == 0) { nm::abi_clear(); return NM_OK; }
    const size_t need = nm_embed_grad_workspace(N, V, D);
    if (need && (!workspace || workspace_bytes < need)) return fail(NM_ERR_WORKSPACE, "%s: workspace of %zu bytes required, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
    if (need && !aligned(workspace, 16)) return fail(NM_ERR_ALIGN, "%s: workspace needs a 16-byte aligned base", fn);
    const Range rg = matrix_range(g, N, D, ldg, g_dtype), ro = matrix_range(out, V, D, ldo, out_dtype), ri = range_of(ids, N * id_bits / 8), rw = range_of(workspace, (int64_t)need);
    if (overlap(ro, rg) || overlap(ro, ri) || overlap(rw, ro) || overlap(rw, rg) || overlap(rw, ri))
        return fail(NM_ERR_ALIAS, "%s: out and the workspace must not overlap an input or each other", fn);
    return launched(fn, nm::launch_embed_grad(g_dtype, out_dtype, g, ldg, ids, id_bits == 64, N, V, D, scale, padding, accumulate != 0, out, ldo, workspace, (hipStream_t)hip_stream));
}

int nm_adamw(const nm_adamw_tensor *tensors, int count, int param_dtype, int grad_dtype, int state, double lr, double beta1, double beta2,
             double eps, double weight_decay, int64_t step, float grad_scale, const float *grad_scale_dev, uint64_t seed, void *hip_stream)
{
    const char *fn = "nm_adamw";
    if (!is_float(param_dtype) || !is_float(grad_dtype)) return fail(NM_ERR_DTYPE, "%s: parameters and gradients are NM_F32 (0) or NM_BF16 (1), got %d and %d", fn, param_dtype, grad_dtype);
    if (state != NM_STATE_F32 && state != NM_STATE_Q8) return fail(NM_ERR_UNSUPPORTED, "%s: state %d is not NM_STATE_F32 (0) or NM_STATE_Q8 (1)", fn, state);
    if (count < 0) return fail(NM_ERR_SHAPE, "%s: negative count", fn);
    if (step < 1 || step > 0x7fffffff) return fail(NM_ERR_SHAPE, "%s: step %lld is not in 1 .. 2^31 - 1", fn, (long long)step);
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0)) return fail(NM_ERR_UNSUPPORTED, "%s: betas %g, %g are not in [0, 1)", fn, beta1, beta2);
    if (!(eps >= 0.0) || !isfinite(eps) || !isfinite(lr) || !isfinite(weight_decay)) return fail(NM_ERR_UNSUPPORTED, "%s: lr, eps and weight_decay must be finite, eps not negative", fn);
    if (count == 0) { nm::abi_clear(); return NM_OK; }
    if (!tensors) return fail(NM_ERR_NULL, "%s: tensors is NULL", fn);
    if (!aligned(grad_scale_dev, 4)) return fail(NM_ERR_ALIGN, "%s: grad_scale_dev is not on a 4-byte boundary", fn);
    const bool q8 = state == NM_STATE_Q8;
    bool master = false, known = false;
    for (int k = 0; k < count; ++k) {
        const nm_adamw_tensor &t = tensors[k];
        if (t.n < 0 || t.n > ((int64_t)1 << 40)) return fail(NM_ERR_SHAPE, "%s: tensor %d has %lld elements", fn, k, (long long)t.n);
        if (t.n == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v || (q8 && (!t.m_scale || !t.v_scale)))
            return fail(NM_ERR_NULL, "%s: param, grad, m, v%s of tensor %d must not be NULL", fn, q8 ? ", m_scale and v_scale" : "", k);
        if (t.master && param_dtype == NM_F32) return fail(NM_ERR_UNSUPPORTED, "%s: tensor %d: a binary32 parameter is its own master copy", fn, k);
        if (known && master != (t.master != nullptr)) return fail(NM_ERR_UNSUPPORTED, "%s: some tensors have a master copy and some have none: two calls", fn);
        known = true;
        master = t.master != nullptr;
        if (!aligned(t.param, esize(param_dtype)) || !aligned(t.grad, esize(grad_dtype)) || !aligned(t.master, 4) ||
            (!q8 && (!aligned(t.m, 4) || !aligned(t.v, 4))) || (q8 && (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))))
            return fail(NM_ERR_ALIGN, "%s: an array of tensor %d is not on its elements' boundary", fn, k);
        const int64_t sb = q8 ? t.n : 4 * t.n, scales = q8 ? (t.n + 255) / 256 * 4 : 0;
        const Range r[7] = {range_of(t.param, t.n * esize(param_dtype)), range_of(t.grad, t.n * esize(grad_dtype)), range_of(t.m, sb), range_of(t.v, sb),
                            range_of(t.master, 4 * t.n), range_of(t.m_scale, scales), range_of(t.v_scale, scales)};
        for (int i = 0; i < 7; ++i)
            for (int j = 0; j < i; ++j)
                if (overlap(r[i], r[j])) return fail(NM_ERR_ALIAS, "%s: the arrays of tensor %d must not overlap", fn, k);
    }
    const nm::AdamwRates rates{lr, beta1, beta2, eps, weight_decay, step, grad_scale, grad_scale_dev};
    nm::AdamwTensor part[nm::ADAMW_MOST];
    int have = 0;
    for (int k = 0; k < count; ++k) {
        const nm_adamw_tensor &t = tensors[k];
        if (t.n > 0) {
            const bool al = aligned(t.param, 16) && aligned(t.grad, 16) && aligned(t.m, 16) && aligned(t.v, 16) && aligned(t.master, 16);
            part[have++] = nm::AdamwTensor{t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.master, t.n, t.number, al};
        }
        if (have == nm::ADAMW_MOST || (k == count - 1 && have)) {
            const hipError_t e = nm::launch_adamw(part, have, param_dtype, grad_dtype, q8, master, rates, seed, (hipStream_t)hip_stream);
            if (e != hipSuccess) return launched(fn, e);
            have = 0;
        }
    }
    return launched(fn, hipSuccess);
}

}  // extern "C"
