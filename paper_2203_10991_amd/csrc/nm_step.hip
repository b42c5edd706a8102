// C ABI of the operators around the update phase: AdamW.  Host-side argument validation and dispatch, as in nm_abi.hip.
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

}  // namespace

extern "C" {

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
