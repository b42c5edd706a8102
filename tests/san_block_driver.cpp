// Host side of csrc/nm_block.hip under AddressSanitizer and UndefinedBehaviorSanitizer: the launchers are stubs that check what they are given, so that calls with any
// sizes, strides and pointers pass through the validation.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "../include/nm_mvue.h"
#include "../paper_2203_10991_amd/csrc/nm_internal.h"

static long launches = 0, errors = 0;

static void expect(const char *what, long got, long want)
{
    if (got != want) { printf("%s: %ld, not %ld\n", what, got, want); ++errors; }
}

namespace nm {
int abi_fail(int code, const char *) { return code; }
void abi_clear() {}
hipError_t launch_layer_norm(const NormArg &, hipStream_t) { ++launches; return hipSuccess; }
size_t layer_norm_grad_workspace(int64_t R, int64_t C) { return (size_t)(R < 512 ? R : 512) * C * 8; }
hipError_t launch_layer_norm_grad(const NormGradArg &, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_rotary(const RotaryArg &, hipStream_t) { ++launches; return hipSuccess; }
size_t attention_workspace(const AttnArg &a) { return a.Tq == 1 ? (size_t)a.B * a.Hq * a.D * 4 : 0; }
size_t attention_grad_workspace(const AttnArg &a) { return (size_t)a.B * a.Hq * a.Tq * 4; }
static void check_group(const AttnArg &a)
{
    ++launches;
    if (a.group < 1 || (int64_t)a.group * a.Hk != a.Hq) { printf("group\n"); ++errors; }
    // row / group by multiplication, at every kind of row
    const int64_t rows = (int64_t)a.Tq * a.group;
    for (int64_t r : {(int64_t)0, (int64_t)1, (int64_t)a.group - 1, (int64_t)a.group, rows / 2, rows - a.group, rows - 1})
        if (r >= 0 && r < rows && (int64_t)((uint64_t)(uint32_t)r * a.group_mul >> a.group_shift) != r / a.group) { printf("row %ld / %d\n", (long)r, a.group); ++errors; }
}
hipError_t launch_attention(AttnArg a, void *, hipStream_t) { check_group(a); return hipSuccess; }
hipError_t launch_attention_grad(AttnArg a, void *, hipStream_t) { check_group(a); return hipSuccess; }
}  // namespace nm

int main()
{
    void *const at[] = {(void *)0x1000000000000, (void *)0x2000000000000, (void *)0x3000000000000, (void *)0x4000000000000, (void *)0x5000000000000, (void *)0x6000000000000,
                        (void *)0x7000000000000, (void *)0x8000000000000, (void *)0x9000000000000};
    const int64_t sizes[] = {-1, 0, 1, 7, 32768, (int64_t)1 << 21, (int64_t)1 << 30, (int64_t)1 << 31, (int64_t)1 << 40, (int64_t)1 << 58, INT64_MAX};
    long calls = 0;
    for (int64_t a : sizes)
        for (int64_t b : sizes)
            for (int64_t ld : sizes)
                for (int dt = 0; dt < 3; ++dt) {
                    nm_layer_norm(at[0], ld, dt, at[1], at[2], dt, a, b, 1e-5f, at[3], ld, (float *)at[4], (float *)at[5], nullptr);
                    nm_layer_norm_grad(at[0], ld, at[1], ld, dt, at[2], dt, (float *)at[3], (float *)at[4], a, b, at[5], ld, at[6], at[7], at[8], SIZE_MAX / 2, nullptr);
                    nm_layer_norm_grad_workspace(a, b);
                    for (int64_t other : {(int64_t)1, (int64_t)3, (int64_t)64, (int64_t)1 << 29}) {
                        const nm_heads x{at[0], ld, a, b}, y{at[1], ld, a, b}, z{at[2], ld, a, b}, o{at[3], ld, a, b}, w{at[4], INT64_MAX, ld, other};
                        nm_rotary(&x, &y, dt, a, b, other, 64, 32, (double *)at[3], at[4], 64, ld, 0, 1.f, 0, nullptr);
                        nm_rotary(&w, &x, dt, other, a, b, ld, 32, (double *)at[3], at[5], 32, ld, 1, 1.f, 1, nullptr);
                        nm_attention(&x, &y, &z, &o, (float *)at[4], nullptr, a, b, other, 8, 2, 64, dt, 1, 0.5f, (int *)at[5], (int *)at[6], at[7], SIZE_MAX / 2, nullptr);
                        nm_attention(&x, &w, &z, &o, (float *)at[5], nullptr, other, a, b, ld, other, 64, dt, 0, 0.5f, nullptr, nullptr, at[7], SIZE_MAX / 2, nullptr);
                        nm_attention_grad(&x, &y, &z, &o, &w, (float *)at[5], at[8], other, a, b, ld, ld, 8, dt, 1, 0.5f, nullptr, nullptr, &x, &y, &z, at[7], SIZE_MAX / 2, nullptr);
                        nm_attention_workspace(a, b, ld, other, other, 64, dt);
                        nm_attention_grad_workspace(other, a, b, ld, other, 64, dt);
                        calls += 7;
                    }
                }
    // groups of every size up to 300, with as many rows as are allowed
    launches = 0;
    for (int64_t g = 1; g <= 300; ++g) {
        const int64_t Tq = (0x7fffffff - 256) / g;
        const nm_heads q{at[0], 0, 64, 64}, k{at[1], 0, 64, 0}, v{at[2], 0, 64, 0}, o{at[3], 0, 64 * g, 64};
        expect("groups", nm_attention(&q, &k, &v, &o, nullptr, nullptr, 1, Tq, 10, g, 1, 64, 1, 0, 1.f, nullptr, nullptr, nullptr, 0, nullptr), NM_OK);
    }
    expect("calls that arrive", launches, 300);
    // outputs that are parts of one tensor, side by side and shifted
    const nm_heads in{at[0], 384 * 1000, 384, 64}, dq{at[1], 384 * 1000, 384, 64}, dk{(char *)at[1] + 256, 384 * 1000, 384, 64}, dv{(char *)at[1] + 512, 384 * 1000, 384, 64}, off{(char *)at[1] + 496, 384 * 1000, 384, 64};
    expect("parts", nm_attention_grad(&in, &in, &in, &in, &in, (float *)at[5], at[8], 3, 100, 100, 2, 2, 64, 1, 1, 1.f, nullptr, nullptr, &dq, &dk, &dv, at[7], 1 << 20, nullptr), NM_OK);
    expect("shifted parts", nm_attention_grad(&in, &in, &in, &in, &in, (float *)at[5], at[8], 3, 100, 100, 2, 2, 64, 1, 1, 1.f, nullptr, nullptr, &dq, &dk, &off, at[7], 1 << 20, nullptr), NM_ERR_ALIAS);
    // arrays at the end of the address space
    expect("norm at the end", nm_layer_norm((void *)(UINTPTR_MAX - 127), 8, 0, nullptr, nullptr, 0, 4, 8, 0.f, at[0], 8, nullptr, nullptr, nullptr), NM_OK);
    if (errors) return 1;
    printf("block sanitizer driver ok: %ld calls\n", calls);
    return 0;
}
