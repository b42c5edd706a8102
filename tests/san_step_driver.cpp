// Host side of csrc/nm_step.hip under AddressSanitizer and UndefinedBehaviorSanitizer: the launchers are stubs that only count, so that calls with any sizes and
// pointers pass through the validation.  Sizes whose byte ranges could overflow, pointers at the end of the address space, tables of many tensors.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "../include/nm_mvue.h"
#include "../paper_2203_10991_amd/csrc/nm_internal.h"

static int launches = 0, tensors_seen = 0, errors = 0;

namespace nm {
int abi_fail(int code, const char *) { return code; }
void abi_clear() {}
hipError_t launch_quant_i8(int, const void *, int64_t, int64_t, int64_t, int8_t *, int64_t, float *, hipStream_t) { ++launches; return hipSuccess; }
int quant_i8_slabs(int64_t, int64_t) { return 64; }
hipError_t launch_quant_i8_t(int, const void *, int64_t, int64_t, int64_t, int8_t *, int64_t, float *, uint32_t *, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_gemm_i8(const I8Arg &, hipStream_t) { ++launches; return hipSuccess; }
bool gemm_i8_few_takes(int64_t M, int64_t) { return M <= 32; }
bool gemm_i8_few_fused(int64_t M, int64_t) { return M <= 4; }
hipError_t launch_gemm_i8_few(const I8Arg &, const void *, int64_t, int, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_embed(int, int, const void *, int64_t, int64_t, int64_t, const void *, bool, int64_t, float, void *, int64_t, hipStream_t) { ++launches; return hipSuccess; }
size_t embed_grad_workspace(int64_t N, int64_t, int64_t) { return (size_t)N; }
hipError_t launch_embed_grad(int, int, const void *, int64_t, const void *, bool, int64_t, int64_t, int64_t, float, int64_t, bool, void *, int64_t, void *, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_adamw(const AdamwTensor *t, int count, int, int, bool, bool, const AdamwRates &, uint64_t, hipStream_t)
{
    ++launches;
    for (int k = 0; k < count; ++k) tensors_seen += t[k].n > 0;          // (reads every entry)
    return hipSuccess;
}
}  // namespace nm

static void expect(const char *what, int rc, int want)
{
    if (rc != want) { printf("%s: %d, not %d\n", what, rc, want); ++errors; }
}

int main()
{
    void *const P = (void *)0x100000, *const Q = (void *)0x10000000000, *const R = (void *)0x20000000000, *const S = (void *)0x30000000000, *const W = (void *)0x40000000000;
    const int64_t sizes[] = {-1, 0, 1, 7, 131072, 131073, (int64_t)1 << 21, (int64_t)1 << 30, (int64_t)1 << 31, (int64_t)1 << 40, (int64_t)1 << 58, INT64_MAX};
    long calls = 0;
    for (int64_t a : sizes)
        for (int64_t b : sizes)
            for (int64_t ld : sizes)
                for (int dt = 0; dt < 3; ++dt) {
                    nm_quant_i8(P, a, b, ld, dt, (int8_t *)Q, (ld + (ld < INT64_MAX - 16 ? 15 : 0)) / 16 * 16, (float *)R, nullptr);
                    nm_quant_i8_t(P, a, b, ld, dt, (int8_t *)Q, ld / 16 * 16, (float *)R, W, SIZE_MAX / 2, nullptr);
                    nm_gemm_i8((int8_t *)P, ld / 16 * 16, (float *)Q, (int8_t *)R, ld / 16 * 16, (float *)S, nullptr, 0, a, b, ld, 0, W, ld, dt, nullptr);
                    nm_linear_i8(P, ld, dt, (int8_t *)R, ld / 16 * 16, (float *)S, Q, dt, a, b, ld, 0, W, b, dt, (void *)0x50000000000, SIZE_MAX / 2, nullptr);
                    nm_embed(P, a, b, ld, dt, Q, dt ? 64 : 32, ld, 1.f, R, b, dt, nullptr);
                    nm_embed_grad(P, ld, dt, Q, 64, a, b, ld, 1.f, -1, dt, R, ld, dt, W, SIZE_MAX / 2, nullptr);
                    nm_linear_i8_workspace(a, b); nm_quant_i8_t_workspace(a, b); nm_embed_grad_workspace(a, b, ld);
                    calls += 6;
                }
    // arrays at the end of the address space
    expect("quant at the end", nm_quant_i8((void *)(UINTPTR_MAX - 63), 4, 8, 8, 0, (int8_t *)P, 16, (float *)Q, nullptr), NM_OK);
    // tables: more tensors than a launch holds, empty ones among them, the last one empty
    for (int count : {1, 47, 48, 49, 96, 200}) {
        std::vector<nm_adamw_tensor> t(count);
        int full = 0;
        for (int k = 0; k < count; ++k) {
            const uintptr_t at = 0x1000000 + (uintptr_t)k * 0x100000;
            t[k] = nm_adamw_tensor{(void *)at, (void *)(at + 0x10000), (void *)(at + 0x20000), (void *)(at + 0x30000), (float *)(at + 0x40000), (float *)(at + 0x50000), nullptr, k % 5 == 4 || k == count - 1 ? 0 : 100, (uint32_t)k};
            full += t[k].n > 0;
        }
        tensors_seen = launches = 0;
        expect("table", nm_adamw(t.data(), count, 0, 0, 1, 1e-3, 0.9, 0.999, 1e-8, 0.01, 3, 1.f, nullptr, 7, nullptr), NM_OK);
        if (tensors_seen != full || launches != (full + nm::ADAMW_MOST - 1) / nm::ADAMW_MOST) { printf("table of %d: %d tensors in %d launches\n", count, tensors_seen, launches); ++errors; }
    }
    if (errors) return 1;
    printf("step sanitizer driver ok: %ld calls\n", calls);
    return 0;
}
