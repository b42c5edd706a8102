// Host side of csrc/nm_block.hip under AddressSanitizer and UndefinedBehaviorSanitizer: which outputs count as overlapping.  Parts of one tensor in every order of its dimensions are
// taken, shifted ones and ones of other strides only where no byte is in two of them, which a set of all bytes decides.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <set>

#include "../include/nm_mvue.h"
#include "../paper_2203_10991_amd/csrc/nm_internal.h"

static long errors = 0;

namespace nm {
int abi_fail(int code, const char *) { return code; }
void abi_clear() {}
hipError_t launch_layer_norm(const NormArg &, hipStream_t) { return hipSuccess; }
size_t layer_norm_grad_workspace(int64_t R, int64_t C) { return (size_t)R * C * 8; }
hipError_t launch_layer_norm_grad(const NormGradArg &, hipStream_t) { return hipSuccess; }
hipError_t launch_rotary(const RotaryArg &, hipStream_t) { return hipSuccess; }
size_t attention_workspace(const AttnArg &) { return 0; }
size_t attention_grad_workspace(const AttnArg &) { return 0; }
hipError_t launch_attention(AttnArg, void *, hipStream_t) { return hipSuccess; }
hipError_t launch_attention_grad(AttnArg, void *, hipStream_t) { return hipSuccess; }
}  // namespace nm

static uint64_t state = 1;
static int64_t below(int64_t n) { state = state * 6364136223846793005ull + 1442695040888963407ull; return (int64_t)((state >> 33) % (uint64_t)n); }

static void expect(const char *what, bool ok) { if (!ok && ++errors < 20) printf("%s\n", what); }

// 16-byte units of a tensor of heads; false: one is there twice
static bool add(std::set<uintptr_t> &all, const nm_heads &t, int64_t B, int64_t T, int64_t H, int64_t D, int64_t e)
{
    bool once = true;
    for (int64_t b = 0; b < B; ++b)
        for (int64_t i = 0; i < T; ++i)
            for (int64_t h = 0; h < H; ++h)
                for (int64_t x = 0; x < D * e; x += 16) once &= all.insert((uintptr_t)t.data + (uintptr_t)((b * t.batch + i * t.token + h * t.head) * e + x)).second;
    return once;
}

int main()
{
    char *const far = (char *)0x1000000000000, *const out = (char *)0x2000000000000;
    const nm_heads in{far, 1 << 20, 1 << 12, 1 << 7};
    float *const lse = (float *)0x3000000000000;
    long taken = 0, refused = 0, careful = 0;
    auto grad = [&](const nm_heads &dq, const nm_heads &dk, const nm_heads &dv, int64_t B, int64_t T, int64_t H, int64_t K, int64_t D, int dt) {
        return nm_attention_grad(&in, &in, &in, &in, &in, lse, nullptr, B, T, T, H, K, D, dt, 0, 1.f, nullptr, nullptr, &dq, &dk, &dv, nullptr, 0, nullptr);
    };
    // a tensor of H + 2 K heads with its dimensions in every order, and room behind a head's elements
    for (int turn = 0; turn < 20000; ++turn) {
        const int64_t K = 1 + below(3), H = K * (1 + below(3)), B = 1 + below(3), T = 1 + below(4), D = 8 * (1 + below(3)), room = 8 * below(2);
        const int dt = (int)below(2);
        const int64_t e = dt == NM_BF16 ? 2 : 4, all = H + 2 * K, n[3] = {B, T, all};
        int order[3] = {0, 1, 2};
        for (int i = 2; i > 0; --i) std::swap(order[i], order[below(i + 1)]);
        int64_t s[3], step = D + room;
        for (int d : order) { s[d] = step; step *= n[d]; step += 8 * below(2); }
        const nm_heads dq{out, s[0], s[1], s[2]}, dk{out + H * s[2] * e, s[0], s[1], s[2]}, dv{out + (H + K) * s[2] * e, s[0], s[1], s[2]};
        expect("parts side by side", grad(dq, dk, dv, B, T, H, K, D, dt) == NM_OK);
        expect("the same part twice", grad(dq, dk, dk, B, T, H, K, D, dt) == NM_ERR_ALIAS);
        // dv moved by some bytes, and with steps of its own now and then
        nm_heads dv2{(char *)dv.data + 16 * (below(2 * step * e / 16) - step * e / 16), s[0], s[1], s[2]};
        if (below(4) == 0) dv2.token += 8 * below(5);
        if (below(4) == 0) dv2.batch += 8 * below(40);
        std::set<uintptr_t> bytes;
        add(bytes, dq, B, T, H, D, e);
        add(bytes, dk, B, T, K, D, e);
        std::set<uintptr_t> own;
        const bool itself = add(own, dv2, B, T, K, D, e), apart = add(bytes, dv2, B, T, K, D, e);
        const int rc = grad(dq, dk, dv2, B, T, H, K, D, dt);
        if (rc == NM_OK) { ++taken; expect("taken, though bytes are in two outputs", apart && itself); }
        else if (apart && itself) ++careful;
        else ++refused;
    }
    // matrices that are columns of one
    for (int turn = 0; turn < 2000; ++turn) {
        const int64_t R = 1 + below(4), C = 1 + below(20), ld = 2 * C + below(4), off = below(2 * ld);
        std::set<int64_t> x;
        bool apart = true;
        for (int64_t r = 0; r < R; ++r)
            for (int64_t c = 0; c < C; ++c) x.insert(r * ld + c);
        for (int64_t r = 0; r < R; ++r)
            for (int64_t c = 0; c < C; ++c) apart &= !x.count(off + r * ld + c);
        const int rc = nm_layer_norm(far, ld, NM_F32, nullptr, nullptr, NM_F32, R, C, 1e-5f, far + 4 * off, ld, nullptr, nullptr, nullptr);
        expect("columns", rc == NM_OK ? apart : rc == NM_ERR_ALIAS);
        if (off >= C && off + C <= ld) expect("columns side by side", rc == NM_OK);
    }
    // turned heads beside those that they come from, sequence first
    const nm_heads x{far, 96, 96 * 5, 16}, y{far + 3 * 16 * 2, 96, 96 * 5, 16}, z{far + 3 * 16 * 2 - 2, 96, 96 * 5, 16};
    double *const freqs = (double *)lse;
    expect("turned beside", nm_rotary(&x, &y, NM_BF16, 5, 7, 3, 16, 16, freqs, nullptr, 32, 0, 0, 1.f, 0, nullptr) == NM_OK);
    expect("turned, shifted", nm_rotary(&x, &z, NM_BF16, 5, 7, 3, 16, 16, freqs, nullptr, 32, 0, 0, 1.f, 0, nullptr) == NM_ERR_ALIAS);
    expect("turned in place", nm_rotary(&x, &x, NM_BF16, 5, 7, 3, 16, 16, freqs, nullptr, 32, 0, 0, 1.f, 0, nullptr) == NM_OK);
    if (errors) return 1;
    printf("block parts driver ok: %ld taken, %ld refused, %ld refused though apart\n", taken, refused, careful);
    return 0;
}
