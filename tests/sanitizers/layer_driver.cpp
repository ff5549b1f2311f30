// Sanitizer driver for the host half of include/sphattn_layer.h and of the distillation in include/sphattn_train.h (argument checks, plans, workspace
// arithmetic).  Built by tests/test_sanitizers_layer.py with the HOST code under -fsanitize=address,undefined.  Every call returns before any launch:
// addresses are made up and never followed, and each call is refused or is arithmetic only.
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/sphattn_layer.h"
#include "../../include/sphattn_train.h"

static int failures = 0;
#define EXPECT(call, want) do { const long long got_ = (long long)(call); if (got_ != (long long)(want)) { \
    fprintf(stderr, "%s:%d: %s = %lld, expected %lld\n", __FILE__, __LINE__, #call, got_, (long long)(want)); ++failures; } } while (0)
#define HOLDS(what) do { if (!(what)) { fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #what); ++failures; } } while (0)

static void* P(uintptr_t a) { return (void*)a; }

int main()
{
    void *X = P(0x10000000), *W = P(0x20000000), *Y = P(0x30000000), *ws = P(0x700000000000);
    float *f = (float*)P(0x40000000), *h = (float*)P(0x41000000), *kept = (float*)P(0x10000000000), *m = (float*)P(0x42000000);
    const int dtypes[] = {SPHATTN_F32, SPHATTN_BF16, SPHATTN_F16};
    // feed-forward: plans over the whole range of sizes, one byte of workspace too few at the end
    const int Ts[] = {0, 1, 16, 17, 64, 65, 129, 1023, 8192, 1 << 20}, Ds[] = {1, 8, 515, 4096, 65536}, Fs[] = {1, 127, 1371, 8192, 65536, 1 << 18};
    for (int dtype : dtypes)
        for (int T : Ts)
            for (int D : Ds)
                for (int F : Fs) {
                    const size_t fwd = sphattn_gated_ffn_workspace_bytes(T, D, F, dtype), bwd = sphattn_gated_ffn_bwd_workspace_bytes(T, D, F, dtype);
                    if ((long long)T * F > 1ll << 36) {
                        EXPECT(fwd, 0);
                        EXPECT(bwd, 0);
                        continue;
                    }
                    HOLDS((T <= 32 || (T <= 64 && (dtype == SPHATTN_F32 || (long long)F * D < 1 << 24))) == (fwd == 0) && bwd >= (size_t)T * F * 4 + (size_t)F * D * 4);
                    if (fwd) EXPECT(sphattn_gated_ffn_fwd(X, W, Y, kept, T, D, F, SPHATTN_GATE_SILU, dtype, ws, fwd - 1, nullptr), SPHATTN_ERR_WORKSPACE);
                    EXPECT(sphattn_gated_ffn_bwd(X, W, Y, kept, P(0x20000000000), nullptr, P(0x30000000000), T, D, F, SPHATTN_GATE_RELU, dtype, ws, bwd - 1, nullptr),
                           SPHATTN_ERR_WORKSPACE);
                }
    EXPECT(sphattn_gated_ffn_workspace_bytes(INT_MAX, INT_MAX, INT_MAX, SPHATTN_F32), 0);
    EXPECT(sphattn_gated_ffn_bwd_workspace_bytes(INT_MIN, INT_MIN, INT_MIN, 77), 0);
    EXPECT(sphattn_gated_ffn_fwd(X, W, Y, X, 5, 5, 5, INT_MAX, SPHATTN_BF16, ws, SIZE_MAX, nullptr), SPHATTN_ERR_VALUE);
    EXPECT(sphattn_gated_ffn_fwd(X, W, Y, P(UINTPTR_MAX - 15), 1 << 20, 65536, 65536, 0, SPHATTN_F32, P(UINTPTR_MAX - 31), SIZE_MAX, nullptr), SPHATTN_ERR_ALIAS);

    // distillation
    const int Vs[] = {1, 127, 50003, 1 << 20, 1 << 24}, Ks[] = {1, 2, 3, 64, 1000, 1024};
    for (int dtype : dtypes)
        for (int T : Ts)
            for (int V : Vs)
                for (int K : Ks)
                    for (int D : {8, 515, 65536}) {
                        const size_t fwd = sphattn_vocab_distill_workspace_bytes(T, V, D, K, dtype), bwd = sphattn_vocab_distill_bwd_workspace_bytes(T, V, D, K, dtype);
                        HOLDS(fwd > sphattn_vocab_loss_workspace_bytes(T, V, D, dtype) - 1 + (size_t)T * K * 12);
                        HOLDS(bwd > sphattn_vocab_loss_bwd_workspace_bytes(T, V, D, dtype) - 1 + (size_t)T * K * 8);
                        // (where blocks of ids begin takes no more than 256 MB)
                        HOLDS(fwd < sphattn_vocab_loss_workspace_bytes(T, V, D, dtype) + (size_t)T * K * 12 + (260ull << 20) + (size_t)T * 4 + 4096);
                        EXPECT(sphattn_vocab_distill_fwd(X, W, Y, 8, kept, f, h, nullptr, m, T, V, D, K, 1.f, 1.f, SPHATTN_LOSS_MEAN, dtype, ws, fwd - 1, nullptr),
                               SPHATTN_ERR_WORKSPACE);
                        EXPECT(sphattn_vocab_distill_bwd(X, W, Y, 8, kept, f, kept, h, P(0x20000000000), nullptr, T, V, D, K, 1.f, 1.f, SPHATTN_LOSS_MEAN, dtype, ws,
                                                         bwd - 1, nullptr), SPHATTN_ERR_WORKSPACE);
                    }
    EXPECT(sphattn_vocab_distill_workspace_bytes(INT_MAX, INT_MAX, INT_MAX, INT_MAX, SPHATTN_F32), 0);
    EXPECT(sphattn_vocab_distill_bwd_workspace_bytes(INT_MIN, INT_MIN, INT_MIN, INT_MIN, 77), 0);
    EXPECT(sphattn_vocab_distill_fwd(X, W, Y, 8, kept, f, h, nullptr, m, 5, 5, 5, 5, NAN, 1.f, 0, SPHATTN_BF16, ws, SIZE_MAX, nullptr), SPHATTN_ERR_VALUE);
    EXPECT(sphattn_vocab_distill_fwd(X, W, Y, 8, kept, f, h, nullptr, m, 5, 5, 5, 5, 1.f, NAN, 0, SPHATTN_BF16, ws, SIZE_MAX, nullptr), SPHATTN_ERR_VALUE);
    EXPECT(sphattn_vocab_distill_fwd(X, W, Y, 8, kept, f, h, f + 1, m, 1 << 20, 5, 5, 1024, 1.f, 1.f, 0, SPHATTN_BF16, ws, SIZE_MAX, nullptr), SPHATTN_ERR_ALIAS);

    // heads: strides of every size
    const long long strides[] = {0, 1, 63, 64, 128, 1 << 20, 1ll << 40, LLONG_MAX, -1, LLONG_MIN};
    for (long long a : strides)
        for (long long b : strides)
            for (long long c : strides) {
                const sphattn_heads x{X, a, b, c}, o{Y, 1ll << 30, 64, 1ll << 20};
                const bool bad = a < 0 || b < 0 || c < 0;
                // (every call is refused: either its strides are, or the output's data is none)
                const sphattn_heads none{nullptr, 1ll << 30, 64, 1ll << 20};
                const int rc = sphattn_head_norm_rotary_fwd(&x, nullptr, nullptr, nullptr, &none, nullptr, nullptr, 3, 5, 7, 0, 64, 1, 0.f, SPHATTN_F32, nullptr);
                HOLDS(rc == SPHATTN_ERR_NULL || rc == SPHATTN_ERR_SHAPE);
                if (bad) EXPECT(rc, SPHATTN_ERR_SHAPE);
                const sphattn_heads out{P(0x10000001), a, b, c};
                const int rc2 = sphattn_head_norm_rotary_fwd(&o, nullptr, nullptr, nullptr, &out, nullptr, nullptr, 3, 5, 7, 0, 64, 1, 0.f, SPHATTN_BF16, nullptr);
                HOLDS(rc2 == SPHATTN_ERR_ALIGN || rc2 == SPHATTN_ERR_SHAPE);
                // positions with such strides
                const sphattn_rotary r{Y, 8, a, b, f, 3, {16, 8, 8}, 1};
                const int rc3 = sphattn_head_norm_rotary_fwd(&o, nullptr, nullptr, nullptr, &none, nullptr, &r, 3, 5, 7, 0, 64, 1, 0.f, SPHATTN_BF16, nullptr);
                HOLDS(rc3 == SPHATTN_ERR_NULL || rc3 == SPHATTN_ERR_SHAPE);
            }
    const sphattn_heads o{Y, 1ll << 30, 64, 1ll << 20};
    const sphattn_rotary sections{Y, 8, 0, 0, f, 3, {INT_MAX, INT_MAX, 34}, 0};
    EXPECT(sphattn_head_norm_rotary_fwd(&o, nullptr, nullptr, nullptr, &o, nullptr, &sections, 3, 5, 7, 0, 64, 1, 0.f, SPHATTN_BF16, nullptr), SPHATTN_ERR_SHAPE);
    EXPECT(sphattn_head_norm_rotary_fwd(&o, &o, nullptr, nullptr, &o, &o, nullptr, 3, 5, INT_MAX, INT_MAX, 64, 1, 0.f, SPHATTN_BF16, nullptr), SPHATTN_ERR_SHAPE);
    EXPECT(sphattn_head_norm_rotary_fwd(&o, &o, nullptr, nullptr, &o, &o, nullptr, INT_MAX, INT_MAX, 1, 1, 64, 1, 0.f, SPHATTN_BF16, nullptr), SPHATTN_ERR_SHAPE);
    EXPECT(sphattn_head_norm_rotary_bwd_workspace_bytes(INT_MIN), 0);
    if (failures == 0) printf("ok\n");
    return failures != 0;
}
