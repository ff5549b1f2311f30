// Sanitizer driver for the host half of include/sphattn_train.h (argument checks, plans, workspace arithmetic).  Built by
// tests/test_sanitizers_train.py from paper_2505_09326_amd/csrc/sphattn_train.hip with the HOST code under -fsanitize=address,undefined.  Every
// call returns before any launch: addresses are made up and never followed, and each call is refused or is arithmetic only.
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/sphattn_train.h"

static int failures = 0;
#define EXPECT(call, want) do { const long long got_ = (long long)(call); if (got_ != (long long)(want)) { \
    fprintf(stderr, "%s:%d: %s = %lld, expected %lld\n", __FILE__, __LINE__, #call, got_, (long long)(want)); ++failures; } } while (0)
#define HOLDS(what) do { if (!(what)) { fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #what); ++failures; } } while (0)

static void* P(uintptr_t a) { return (void*)a; }

int main()
{
    void *X = P(0x10000000), *W = P(0x20000000), *Y = P(0x30000000), *ws = P(0x7000000000);
    float *f = (float*)P(0x40000000), *h = (float*)P(0x41000000), *m = (float*)P(0x42000000);
    const int dtypes[] = {SPHATTN_F32, SPHATTN_BF16, SPHATTN_F16};
    // plans over the whole range of sizes: every number that an int or a size_t holds on the way, one byte of workspace too few at the end
    const int Ts[] = {0, 1, 16, 17, 32, 33, 64, 65, 1023, 1025, 8192, 1 << 20}, Vs[] = {1, 127, 129, 50003, 1 << 20, 1 << 24}, Ds[] = {1, 8, 515, 4096, 65536};
    for (int dtype : dtypes)
        for (int T : Ts)
            for (int V : Vs)
                for (int D : Ds) {
                    const size_t fwd = sphattn_vocab_loss_workspace_bytes(T, V, D, dtype), bwd = sphattn_vocab_loss_bwd_workspace_bytes(T, V, D, dtype);
                    HOLDS(fwd > (size_t)V * D * 2 && bwd > (size_t)T * D * 4);
                    EXPECT(sphattn_vocab_loss_fwd(X, W, Y, 8, f, h, m, T, V, D, 1.f, SPHATTN_LOSS_MEAN, 1, dtype, ws, fwd - 1, nullptr), SPHATTN_ERR_WORKSPACE);
                    EXPECT(sphattn_vocab_loss_bwd(X, W, Y, 8, f, h, P(0x100000000), P(0x5000000000), T, V, D, 1.f, SPHATTN_LOSS_MEAN, dtype, ws, bwd - 1, nullptr),
                           SPHATTN_ERR_WORKSPACE);
                }
    for (int T : {0, 1, 1000, INT_MAX})
        for (int V : {1, 131073, 1 << 30})
            for (int D : Ds) {
                const size_t need = sphattn_embed_bwd_workspace_bytes(T, V, D);
                HOLDS(need > (size_t)V * 4 + (size_t)T * 4);
                EXPECT(sphattn_embed_bwd(Y, 4, nullptr, X, W, T, V, D, 1.f, SPHATTN_F32, ws, need - 1, nullptr), SPHATTN_ERR_WORKSPACE);
            }
    EXPECT(sphattn_vocab_loss_workspace_bytes(INT_MAX, INT_MAX, INT_MAX, SPHATTN_F32), 0);
    EXPECT(sphattn_vocab_loss_bwd_workspace_bytes(INT_MIN, INT_MIN, INT_MIN, 77), 0);
    EXPECT(sphattn_embed_bwd_workspace_bytes(INT_MIN, INT_MAX, INT_MAX), 0);
    // refusals, the last with ranges that end at the top of the address space
    EXPECT(sphattn_vocab_loss_fwd(X, W, Y, 8, f, h, m, 5, 5, 5, NAN, 0, 1, SPHATTN_BF16, ws, SIZE_MAX, nullptr), SPHATTN_ERR_VALUE);
    EXPECT(sphattn_vocab_loss_fwd(X, W, Y, 8, f, h, m, 5, 5, 5, 1.f, INT_MAX, 1, SPHATTN_BF16, ws, SIZE_MAX, nullptr), SPHATTN_ERR_VALUE);
    EXPECT(sphattn_vocab_loss_fwd(X, W, Y, INT_MIN, f, h, m, 5, 5, 5, 1.f, 0, 1, SPHATTN_BF16, ws, SIZE_MAX, nullptr), SPHATTN_ERR_DTYPE);
    EXPECT(sphattn_vocab_loss_bwd(X, W, Y, 8, f, h, X, nullptr, 5, 5, 5, 1.f, 0, SPHATTN_BF16, ws, SIZE_MAX, nullptr), SPHATTN_ERR_ALIAS);
    EXPECT(sphattn_vocab_loss_bwd(X, W, Y, 8, f, h, P(UINTPTR_MAX - 15), P(UINTPTR_MAX - 15), 1 << 20, 1 << 24, 65536, 1.f, 0, SPHATTN_F16, ws, SIZE_MAX, nullptr),
           SPHATTN_ERR_ALIAS);
    EXPECT(sphattn_embed_fwd(Y, 8, W, nullptr, P(UINTPTR_MAX - 15), INT_MAX, 1 << 30, 65536, 1.f, 9, nullptr), SPHATTN_ERR_DTYPE);
    EXPECT(sphattn_embed_fwd(Y, 8, W, nullptr, W, INT_MAX, 1 << 30, 65536, 1.f, SPHATTN_F32, nullptr), SPHATTN_ERR_ALIAS);
    // clipping: lists of every length about a launch's 120, sizes up to the limit and past it
    constexpr int MOST = 500;
    static const void* in[MOST];
    static void* out[MOST];
    static long long size[MOST];
    static int type[MOST];
    for (int i = 0; i < MOST; ++i) in[i] = out[i] = P(0x100000000ull * (i + 0x1000)), size[i] = i % 7 ? 1000 * i : 0, type[i] = dtypes[i % 3];
    for (int n : {0, 1, 119, 120, 121, 240, 241, MOST}) {
        const size_t need = sphattn_clip_grads_workspace_bytes(n);
        HOLDS(need >= (size_t)8);
        EXPECT(sphattn_clip_grads(in, out, size, type, n, 1.f, f, ws, need - 1, nullptr), SPHATTN_ERR_WORKSPACE);
    }
    EXPECT(sphattn_clip_grads_workspace_bytes(INT_MIN), 0);
    HOLDS(sphattn_clip_grads_workspace_bytes(INT_MAX) > (size_t)INT_MAX);
    size[3] = LLONG_MAX;
    EXPECT(sphattn_clip_grads(in, out, size, type, MOST, 1.f, f, ws, sphattn_clip_grads_workspace_bytes(MOST), nullptr), SPHATTN_ERR_SHAPE);
    size[3] = LLONG_MIN;
    EXPECT(sphattn_clip_grads(in, out, size, type, MOST, 1.f, f, ws, sphattn_clip_grads_workspace_bytes(MOST), nullptr), SPHATTN_ERR_SHAPE);
    EXPECT(sphattn_clip_grads(in, out, size, type, 2, -0.5f, f, ws, sphattn_clip_grads_workspace_bytes(MOST), nullptr), SPHATTN_ERR_VALUE);
    if (failures == 0) printf("ok\n");
    return failures != 0;
}
