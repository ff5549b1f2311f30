// Host side of the C ABI declared in include/sphattn_layer.h: argument checks, choice of launches on the caller's
// stream.  Allocates nothing and never synchronises.
#include "sphattn_heads.hpp"
#include "sphattn_host.hpp"
#include "../../include/sphattn_layer.h"

#include <climits>
#include <cmath>

namespace {

using namespace sphattn;

// ---- norms and rotation of heads -------------------------------------------------------------------------

// Elements from a view's first to behind its last; 0 where there are none, -1 where that is no number
long long extent(const sphattn_heads& v, int B, int N, int H, int d)
{
    if (B == 0 || N == 0 || H == 0) return 0;
    __int128 last = (__int128)(B - 1) * v.batch + (__int128)(N - 1) * v.token + (__int128)(H - 1) * v.head + d;
    return last < (__int128)1 << 59 ? (long long)last : -1;
}

// Whether every row has a place of its own: each stride reaches over all that the smaller ones cover
bool rows_apart(const sphattn_heads& v, int B, int N, int H, int d)
{
    long long stride[3] = {v.batch, v.token, v.head};
    int size[3] = {B, N, H};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (stride[j] < stride[i]) std::swap(stride[i], stride[j]), std::swap(size[i], size[j]);
    __int128 covered = d;
    for (int i = 0; i < 3; ++i) {
        if (size[i] <= 1) continue;
        if (stride[i] < covered) return false;
        covered += (__int128)(size[i] - 1) * stride[i];
    }
    return true;
}

int view_check(const sphattn_heads* v, int B, int N, int H, int d, size_t e, bool written, Range& range)
{
    range = Range{nullptr, 0};
    if (H == 0 || !v) return SPHATTN_OK;
    if (v->batch < 0 || v->token < 0 || v->head < 0) return SPHATTN_ERR_SHAPE;
    const long long n = extent(*v, B, N, H, d);
    if (n < 0) return SPHATTN_ERR_SHAPE;
    if (n > 0 && !v->data) return SPHATTN_ERR_NULL;
    if (off(v->data, e)) return SPHATTN_ERR_ALIGN;
    if (written && !rows_apart(*v, B, N, H, d)) return SPHATTN_ERR_ALIAS;
    range = Range{v->data, (size_t)n * e};
    return SPHATTN_OK;
}

struct HeadsCall {
    HeadsArgs a{};
    size_t e;
    Range pos{nullptr, 0}, freq{nullptr, 0}, w[2], x[2];
};

HeadRows rows_of(const sphattn_heads* v, size_t e)
{
    if (!v || !v->data) return HeadRows{};
    return HeadRows{(unsigned char*)v->data, v->batch * (long long)e, v->token * (long long)e, v->head * (long long)e};
}

int heads_check(HeadsCall& c, const sphattn_heads* Xq, const sphattn_heads* Xk, const void* wq, const void* wk, const sphattn_rotary* rotary,
                int B, int N, int Hq, int Hk, int d, int norm, float eps, int dtype)
{
    if (B < 0 || N < 0 || (long long)B * N > INT_MAX || Hq < 1 || Hk < 0 || (long long)Hq + Hk > 65536) return SPHATTN_ERR_SHAPE;
    if (d != 64 && d != 128) return SPHATTN_ERR_HEAD_DIM;
    c.e = (size_t)element_bytes(dtype);
    if (!c.e) return SPHATTN_ERR_DTYPE;
    if (norm != 0 && norm != 1) return SPHATTN_ERR_VALUE;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return SPHATTN_ERR_VALUE;
    if (!Xq || (Hk > 0 && !Xk)) return SPHATTN_ERR_NULL;
    int rc = view_check(Xq, B, N, Hq, d, c.e, false, c.x[0]);
    if (rc == SPHATTN_OK) rc = view_check(Xk, B, N, Hk, d, c.e, false, c.x[1]);
    if (rc != SPHATTN_OK) return rc;
    if (off(wq, c.e) || off(wk, c.e)) return SPHATTN_ERR_ALIGN;
    c.w[0] = Range{wq, wq ? (size_t)d * c.e : 0};
    c.w[1] = Range{wk, wk ? (size_t)d * c.e : 0};
    HeadsArgs& a = c.a;
    a.B = B, a.N = N, a.norm = norm, a.eps = eps, a.id_bytes = 4;
    a.side[0].x = rows_of(Xq, c.e), a.side[0].w = wq, a.side[0].heads = Hq;
    a.side[1].x = Hk ? rows_of(Xk, c.e) : HeadRows{}, a.side[1].w = Hk ? wk : nullptr, a.side[1].heads = Hk;
    if (!rotary || !rotary->positions) return SPHATTN_OK;
    const sphattn_rotary& r = *rotary;
    if (r.id_bytes != 4 && r.id_bytes != 8) return SPHATTN_ERR_DTYPE;
    if (r.axes < 1 || r.axes > 3 || r.axis < 0 || r.batch < 0) return SPHATTN_ERR_SHAPE;
    int all = 0;
    for (int i = 0; i < r.axes; ++i) {
        if (r.sections[i] < 0 || r.sections[i] > d / 2) return SPHATTN_ERR_SHAPE;
        all += r.sections[i];
    }
    if (all != d / 2) return SPHATTN_ERR_SHAPE;
    if (!r.inv_freq) return SPHATTN_ERR_NULL;
    if (off(r.positions, r.id_bytes) || off(r.inv_freq, 4)) return SPHATTN_ERR_ALIGN;
    if (B > 0 && N > 0) {
        const __int128 n = (__int128)(r.axes - 1) * r.axis + (__int128)(B - 1) * r.batch + N;
        if (n >= (__int128)1 << 59) return SPHATTN_ERR_SHAPE;
        c.pos = Range{r.positions, (size_t)n * r.id_bytes};
    }
    c.freq = Range{r.inv_freq, (size_t)d / 2 * 4};
    a.positions = r.positions, a.id_bytes = r.id_bytes, a.pos_axis = r.axis, a.pos_batch = r.batch;
    a.inv_freq = r.inv_freq, a.interleaved = r.interleaved != 0;
    a.until[0] = r.axes == 1 ? d / 2 : r.sections[0];
    a.until[1] = r.axes < 3 ? d / 2 : r.sections[0] + r.sections[1];
    return SPHATTN_OK;
}

// Groups of lanes per token: one takes all heads of its token, for which it forms the angles once, where tokens alone make two waves for every
// SIMD; else as many more as that takes.  (waves: 256 CUs with four SIMDs)
int heads_share(long long tokens, int heads, int d)
{
    int share = 1;
    while (share * 4 <= heads && tokens * share * (d / 8) < 64ll * 4 * kCus * 2) share *= 2;
    while (share < heads && tokens * share * (d / 8) < 64ll * kCus) share *= 2;
    return share;
}

template <Store S, bool FORWARD>
int run_heads(const HeadsArgs& a, int d, int groups, hipStream_t s)
{
#define SPH_HEADS(D, R)                                                                                                          \
    do {                                                                                                                         \
        if constexpr (FORWARD) hipLaunchKernelGGL((heads_fwd_kernel<S, D, R>), dim3((unsigned)groups), dim3(kHeadsThreads), 0, s, a); \
        else hipLaunchKernelGGL((heads_bwd_kernel<S, D, R>), dim3((unsigned)groups), dim3(kHeadsThreads), 0, s, a);              \
    } while (0)
    if (d == 128) {
        if (a.positions) SPH_HEADS(128, true);
        else SPH_HEADS(128, false);
    } else {
        if (a.positions) SPH_HEADS(64, true);
        else SPH_HEADS(64, false);
    }
#undef SPH_HEADS
    return launched();
}

long long heads_groups(const HeadsArgs& a, int d)
{
    const int per = kHeadsThreads / (d / 8);
    return ((long long)a.B * a.N * a.share + per - 1) / per;
}

}  // namespace

extern "C" {

int sphattn_head_norm_rotary_fwd(const sphattn_heads* Xq, const sphattn_heads* Xk, const void* wq, const void* wk, const sphattn_heads* Q, const sphattn_heads* K,
                                 const sphattn_rotary* rotary, int B, int N, int Hq, int Hk, int d, int norm, float eps, int dtype, void* stream)
{
    HeadsCall c;
    int rc = heads_check(c, Xq, Xk, wq, wk, rotary, B, N, Hq, Hk, d, norm, eps, dtype);
    if (rc != SPHATTN_OK) return rc;
    if (!Q || (Hk > 0 && !K)) return SPHATTN_ERR_NULL;
    Range o[2];
    rc = view_check(Q, B, N, Hq, d, c.e, true, o[0]);
    if (rc == SPHATTN_OK) rc = view_check(K, B, N, Hk, d, c.e, true, o[1]);
    if (rc != SPHATTN_OK) return rc;
    const Range read[] = {c.x[0], c.x[1], c.w[0], c.w[1], c.pos, c.freq};
    for (const Range& r : read)
        if (meet(o[0], r) || meet(o[1], r)) return SPHATTN_ERR_ALIAS;
    if (B == 0 || N == 0) return SPHATTN_OK;
    c.a.side[0].o = rows_of(Q, c.e);
    c.a.side[1].o = Hk ? rows_of(K, c.e) : HeadRows{};
    c.a.share = heads_share((long long)B * N, Hq > Hk ? Hq : Hk, d);
    const long long groups = heads_groups(c.a, d);
    const int n = (int)(groups < 1 << 22 ? groups : 1 << 22);         // (a launch has less than 2^32 threads)
    switch (dtype) {
    case SPHATTN_F32: return run_heads<Store::F32, true>(c.a, d, n, (hipStream_t)stream);
    case SPHATTN_BF16: return run_heads<Store::Bf16, true>(c.a, d, n, (hipStream_t)stream);
    default: return run_heads<Store::F16, true>(c.a, d, n, (hipStream_t)stream);
    }
}

size_t sphattn_head_norm_rotary_bwd_workspace_bytes(int d) { return d == 64 || d == 128 ? (size_t)kHeadsMostGroups * 2 * d * 4 : 0; }

int sphattn_head_norm_rotary_bwd(const sphattn_heads* Xq, const sphattn_heads* Xk, const void* wq, const void* wk, const sphattn_heads* dQ, const sphattn_heads* dK,
                                 const sphattn_heads* dXq, const sphattn_heads* dXk, void* dwq, void* dwk, const sphattn_rotary* rotary,
                                 int B, int N, int Hq, int Hk, int d, int norm, float eps, int dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    HeadsCall c;
    int rc = heads_check(c, Xq, Xk, wq, wk, rotary, B, N, Hq, Hk, d, norm, eps, dtype);
    if (rc != SPHATTN_OK) return rc;
    if (!dQ || (Hk > 0 && !dK) || (!dXq && !dXk && !dwq && !dwk)) return SPHATTN_ERR_NULL;
    Range g[2], dx[2];
    rc = view_check(dQ, B, N, Hq, d, c.e, false, g[0]);
    if (rc == SPHATTN_OK) rc = view_check(dK, B, N, Hk, d, c.e, false, g[1]);
    if (rc == SPHATTN_OK) rc = view_check(dXq, B, N, Hq, d, c.e, true, dx[0]);
    if (rc == SPHATTN_OK) rc = view_check(dXk, B, N, Hk, d, c.e, true, dx[1]);
    if (rc != SPHATTN_OK) return rc;
    if (off(dwq, c.e) || off(dwk, c.e)) return SPHATTN_ERR_ALIGN;
    const bool sums = dwq || dwk;
    const size_t need = sums ? sphattn_head_norm_rotary_bwd_workspace_bytes(d) : 0;
    if (sums && (!workspace || off(workspace, 16) || workspace_bytes < need)) return SPHATTN_ERR_WORKSPACE;
    const Range written[] = {{dwq, dwq ? (size_t)d * c.e : 0}, {dwk, dwk ? (size_t)d * c.e : 0}, {workspace, need}};
    const Range read[] = {c.x[0], c.x[1], c.w[0], c.w[1], c.pos, c.freq, g[0], g[1]};
    if (any_meet(written, read)) return SPHATTN_ERR_ALIAS;
    for (const Range& d2 : dx) {
        for (const Range& r : read)
            if (meet(d2, r)) return SPHATTN_ERR_ALIAS;
        for (const Range& r : written)
            if (meet(d2, r)) return SPHATTN_ERR_ALIAS;
    }
    const hipStream_t s = (hipStream_t)stream;
    HeadsArgs& a = c.a;
    a.side[0].o = rows_of(dQ, c.e), a.side[0].dx = rows_of(dXq, c.e);
    a.side[1].o = Hk ? rows_of(dK, c.e) : HeadRows{}, a.side[1].dx = Hk ? rows_of(dXk, c.e) : HeadRows{};
    a.share = heads_share((long long)B * N, Hq > Hk ? Hq : Hk, d);
    a.partial = sums ? (float*)workspace : nullptr;
    const long long groups = heads_groups(a, d);
    const int n = (int)(groups < kHeadsMostGroups ? groups : kHeadsMostGroups);
    if (n > 0) {
        switch (dtype) {
        case SPHATTN_F32: rc = run_heads<Store::F32, false>(a, d, n, s); break;
        case SPHATTN_BF16: rc = run_heads<Store::Bf16, false>(a, d, n, s); break;
        default: rc = run_heads<Store::F16, false>(a, d, n, s);
        }
        if (rc != SPHATTN_OK) return rc;
    }
    if (sums) {
        const dim3 grid((unsigned)(2 * d / 16));
        switch (dtype) {
        case SPHATTN_F32: hipLaunchKernelGGL((heads_dw_kernel<Store::F32>), grid, dim3(1024), 0, s, a.partial, n, d, dwq, dwk); break;
        case SPHATTN_BF16: hipLaunchKernelGGL((heads_dw_kernel<Store::Bf16>), grid, dim3(1024), 0, s, a.partial, n, d, dwq, dwk); break;
        default: hipLaunchKernelGGL((heads_dw_kernel<Store::F16>), grid, dim3(1024), 0, s, a.partial, n, d, dwq, dwk);
        }
    }
    return launched();
}

}  // extern "C"
