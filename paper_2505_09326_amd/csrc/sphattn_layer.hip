// Host side of the C ABI declared in include/sphattn_layer.h: argument checks, choice of launches on the caller's
// stream.  Allocates nothing and never synchronises.
#include "sphattn_ffn.hpp"
#include "sphattn_heads.hpp"
#include "sphattn_tile_choice.hpp"
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
int heads_log_share(long long tokens, int heads, int d)
{
    int log = 0;
    while (4 << log <= heads && (tokens << log) * (d / 8) < 64ll * 4 * kCus * 2) ++log;
    while (1 << log < heads && (tokens << log) * (d / 8) < 64ll * kCus) ++log;
    return log;
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
    return (((long long)a.B * a.N << a.log_share) + per - 1) / per;
}

// ---- gated feed-forward ------------------------------------------------------------------------------------

constexpr long long kFfnFew = 1 << 18;             // values of dA up to which they are kept in two parts
// Whether forward reads the weights straight into registers: up to 32 rows, and up to 64 where the tiles' way is longer, in fp32 (parts) and for small weights.  (17 and 32 rows in bf16:
// 1024 x 4096 5.8 and 6.1 us, in tiles 11.3 and 11.4; 2048 x 8192 15.5 and 18.4, 21.3 and 21.5; 4096 x 12000 40.2 and 48.1, 39.9 and 44.3, the one where tiles win; in fp32 2048 x 8192
// 43.7 and 46.5, in tiles 120.  33 and
// 64 rows in bf16: 1024 x 4096 6.9 and 8.3 us, in tiles 11.3; 2000 x 5001 16.2 and 19.8, 19.0 and 21.4; 2048 x 8192 25.2 and 30.5, 21.3 and 22.2; 4096 x 12000 52.6 and 68.9, 45;
// 64 rows of 2048 x 8192 in fp32 74, 65 in tiles 123.)
bool ffn_rows_form(int T, int D, int F, int dtype) { return T <= 32 || (T <= 64 && (dtype == SPHATTN_F32 || (long long)F * D < 1 << 24)); }

bool ffn_shape(int T, int D, int F)
{
    return T >= 0 && T <= 1 << 20 && D >= 1 && D <= 65536 && F >= 1 && F <= 1 << 18 && (long long)T * F <= 1ll << 36;   // (a launch has less than 2^32 threads)
}

// The tile and slices of a sum over k for `count` results of rows x cols, by the time that its rounds take: in a round of 256 Big tiles each takes 27 ns
// per k, in one of 512 Mid tiles 20, and every slice is written and read again as fp32.
struct SumChoice { bool big; int slices; };
SumChoice sum_choice(long long rows, long long cols, long long k, int count, int products, bool may_big)
{
    SumChoice c{false, 1};
    double best = 0.0;
    for (int b = may_big; b >= 0; --b) {
        const int tile = b ? 256 : 128, at_once = b ? kCus : 2 * kCus;
        const long long tiles = count * ((rows + tile - 1) / tile) * ((cols + tile - 1) / tile);
        for (int s = 1; s <= 64 && (s == 1 || (k / s >= 256 && (double)s * count * rows * cols <= 2.5e8)); s *= 2) {
            const double rounds = (double)((tiles * s + at_once - 1) / at_once);
            const double us = rounds * (double)(k / s) * products * (b ? 0.027 : 0.020) + (s > 1 ? 4.0 + s * (double)(count * rows * cols) * 8.0 / 4.5e6 : 0.0);
            if (best == 0.0 || us < best) best = us, c = SumChoice{b != 0, s};
        }
    }
    return c;
}

struct Ffn {
    int T, D, F, ld, ldf, parts, g_parts;          // ld, ldf: elements per packed row of D, of F; parts: of X and W, of dA and dB
    bool two;                                      // few values of dA and dB in 16 bits: two parts
    SumChoice dx, dw;
    int *x_exp, *g_exp, *u_exp;                    // fp32
    unsigned short *x, *g, *u, *x_sum, *g_sum, *u_sum;
    unsigned short *dA, *dB, *dA_all, *dB_all;
    float *x_norm, *w_norm;                        // fp16 and relu's slopes; w_norm: Wg's rows, fp16 Wu's behind them
    // fp16: the largest of dH by row and by column in parts, factors by row and by column
    float *row_top, *col_top, *row_up, *row_down, *down_a, *down_b;
    int *col_up, top_rows, top_parts;
    float *part, *part_w;                          // slices of dX and of dW
    size_t bytes;
};

Ffn ffn_plan(int T, int D, int F, int dtype, bool back, void* workspace)
{
    Ffn p{};
    p.T = T, p.D = D, p.F = F, p.ld = (int)up_to(D, 8), p.ldf = (int)up_to(F, 8);
    p.two = back && dtype != SPHATTN_F32 && (long long)T * F <= kFfnFew;
    p.parts = dtype == SPHATTN_F32 ? 2 : 1, p.g_parts = dtype == SPHATTN_F32 ? 3 : p.two ? 2 : 1;
    if (!back && ffn_rows_form(T, D, F, dtype)) return p;
    const bool f32 = dtype == SPHATTN_F32, f16 = dtype == SPHATTN_F16;
    Carve c(workspace);
    p.x_exp = c.take<int>(f32 ? T : 0);
    p.g_exp = c.take<int>(f32 ? up_to(F, 256) : 0);
    p.u_exp = c.take<int>(f32 ? up_to(F, 256) : 0);
    // (rows that the products can read as they are need no copy, but who asks for the size knows no addresses)
    p.x = c.take<unsigned short>((size_t)p.parts * T * p.ld);
    p.g = c.take<unsigned short>((size_t)p.parts * F * p.ld);
    p.u = c.take<unsigned short>((size_t)p.parts * F * p.ld);
    if (back) {
        p.x_sum = c.take<unsigned short>(f32 ? (size_t)3 * T * p.ld : 0);
        p.g_sum = c.take<unsigned short>(f32 ? (size_t)3 * F * p.ld : 0);
        p.u_sum = c.take<unsigned short>(f32 ? (size_t)3 * F * p.ld : 0);
        const size_t n = (size_t)p.g_parts * T * p.ldf;
        p.dA = c.take<unsigned short>(n);
        p.dB = c.take<unsigned short>(n);
        p.dA_all = c.take<unsigned short>(f16 ? n : 0);
        p.dB_all = c.take<unsigned short>(f16 ? n : 0);
        p.x_norm = c.take<float>(T);
        p.w_norm = c.take<float>(up_to(f16 ? 2ll * F : F, 256));
        p.top_rows = (int)up_to((T + kTopMost - 1) / kTopMost, kTopRows);
        p.top_parts = T > 0 ? (T + p.top_rows - 1) / p.top_rows : 0;
        p.row_top = c.take<float>(f16 ? (size_t)((F + kTopCols - 1) / kTopCols) * T : 0);
        p.col_top = c.take<float>(f16 ? (size_t)p.top_parts * F : 0);
        p.row_up = c.take<float>(f16 ? T : 0);
        p.row_down = c.take<float>(f16 ? T : 0);
        p.col_up = c.take<int>(f16 ? up_to(F, 256) : 0);
        p.down_a = c.take<float>(f16 ? F : 0);
        p.down_b = c.take<float>(f16 ? F : 0);
        const int products = f32 ? 6 : p.two ? 2 : 1;
        p.dx = sum_choice(T > 0 ? T : 1, p.ld, 2ll * F, 1, products, !p.two);
        p.dw = T > 0 ? sum_choice(F, p.ld, T, 2, products, !p.two) : SumChoice{false, 1};
        p.part = c.take<float>(p.dx.slices > 1 ? (size_t)p.dx.slices * T * p.ld : 0);
        p.part_w = c.take<float>(p.dw.slices > 1 ? (size_t)p.dw.slices * 2 * F * p.ld : 0);
    }
    p.bytes = c.used();
    return p;
}

template <class T, Store S, bool BACK, bool TWO = false>
int launch_gate(FfnArgs& a, int act, hipStream_t stream)
{
    const auto kern = ffn_gate_kernel<T, S, BACK, TWO>;
    static std::atomic<uint64_t> done{0};
    if (T::LDS > 65536 && !raise_lds_limit(kern, T::LDS, done)) return SPHATTN_ERR_LAUNCH;
    a.tiles_p = (a.F + T::BP / 2 - 1) / (T::BP / 2);
    const long long tiles = (long long)a.tiles_p * ((a.T + T::BQ - 1) / T::BQ);
    if (tiles > 1 << 22) return SPHATTN_ERR_SHAPE;                    // (a launch has less than 2^32 threads)
    hipLaunchKernelGGL(kern, dim3((unsigned)tiles), dim3(T::THREADS), T::LDS, stream, a, act);
    return launched();
}

template <Store S, bool BACK>
int run_gate(FfnArgs& a, int act, hipStream_t stream)
{
    return big_tiles(2ll * a.F, a.T) ? launch_gate<Big, S, BACK>(a, act, stream) : launch_gate<Mid, S, BACK>(a, act, stream);
}

// X, Wg and Wu as the products take them (what can be read as it is stays where it is), and the norms of X's and Wg's rows, of Wu's too
template <Store S>
FfnArgs ffn_pack(const Ffn& p, const void* X, const void* Wg, const void* Wu, bool norms, bool norms_u, hipStream_t stream)
{
    FfnArgs a{};
    FfnPack k{};
    int groups = 0;
    auto take = [&](int m, const void* in, int n, unsigned short* out, unsigned short* sum_out, int* exp, float* norm) {
        Operand o{(const unsigned char*)in, 0, p.D * 2, n};
        const bool copy = !ready(in, p.D, S);
        if (copy || norm) {
            k.m[m] = PackRows{in, copy ? out : nullptr, n, p.D, p.ld, (long long)n * p.ld, sum_out, exp};
            k.norm[m] = norm;
            groups += (n + kFfnPackRows - 1) / kFfnPackRows;
        }
        if (copy) o = Operand{(const unsigned char*)out, k.m[m].part * 2, p.ld * 2, n};
        if (m < 2) k.until[m] = groups;
        return o;
    };
    a.X = take(0, X, p.T, p.x, p.x_sum, p.x_exp, norms ? p.x_norm : nullptr);
    a.G = take(1, Wg, p.F, p.g, p.g_sum, p.g_exp, norms ? p.w_norm : nullptr);
    a.U = take(2, Wu, p.F, p.u, p.u_sum, p.u_exp, norms_u ? p.w_norm + p.F : nullptr);
    if (groups) hipLaunchKernelGGL((ffn_pack_kernel<S>), dim3((unsigned)groups), dim3(kFfnPackThreads), 0, stream, k);
    a.x_norm = p.x_norm, a.g_norm = p.w_norm;
    a.g_exp = p.g_exp, a.u_exp = p.u_exp, a.x_exp = p.x_exp;
    a.g_whole = (const float*)Wg, a.u_whole = (const float*)Wu, a.x_whole = (const float*)X, a.D = p.D;
    a.k = p.ld, a.T = p.T, a.F = p.F;
    return a;
}

template <Store S, int FQ>
int launch_rows(const void* X, const void* Wg, const void* Wu, void* H, int T, int D, int F, int act, hipStream_t stream)
{
    const dim3 grid((unsigned)(F + 15) / 16), block(64 * ffn_row_waves<FQ>());
    const bool wide = !off(X, 16) && !off(Wg, 16) && !off(Wu, 16) && D % per16<S>() == 0;
    if (wide) hipLaunchKernelGGL((ffn_rows_kernel<S, FQ, true>), grid, block, 0, stream, X, Wg, Wu, H, T, D, F, act);
    else hipLaunchKernelGGL((ffn_rows_kernel<S, FQ, false>), grid, block, 0, stream, X, Wg, Wu, H, T, D, F, act);
    return launched();
}

template <Store S>
int run_ffn_fwd(const Ffn& p, const void* X, const void* Wg, const void* Wu, void* H, int act, hipStream_t stream)
{
    if (p.bytes == 0) {                            // (the plan of the rows' form)
        if (p.T <= 16) return launch_rows<S, 1>(X, Wg, Wu, H, p.T, p.D, p.F, act, stream);
        if (p.T <= 32) return launch_rows<S, 2>(X, Wg, Wu, H, p.T, p.D, p.F, act, stream);
        return launch_rows<S, 4>(X, Wg, Wu, H, p.T, p.D, p.F, act, stream);
    }
    FfnArgs a = ffn_pack<S>(p, X, Wg, Wu, false, false, stream);
    a.H = H;
    return run_gate<S, false>(a, act, stream);
}

template <class T, Store S, bool DX, bool TWO = false>
int launch_sum(FfnSum& a, FfnSum* b, hipStream_t stream)
{
    a.tiles_p = (a.P.size + T::BP - 1) / T::BP;
    const long long each = (long long)a.tiles_p * ((a.out_rows + T::BQ - 1) / T::BQ) * a.slices;
    if (each > 1 << 21) return SPHATTN_ERR_SHAPE;                     // (a launch has less than 2^32 threads)
    static std::atomic<uint64_t> done{0};
    if constexpr (DX) {
        const auto kern = ffn_dx_kernel<T, S, TWO>;
        if (T::LDS > 65536 && !raise_lds_limit(kern, T::LDS, done)) return SPHATTN_ERR_LAUNCH;
        hipLaunchKernelGGL(kern, dim3((unsigned)each), dim3(T::THREADS), T::LDS, stream, a);
    } else {
        const auto kern = ffn_dw_kernel<T, S, TWO>;
        if (T::LDS > 65536 && !raise_lds_limit(kern, T::LDS, done)) return SPHATTN_ERR_LAUNCH;
        if (b) b->tiles_p = a.tiles_p;
        hipLaunchKernelGGL(kern, dim3((unsigned)(b ? 2 * each : each)), dim3(T::THREADS), T::LDS, stream, a, b ? *b : a, (int)each);
    }
    return launched();
}

template <Store S>
int join_slices(const FfnSum (&sums)[3], int n, hipStream_t stream)
{
    FfnJoin j{};
    long long waves = 0;
    for (int i = 0; i < 3; ++i) {
        if (i < n) {
            j.sum[i] = sums[i];
            j.columns[i] = (sums[i].out_cols + 255) / 256;
            waves += (long long)sums[i].out_rows * j.columns[i];
        }
        if (i < 2) j.until[i] = waves;
    }
    if (waves > 1ll << 26) return SPHATTN_ERR_LAUNCH;                 // (slices are for results that fit memory many times over: 2^26 waves are 2^34 elements)
    hipLaunchKernelGGL((ffn_join_kernel<S>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, stream, j);
    return launched();
}

template <Store S>
int run_ffn_bwd(const Ffn& p, const void* X, const void* Wg, const void* Wu, const void* dH, void* dX, void* dWg, void* dWu, int act, hipStream_t stream)
{
    constexpr bool F32 = S == Store::F32, F16 = S == Store::F16;
    const bool dw = dWg || dWu;
    FfnArgs a{};
    a.X = Operand{nullptr, 0, p.ld * 2, 0};
    int rc = SPHATTN_OK;
    if (p.T > 0) {
        a = ffn_pack<S>(p, X, Wg, Wu, F16 || act == SPHATTN_GATE_RELU, F16, stream);
        a.dH = dH, a.dA = p.dA, a.dB = p.dB, a.part = (long long)p.T * p.ldf, a.ld = p.ldf;
        if (F16) {
            const long long tiles = (p.F + kTopCols - 1) / kTopCols, units = (long long)p.T + p.F;
            const auto tops = p.F >= 8 ? ffn_tops_kernel<true> : ffn_tops_kernel<false>;
            hipLaunchKernelGGL(tops, dim3((unsigned)(tiles * p.top_parts)), dim3(256), 0, stream, dH, p.x_norm, p.T, p.F, p.top_rows, p.row_top, p.col_top);
            hipLaunchKernelGGL(ffn_factors_kernel, dim3((unsigned)((units + kFactorThreads - 1) / kFactorThreads)), dim3(kFactorThreads), 0, stream, p.x_norm, p.w_norm, p.row_top,
                               p.col_top, p.T, p.F, p.top_parts, p.row_up, p.row_down, p.col_up, p.down_a, p.down_b);
            a.row_up = p.row_up, a.col_up = p.col_up, a.dA_all = dw ? p.dA_all : nullptr, a.dB_all = p.dB_all;
        }
        if constexpr (F32) rc = run_gate<S, true>(a, act, stream);
        else rc = p.two ? launch_gate<Mid, S, true, true>(a, act, stream) : run_gate<S, true>(a, act, stream);
    }
    const long long part = p.g_parts > 1 ? (long long)p.T * p.ldf * 2 : 0;
    auto sum = [&](auto is_dx, FfnSum& s, FfnSum* second, bool big) {
        constexpr bool DX = decltype(is_dx)::value;
        if constexpr (!F32)
            if (p.two) return launch_sum<Mid, S, DX, true>(s, second, stream);
        return big ? launch_sum<Big, S, DX>(s, second, stream) : launch_sum<Mid, S, DX>(s, second, stream);
    };
    // (fp32: what dA and dB are multiplied with are parts of their own)
    auto columns = [&](const Operand& o, const unsigned short* sum, int rows) {
        return F32 ? Operand{(const unsigned char*)sum, (long long)rows * p.ld * 2, p.ld * 2, p.ld} : Operand{o.data, 0, o.ld, p.ld};
    };
    FfnSum cut[3];                                 // in slices
    int n_cut = 0;
    if (rc == SPHATTN_OK && dX && p.T > 0) {
        FfnSum s{};
        s.P = columns(a.G, p.g_sum, p.F), s.P2 = columns(a.U, p.u_sum, p.F);
        s.Q = Operand{(const unsigned char*)p.dA, part, p.ldf * 2, p.T}, s.Q2 = Operand{(const unsigned char*)p.dB, part, p.ldf * 2, p.T};
        s.k = p.F, s.slices = p.dx.slices, s.out = dX, s.out_ld = s.out_cols = p.D, s.out_rows = p.T, s.part = p.part, s.part_ld = p.ld;
        if (F16) s.row_down = p.row_down;
        rc = sum(std::true_type{}, s, nullptr, p.dx.big);
        if (s.slices > 1) cut[n_cut++] = s;
    }
    if (rc == SPHATTN_OK && dw) {
        FfnSum s[2]{};
        int n = 0;
        for (int m = 0; m < 2; ++m) {
            void* out = m ? dWu : dWg;
            if (!out) continue;
            const unsigned short* q = m ? (F16 ? p.dB_all : p.dB) : (F16 ? p.dA_all : p.dA);
            s[n].P = columns(a.X, p.x_sum, p.T);
            s[n].Q = Operand{(const unsigned char*)q, part, p.ldf * 2, p.ldf};
            s[n].k = p.T, s[n].slices = p.dw.slices, s[n].out = out, s[n].out_ld = s[n].out_cols = p.D, s[n].out_rows = p.F;
            s[n].part = p.part_w ? p.part_w + (size_t)n * p.dw.slices * p.F * p.ld : nullptr, s[n].part_ld = p.ld;
            if (F16 && p.T > 0) s[n].row_down = m ? p.down_b : p.down_a;
            ++n;
        }
        FfnSum* second = n == 2 ? &s[1] : nullptr;
        rc = sum(std::false_type{}, s[0], second, p.dw.big);
        for (int m = 0; m < n && s[m].slices > 1; ++m) cut[n_cut++] = s[m];
    }
    if (rc == SPHATTN_OK && n_cut) rc = join_slices<S>(cut, n_cut, stream);
    return rc;
}

int ffn_check(const void* X, const void* Wg, const void* Wu, int T, int D, int F, int gate, int dtype)
{
    if (!ffn_shape(T, D, F)) return SPHATTN_ERR_SHAPE;
    const size_t e = (size_t)element_bytes(dtype);
    if (!e) return SPHATTN_ERR_DTYPE;
    if (!Wg || !Wu || (T > 0 && !X)) return SPHATTN_ERR_NULL;
    if (off(X, e) || off(Wg, e) || off(Wu, e)) return SPHATTN_ERR_ALIGN;
    if (gate < SPHATTN_GATE_SILU || gate > SPHATTN_GATE_RELU) return SPHATTN_ERR_VALUE;
    return SPHATTN_OK;
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
    c.a.log_share = heads_log_share((long long)B * N, Hq > Hk ? Hq : Hk, d);
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
    a.log_share = heads_log_share((long long)B * N, Hq > Hk ? Hq : Hk, d);
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

size_t sphattn_gated_ffn_workspace_bytes(int T, int D, int F, int dtype)
{
    return ffn_shape(T, D, F) && element_bytes(dtype) ? ffn_plan(T, D, F, dtype, false, nullptr).bytes : 0;
}

int sphattn_gated_ffn_fwd(const void* X, const void* Wg, const void* Wu, void* H, int T, int D, int F, int gate, int dtype,
                          void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = ffn_check(X, Wg, Wu, T, D, F, gate, dtype);
    if (rc != SPHATTN_OK) return rc;
    if (T > 0 && !H) return SPHATTN_ERR_NULL;
    const size_t e = (size_t)element_bytes(dtype);
    if (off(H, e)) return SPHATTN_ERR_ALIGN;
    const Ffn p = ffn_plan(T, D, F, dtype, false, workspace);
    if (p.bytes && (!workspace || off(workspace, 16) || workspace_bytes < p.bytes)) return SPHATTN_ERR_WORKSPACE;
    const Range written[] = {{H, (size_t)T * F * e}, {workspace, p.bytes}};
    const Range read[] = {{X, (size_t)T * D * e}, {Wg, (size_t)F * D * e}, {Wu, (size_t)F * D * e}};
    if (any_meet(written, read)) return SPHATTN_ERR_ALIAS;
    if (T == 0) return SPHATTN_OK;
    const hipStream_t s = (hipStream_t)stream;
    switch (dtype) {
    case SPHATTN_F32: return run_ffn_fwd<Store::F32>(p, X, Wg, Wu, H, gate, s);
    case SPHATTN_BF16: return run_ffn_fwd<Store::Bf16>(p, X, Wg, Wu, H, gate, s);
    default: return run_ffn_fwd<Store::F16>(p, X, Wg, Wu, H, gate, s);
    }
}

size_t sphattn_gated_ffn_bwd_workspace_bytes(int T, int D, int F, int dtype)
{
    return ffn_shape(T, D, F) && element_bytes(dtype) ? ffn_plan(T, D, F, dtype, true, nullptr).bytes : 0;
}

int sphattn_gated_ffn_bwd(const void* X, const void* Wg, const void* Wu, const void* dH, void* dX, void* dWg, void* dWu, int T, int D, int F,
                          int gate, int dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = ffn_check(X, Wg, Wu, T, D, F, gate, dtype);
    if (rc != SPHATTN_OK) return rc;
    if (T > 0 && (!dH || (!dX && !dWg && !dWu))) return SPHATTN_ERR_NULL;   // (an array of no rows has no address)
    const size_t e = (size_t)element_bytes(dtype);
    if (off(dH, e) || off(dX, e) || off(dWg, e) || off(dWu, e)) return SPHATTN_ERR_ALIGN;
    const Ffn p = ffn_plan(T, D, F, dtype, true, workspace);
    if (!workspace || off(workspace, 16) || workspace_bytes < p.bytes) return SPHATTN_ERR_WORKSPACE;
    const size_t x = (size_t)T * D * e, w = (size_t)F * D * e;
    const Range written[] = {{dX, x}, {dWg, w}, {dWu, w}, {workspace, p.bytes}};
    const Range read[] = {{X, x}, {Wg, w}, {Wu, w}, {dH, (size_t)T * F * e}};
    if (any_meet(written, read)) return SPHATTN_ERR_ALIAS;
    if (T == 0 && !dWg && !dWu) return SPHATTN_OK;
    const hipStream_t s = (hipStream_t)stream;
    switch (dtype) {
    case SPHATTN_F32: return run_ffn_bwd<Store::F32>(p, X, Wg, Wu, dH, dX, dWg, dWu, gate, s);
    case SPHATTN_BF16: return run_ffn_bwd<Store::Bf16>(p, X, Wg, Wu, dH, dX, dWg, dWu, gate, s);
    default: return run_ffn_bwd<Store::F16>(p, X, Wg, Wu, dH, dX, dWg, dWu, gate, s);
    }
}

}  // extern "C"
