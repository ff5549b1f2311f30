// Norms of queries and keys for each head and the rotation by their positions, in one pass, for gfx950.
//
//   r = 1 / sqrt(mean(x^2) + eps)      y = x r w      o = R y      R turns each pair of dimensions by position times frequency
//   dy = R^T do      dw = sum dy x r      dx = r (dy w - x r mean(dy w x r))
//
// Bound by memory: every row is read and written once (backward: two read, one written): 16384 tokens of 32 heads of 128 in bf16 51.5 us, 5.2 TB/s, what a copy of that size
// past the last-level cache reaches (5.15); with gradients 16384 tokens of 20 heads 31 forward and 50 backward.  One token: 5 us, a chain of two loads, an angle and a root.  A row is d elements on d / 8 lanes, a lane
// holding four neighbouring dimensions of each half, so that both kinds of pairs lie in one lane and a rotation exchanges nothing between lanes.
// cos and sin are formed once per token and lane, for all heads that the lane's group of lanes takes of that token.
#pragma once
#include "sphattn_store.hpp"

namespace sphattn {

struct HeadRows { unsigned char* data; long long batch, token, head; };   // strides in bytes

struct HeadSide {
    HeadRows x, o, dx;                             // backward: o is the gradient that comes in
    const void* w;
    int heads;
};

struct HeadsArgs {
    HeadSide side[2];                              // queries, keys
    const void* positions; int id_bytes; long long pos_axis, pos_batch;
    const float* inv_freq; int until[2];           // frequencies below until[0] go by the first axis, below until[1] by the second, the rest by the third
    int interleaved, norm;
    float eps;
    int B, N, log_share;                           // groups of lanes that share a token's heads: 1 << log_share
    float* partial;                                // backward: [workgroups][2][d] sums of dw, or NULL
};

constexpr int kHeadsThreads = 256;
constexpr int kHeadsMostGroups = 1024;             // backward: workgroups, each with a sum of dw for the joining kernel

// What D / 8 neighbouring lanes have, joined in each of them: exchanges within a row of sixteen lanes, no LDS
template <int D, typename Join>
__device__ __forceinline__ float over_row(float x, Join join)
{
    auto with = [&](auto ctrl) { x = join(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true))); };
    with(std::integral_constant<int, 0xB1>{});     // lane ^ 1
    with(std::integral_constant<int, 0x4E>{});     // lane ^ 2
    with(std::integral_constant<int, 0x141>{});    // the other four of eight
    if constexpr (D == 128) with(std::integral_constant<int, 0x140>{});   // the other eight of sixteen
    return x;
}
template <int D> __device__ __forceinline__ float sum_over_row(float x)
{
    return over_row<D>(x, [](float a, float b) { return a + b; });
}

// mean(x^2) + eps of a row of which this lane has eight elements, in each of its lanes
template <int D>
__device__ __forceinline__ float square_mean(const float (&x)[8], float eps)
{
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) ss = __builtin_fmaf(x[k], x[k], ss);
    return __builtin_fmaf(sum_over_row<D>(ss), 1.f / D, eps);
}

// Where fp32 has no square of the elements (1e20, or 1e-25 with an eps as small) a row is first multiplied by a power of two that brings the larger of its elements and eps's root to
// 1; it is left as it is where it is not finite, or zeros without eps, which are what the formula makes of them.  Rare.
template <Store S> __device__ __forceinline__ bool no_square(float size) { return S != Store::F16 && !(size >= 0x1p-96f && size < __builtin_inff()); }
template <Store S, int D>
__device__ __forceinline__ int bring_near(float (&x)[8], float& size, float eps)
{
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = fmaxf(top, __builtin_fabsf(x[k]));
    top = fmaxf(over_row<D>(top, [](float a, float b) { return fmaxf(a, b); }), __builtin_sqrtf(eps));
    const bool far = no_square<S>(size) && size == size && top > 0.f && top < __builtin_inff();
    const int power = far ? -__builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __builtin_ldexpf(x[k], power);
    const float again = square_mean<D>(x, __builtin_ldexpf(eps, 2 * power));
    size = far ? again : size;
    return power;
}

// Four neighbouring elements.  (aligned to an element: the memory pipe takes them in one access all the same)
template <Store S> struct Four { int w[S == Store::F32 ? 4 : 2]; };

template <Store S> __device__ __forceinline__ Four<S> load4(const unsigned char* p)
{
    Four<S> f;
    __builtin_memcpy(&f, p, sizeof(f));
    return f;
}
template <Store S> __device__ __forceinline__ void widen4(const Four<S>& f, float* x)
{
    if constexpr (S == Store::F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(float, f.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (S == Store::Bf16) {
                x[2 * i] = __builtin_bit_cast(float, f.w[i] << 16);
                x[2 * i + 1] = __builtin_bit_cast(float, f.w[i] & (int)0xffff0000);
            } else {
                const f16x2 h = __builtin_bit_cast(f16x2, f.w[i]);
                x[2 * i] = (float)h[0];
                x[2 * i + 1] = (float)h[1];
            }
        }
    }
}
template <Store S> __device__ __forceinline__ void store4(unsigned char* p, const float* x)
{
    Four<S> f;
#pragma unroll
    for (int i = 0; i < (S == Store::F32 ? 4 : 2); ++i) {
        if constexpr (S == Store::F32) f.w[i] = __builtin_bit_cast(int, x[i]);
        else f.w[i] = pack2<S == Store::F16>(x[2 * i], x[2 * i + 1]);
    }
    __builtin_memcpy(p, &f, sizeof(f));
}

// A row's eight dimensions of this lane: 0..3 of the first half, 4..7 of the second
template <Store S, int D> struct HeadRow { Four<S> lo, hi; };
template <Store S, int D> __device__ __forceinline__ HeadRow<S, D> load_row(const unsigned char* p, int l)
{
    constexpr int E = store_bytes<S>();
    return HeadRow<S, D>{load4<S>(p + 4 * l * E), load4<S>(p + (D / 2 + 4 * l) * E)};
}
template <Store S, int D> __device__ __forceinline__ void widen_row(const HeadRow<S, D>& r, float (&x)[8])
{
    widen4<S>(r.lo, x);
    widen4<S>(r.hi, x + 4);
}
template <Store S, int D> __device__ __forceinline__ void store_row(unsigned char* p, int l, const float (&x)[8])
{
    constexpr int E = store_bytes<S>();
    store4<S>(p + 4 * l * E, x);
    store4<S>(p + (D / 2 + 4 * l) * E, x + 4);
}

// Pairs of a lane's eight dimensions: (i, 4 + i), or neighbours.  `back`: turned the other way.
__device__ __forceinline__ void rotate(float (&x)[8], const float (&cos)[4], const float (&sin)[4], bool interleaved, float back)
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int a0 = i, b0 = 4 + i, a1 = 2 * i, b1 = 2 * i + 1;
        const float a = interleaved ? x[a1] : x[a0], b = interleaved ? x[b1] : x[b0], s = sin[i] * back;
        const float ta = __builtin_fmaf(a, cos[i], -b * s), tb = __builtin_fmaf(b, cos[i], a * s);
        y[i] = ta;
        y[4 + i] = tb;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = interleaved ? (i & 1 ? y[4 + i / 2] : y[i / 2]) : y[i];
        x[4 + i] = interleaved ? (i & 1 ? y[4 + 2 + i / 2] : y[2 + i / 2]) : y[4 + i];
    }
}

// What a lane keeps for all rows: frequencies in turns per position, axes, weights
template <Store S, int D>
struct HeadsLane {
    double turns[4];
    int axes;                                      // two bits each (four registers would be what the backward kernel has not)
    float w[2][8];

    __device__ __forceinline__ void begin(const HeadsArgs& a, int l)
    {
        axes = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int f = !a.interleaved ? 4 * l + i : i < 2 ? 2 * l + i : D / 4 + 2 * l + i - 2;
            turns[i] = a.positions ? (double)a.inv_freq[f] * 0.15915494309189533577 : 0.0;
            axes |= (f < a.until[0] ? 0 : f < a.until[1] ? 1 : 2) << (2 * i);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (a.side[s].w) {
                const HeadRow<S, D> r = load_row<S, D>((const unsigned char*)a.side[s].w, l);
                widen_row<S, D>(r, w[s]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) w[s][i] = 1.f;
            }
        }
    }
    // Turns are formed in fp64, off by 2^-51 of themselves (the frequency in turns, 1 / 2 pi and the product are rounded once each), and so is their fraction, which is then
    // rounded to fp32; what fp32 would leave of an angle of a far position is no angle any more.
    // (loaded before a token's rows are, used behind that)
    struct Place { long long at[4]; };
    __device__ __forceinline__ Place place(const HeadsArgs& a, long long b, long long n) const
    {
        Place p;
        int axes = this->axes;
        asm volatile("" : "+v"(axes));             // (or the strides' products are kept for all tokens, two registers each)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long at = (axes >> (2 * i) & 3) * a.pos_axis + b * a.pos_batch + n;
            p.at[i] = a.id_bytes == 4 ? (long long)((const int*)a.positions)[at] : ((const long long*)a.positions)[at];
        }
        return p;
    }
    __device__ __forceinline__ void angles(const Place& p, float (&cos)[4], float (&sin)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double t = (double)p.at[i] * turns[i];
            sincospif(2.f * (float)(t - __builtin_rint(t)), &sin[i], &cos[i]);
        }
    }
};

// Which token and which of its heads a group of lanes takes.  (32-bit numbers: a division of 64 bits is a long program; there are less than 2^31 tokens, and
// they are shared only where they are few)
struct HeadsUnit {
    long long b, n;
    int first;
    __device__ __forceinline__ HeadsUnit(const HeadsArgs& a, unsigned u)
    {
        const unsigned token = u >> a.log_share, batch = token / (unsigned)a.N;
        b = batch;
        n = token - batch * (unsigned)a.N;
        first = (int)(u - (token << a.log_share));
    }
};

// Groups of d / 8 lanes take tokens, or (where tokens are few) every share-th head of one.
template <Store S, int D, bool ROTATE>
__global__ __launch_bounds__(kHeadsThreads)
void heads_fwd_kernel(HeadsArgs a)
{
    constexpr int LANES = D / 8, AHEAD = 4;
    const int l = threadIdx.x % LANES;
    HeadsLane<S, D> lane;
    lane.begin(a, l);
    const unsigned units = (unsigned)a.B * (unsigned)a.N << a.log_share, step = gridDim.x * (kHeadsThreads / LANES);
    const int share = 1 << a.log_share;
    for (unsigned u = blockIdx.x * (kHeadsThreads / LANES) + threadIdx.x / LANES; u < units; u += step) {
        const HeadsUnit unit(a, u);
        typename HeadsLane<S, D>::Place place;
        if constexpr (ROTATE) place = lane.place(a, unit.b, unit.n);
        HeadRow<S, D> rows[2][AHEAD];
        auto fetch = [&](int s, int h0) {
            const HeadSide& side = a.side[s];
            const unsigned char* from = side.x.data + unit.b * side.x.batch + unit.n * side.x.token;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) rows[s][i] = load_row<S, D>(from + min(h0 + i * share, side.heads - 1) * side.x.head, l);
        };
        fetch(0, unit.first);
        if (unit.first < a.side[1].heads) fetch(1, unit.first);
        float cos[4], sin[4];
        if constexpr (ROTATE) lane.angles(place, cos, sin);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const HeadSide& side = a.side[s];
            unsigned char* to = side.o.data + unit.b * side.o.batch + unit.n * side.o.token;
            for (int h0 = unit.first; h0 < side.heads; h0 += AHEAD * share) {
                if (h0 > unit.first) fetch(s, h0);
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int h = h0 + i * share;
                    float x[8], size = 1.f;
                    widen_row<S, D>(rows[s][i], x);
                    if (a.norm) {
                        size = square_mean<D>(x, a.eps);
                        if (__ballot(no_square<S>(size))) bring_near<S, D>(x, size, a.eps);
                    }
                    const float r = 1.f / __builtin_sqrtf(size);
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = x[k] * r * lane.w[s][k];
                    if constexpr (ROTATE) rotate(x, cos, sin, a.interleaved, 1.f);
                    if (h < side.heads) store_row<S, D>(to + h * side.o.head, l, x);
                }
            }
        }
    }
}

// (one register more than four waves have room for took 16384 tokens of 20 heads in bf16 from 51.8 us to 59.2)
template <Store S, int D, bool ROTATE>
__global__ __launch_bounds__(kHeadsThreads, 4)
void heads_bwd_kernel(HeadsArgs a)
{
    constexpr int LANES = D / 8, AHEAD = 2;
    const int l = threadIdx.x % LANES;
    HeadsLane<S, D> lane;
    lane.begin(a, l);
    float dw[2][8];
#pragma unroll
    for (int k = 0; k < 8; ++k) dw[0][k] = dw[1][k] = 0.f;
    const unsigned units = (unsigned)a.B * (unsigned)a.N << a.log_share, step = gridDim.x * (kHeadsThreads / LANES);
    const int share = 1 << a.log_share;
    for (unsigned u = blockIdx.x * (kHeadsThreads / LANES) + threadIdx.x / LANES; u < units; u += step) {
        const HeadsUnit unit(a, u);
        const long long b = unit.b, n = unit.n;
        const int first = unit.first;
        float cos[4], sin[4];
        if constexpr (ROTATE) lane.angles(lane.place(a, b, n), cos, sin);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const HeadSide& side = a.side[s];
            const unsigned char* from = side.x.data + b * side.x.batch + n * side.x.token;
            const unsigned char* grad = side.o.data + b * side.o.batch + n * side.o.token;
            unsigned char* to = side.dx.data ? side.dx.data + b * side.dx.batch + n * side.dx.token : nullptr;
            for (int h0 = first; h0 < side.heads; h0 += AHEAD * share) {
                HeadRow<S, D> rows[AHEAD], grads[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int h = min(h0 + i * share, side.heads - 1);
                    rows[i] = load_row<S, D>(from + h * side.x.head, l);
                    grads[i] = load_row<S, D>(grad + h * side.o.head, l);
                }
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int h = h0 + i * share;
                    float x[8], dy[8];
                    widen_row<S, D>(rows[i], x);
                    widen_row<S, D>(grads[i], dy);
                    if constexpr (ROTATE) rotate(dy, cos, sin, a.interleaved, -1.f);
                    float r = 1.f, along = 0.f;
                    if (a.norm) {
                        float size = square_mean<D>(x, a.eps);
                        int power = 0;
                        if (__ballot(no_square<S>(size))) power = bring_near<S, D>(x, size, a.eps);
                        r = 1.f / __builtin_sqrtf(size);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            x[k] *= r;
                            along = __builtin_fmaf(dy[k] * lane.w[s][k], x[k], along);
                        }
                        if constexpr (S != Store::F16) r = __builtin_ldexpf(r, power);
                        along = sum_over_row<D>(along) * (1.f / D);
                    }
                    if (h >= side.heads) continue;
                    float dx[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        dw[s][k] = __builtin_fmaf(dy[k], x[k], dw[s][k]);
                        const float dn = dy[k] * lane.w[s][k];
                        dx[k] = a.norm ? r * __builtin_fmaf(-x[k], along, dn) : dn;
                    }
                    if (to) store_row<S, D>(to + h * side.dx.head, l, dx);
                }
            }
        }
    }
    if (!a.partial) return;
    // the workgroup's sums: over the groups of lanes of a wave, then over the waves
    constexpr int WAVES = kHeadsThreads / 64;
    __shared__ float sums[WAVES][2][D];
    const int wave = threadIdx.x >> 6, in = threadIdx.x & 63;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float x = dw[s][k];
#pragma unroll
            for (int m = LANES; m < 64; m <<= 1) x += __shfl_xor(x, m);
            if (in < LANES) sums[wave][s][(k < 4 ? 0 : D / 2) + 4 * l + (k & 3)] = x;
        }
    __syncthreads();
    if ((int)threadIdx.x < 2 * D) {
        const float* at = &sums[0][0][0] + threadIdx.x;
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x += at[w * 2 * D];
        a.partial[(size_t)blockIdx.x * 2 * D + threadIdx.x] = x;
    }
}

// dw from the workgroups' sums, in fp64: a workgroup takes sixteen columns, 16 lanes' worth of rows at a time
template <Store S>
__global__ __launch_bounds__(1024)
void heads_dw_kernel(const float* __restrict__ partial, int groups, int D, void* __restrict__ dwq, void* __restrict__ dwk)
{
    __shared__ double shared[64][16];
    const int col = (int)blockIdx.x * 16 + (threadIdx.x & 15), row = threadIdx.x >> 4;
    double x = 0.0;
#pragma unroll 8
    for (int g = row; g < groups; g += 64) x += partial[(size_t)g * 2 * D + col];
    shared[row][threadIdx.x & 15] = x;
    __syncthreads();
    if (threadIdx.x >= 16) return;
    x = 0.0;
#pragma unroll 16
    for (int r = 0; r < 64; ++r) x += shared[r][threadIdx.x];
    void* out = col < D ? dwq : dwk;
    if (out) store_el<S>(out, col < D ? col : col - D, (float)x);
}

}  // namespace sphattn
