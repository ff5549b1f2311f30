// The 2-norm of many tensors together and their scaling down to a limit, for gfx950.
//
//   n = sqrt(sum over all elements of g^2)          out = g * min(1, limit / (n + 1e-6))
//
// Bound by memory (every element is read twice and written once) and, for small models, by launches: one for the squares
// and one for the scaling, whatever the number of tensors up to kClipBatch.  The list of tensors travels in the
// kernels' arguments: no copy to the device, nothing to keep, and a captured graph holds it.  The scaling walks backwards through what the squares
// read last and stores past the caches, so that a part of the second reading, and of the next call's first, comes from the last-level cache:
// 200 million bf16 201 us a call (squares 66, scaling 135: 6 TB/s), forwards with ordinary stores 237 (99 and 134); 400 000 fp32 in twelve tensors 10.8, two launches.
#pragma once
#include "sphattn_embed.hpp"

namespace sphattn {

constexpr int kClipThreads = 256, kClipBatch = 120;
constexpr int kClipChunk = 8192;                   // elements that a workgroup takes at a time, of one tensor
constexpr long long kClipMostElements = 1ll << 40; // of a call: chunk numbers are ints
constexpr int kClipMostGroups = 1024;              // workgroups of a launch: four per CU

struct ClipList {
    const void* in[kClipBatch];
    void* out[kClipBatch];
    long long size[kClipBatch];
    int first[kClipBatch];                         // number of its first chunk; INT_MAX behind the last tensor
    unsigned char type[kClipBatch];                // Store; bit 7: in and out are 16-byte aligned
    long long chunks;
};
static_assert(sizeof(ClipList) <= 4000, "a launch's arguments are 4 KB");

// Which tensor chunk c lies in: every lane looks at two entries, instead of a search whose loads wait for each other.
__device__ __forceinline__ int clip_tensor(const ClipList& list, int c, int lane)
{
    int n = __builtin_popcountll(__ballot(list.first[lane] <= c));
    n += __builtin_popcountll(__ballot(lane + 64 < kClipBatch && list.first[lane + 64 < kClipBatch ? lane + 64 : 0] <= c));
    return n - 1;
}

// Squares and their sums in fp64: no value of any of the three types overflows or vanishes there, and at two fp64
// instructions per element the vector units have ten times the rate that memory has.
template <Store S>
__device__ __forceinline__ double clip_squares(const void* in, long long at, int n, bool wide, int tid)
{
    double sum = 0.0;
    if (wide) {
        constexpr int N = per16<S>(), ROUNDS = kClipChunk / N / kClipThreads;
        const i32x4* p = (const i32x4*)in + at / N;
        i32x4 w[ROUNDS];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int c = r * kClipThreads + tid;
            w[r] = i32x4{0, 0, 0, 0};
            if ((c + 1) * N <= n) w[r] = p[c];
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            float x[N];
            widen16<S>(w[r], x);
#pragma unroll
            for (int i = 0; i < N; ++i) sum = __builtin_fma((double)x[i], (double)x[i], sum);
        }
        const int rest = n / N * N + tid;
        if (rest < n) {
            const double x = load_el<S>(in, at + rest);
            sum = __builtin_fma(x, x, sum);
        }
    } else {
        for (int c = tid; c < n; c += kClipThreads) {
            const double x = load_el<S>(in, at + c);
            sum = __builtin_fma(x, x, sum);
        }
    }
    return sum;
}

__device__ __forceinline__ double sum_over_group(double x, double* shared, int tid)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    __syncthreads();
    if ((tid & 63) == 0) shared[tid >> 6] = x;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < kClipThreads / 64; ++w) s += shared[w];
    return s;
}

__global__ __launch_bounds__(kClipThreads)
void clip_squares_kernel(ClipList list, double* __restrict__ sums)
{
    __shared__ double shared[kClipThreads / 64];
    const int tid = threadIdx.x;
    double sum = 0.0;
    for (long long c = blockIdx.x; c < list.chunks; c += gridDim.x) {
        const int k = __builtin_amdgcn_readfirstlane(clip_tensor(list, (int)c, tid & 63));
        const long long at = (c - list.first[k]) * kClipChunk;
        const int n = (int)min((long long)kClipChunk, list.size[k] - at), type = list.type[k];
        switch (type & 127) {
        case (int)Store::F32: sum += clip_squares<Store::F32>(list.in[k], at, n, type & 128, tid); break;
        case (int)Store::Bf16: sum += clip_squares<Store::Bf16>(list.in[k], at, n, type & 128, tid); break;
        default: sum += clip_squares<Store::F16>(list.in[k], at, n, type & 128, tid); break;
        }
    }
    sum = sum_over_group(sum, shared, tid);
    if (tid == 0) sums[blockIdx.x] = sum;
}

template <Store S>
__device__ __forceinline__ void clip_scale(const void* in, void* out, long long at, int n, bool wide, float f, int tid)
{
    if (wide) {
        constexpr int N = per16<S>(), ROUNDS = kClipChunk / N / kClipThreads;
        const i32x4* p = (const i32x4*)in + at / N;
        i32x4* q = (i32x4*)out + at / N;
        i32x4 w[ROUNDS];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int c = r * kClipThreads + tid;
            w[r] = i32x4{0, 0, 0, 0};
            if ((c + 1) * N <= n) w[r] = p[c];
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int c = r * kClipThreads + tid;
            float x[N];
            widen16<S>(w[r], x);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] *= f;
            if ((c + 1) * N <= n) __builtin_nontemporal_store(narrow16<S>(x), &q[c]);
        }
        const int rest = n / N * N + tid;
        if (rest < n) store_el<S>(out, at + rest, load_el<S>(in, at + rest) * f);
    } else {
        for (int c = tid; c < n; c += kClipThreads) store_el<S>(out, at + c, load_el<S>(in, at + c) * f);
    }
}

// Every workgroup adds the squares' sums up for itself, in the same order: cheaper than a launch in between.  Where nothing is to
// be scaled, tensors that are their own output are left alone.
__global__ __launch_bounds__(kClipThreads)
void clip_scale_kernel(ClipList list, const double* __restrict__ sums, int n_sums, float limit, float* __restrict__ norm, int first_launch)
{
    __shared__ double shared[kClipThreads / 64];
    const int tid = threadIdx.x;
    double sum = 0.0;
    for (int i = tid; i < n_sums; i += kClipThreads) sum += sums[i];
    const double n = __builtin_sqrt(sum_over_group(sum, shared, tid));
    const double ratio = (double)limit / (n + 1e-6);
    const float f = ratio < 1.0 ? (float)ratio : ratio >= 1.0 ? 1.f : __builtin_nanf("");   // (NaN stays NaN)
    if (first_launch && blockIdx.x == 0 && tid == 0) *norm = (float)n;
    for (long long c = list.chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
        const int k = __builtin_amdgcn_readfirstlane(clip_tensor(list, (int)c, tid & 63));
        if (f == 1.f && list.in[k] == list.out[k]) continue;
        const long long at = (c - list.first[k]) * kClipChunk;
        const int m = (int)min((long long)kClipChunk, list.size[k] - at), type = list.type[k];
        switch (type & 127) {
        case (int)Store::F32: clip_scale<Store::F32>(list.in[k], list.out[k], at, m, type & 128, f, tid); break;
        case (int)Store::Bf16: clip_scale<Store::Bf16>(list.in[k], list.out[k], at, m, type & 128, f, tid); break;
        default: clip_scale<Store::F16>(list.in[k], list.out[k], at, m, type & 128, f, tid); break;
        }
    }
}

}  // namespace sphattn
