// Tensors of fp32, bf16 and fp16 in registers: loads, stores and roundings that the kernels around the attention share.
#pragma once
#include "sphattn_device.hpp"

namespace sphattn {

// ---- element types --------------------------------------------------------------------------------

enum class Store { F32, Bf16, F16 };
template <Store S> constexpr int store_bytes() { return S == Store::F32 ? 4 : 2; }

template <Store S> __device__ __forceinline__ float load_el(const void* p, size_t i)
{
    if constexpr (S == Store::F32) return ((const float*)p)[i];
    else if constexpr (S == Store::Bf16) return (float)((const __bf16*)p)[i];
    else return (float)((const _Float16*)p)[i];
}
template <Store S> __device__ __forceinline__ void store_el(void* p, size_t i, float x)
{
    if constexpr (S == Store::F32) ((float*)p)[i] = x;
    else if constexpr (S == Store::Bf16) ((__bf16*)p)[i] = (__bf16)x;
    else ((_Float16*)p)[i] = (_Float16)x;
}

// 16 bytes of elements as floats, and back (to nearest even)
template <Store S> constexpr int per16() { return 16 / store_bytes<S>(); }
template <Store S> __device__ __forceinline__ void widen16(i32x4 w, float (&x)[per16<S>()])
{
    if constexpr (S == Store::F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int bits = w[i];                 // (a bit cast of the vector's element itself takes the vector's first)
            x[i] = __builtin_bit_cast(float, bits);
        }
    } else if constexpr (S == Store::Bf16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, w[i] & (int)0xffff0000);
        }
    } else {
        const f16x8 h = __builtin_bit_cast(f16x8, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)h[i];
    }
}
template <Store S> __device__ __forceinline__ i32x4 narrow16(const float (&x)[per16<S>()])
{
    i32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (S == Store::F32) w[i] = __builtin_bit_cast(int, x[i]);
        else w[i] = pack2<S == Store::F16>(x[2 * i], x[2 * i + 1]);
    }
    return w;
}

// per16 elements from element `at` on, `left` of which are wanted (the rest zeros), and back.  WIDE: 16-byte aligned and all wanted;
// otherwise aligned to an element only, which the memory pipe takes in one access too (with one element a lane 8192 rows of 515 took
// two to three times as long).  room: elements to the end of the tensor, up to which more than is wanted may be read.
template <Store S, bool WIDE> __device__ __forceinline__ i32x4 load16(const void* p, size_t at, int left, size_t room)
{
    constexpr int N = per16<S>();
    if constexpr (WIDE) return ((const i32x4*)p)[at / N];
    i32x4 w = {0, 0, 0, 0};
    const unsigned char* from = (const unsigned char*)p + at * store_bytes<S>();
    if (room >= (size_t)N) {
        __builtin_memcpy(&w, from, 16);
    } else {
#pragma unroll
        for (int i = 0; i < N - 1; ++i) {
            if (i >= left) break;
            if constexpr (S == Store::F32) w[i] = ((const int*)from)[i];
            else w[i / 2] |= (int)((uint32_t)((const unsigned short*)from)[i] << (16 * (i & 1)));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (S == Store::F32) w[i] = i < left ? w[i] : 0;
        else w[i] = 2 * i + 1 < left ? w[i] : 2 * i < left ? w[i] & 0xffff : 0;
    }
    return w;
}
template <Store S, bool WIDE> __device__ __forceinline__ void store16(void* p, size_t at, i32x4 w, int left)
{
    constexpr int N = per16<S>();
    if constexpr (WIDE) {
        ((i32x4*)p)[at / N] = w;
        return;
    }
    unsigned char* to = (unsigned char*)p + at * store_bytes<S>();
    if (left >= N) {
        __builtin_memcpy(to, &w, 16);
    } else {
#pragma unroll
        for (int i = 0; i < N - 1; ++i) {
            if (i >= left) break;
            if constexpr (S == Store::F32) ((int*)to)[i] = w[i];
            else ((unsigned short*)to)[i] = (unsigned short)((uint32_t)w[i / 2] >> (16 * (i & 1)));
        }
    }
}

// Token ids of 4 or 8 bytes as ints: what does not fit an int is no valid id (negative stays negative, the rest too large).
__device__ __forceinline__ int load_id(const void* ids, int id_bytes, size_t i)
{
    if (id_bytes == 4) return ((const int*)ids)[i];
    const long long x = ((const long long*)ids)[i];
    return x < 0 ? -1 : x > 0x7fffffff ? 0x7fffffff : (int)x;
}

}  // namespace sphattn
