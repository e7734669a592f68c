// 16-byte vectors of float32 or bfloat16 elements at any address, as float32 values (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

namespace sfda {
namespace vec {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// (global memory takes unaligned vectors)
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1), may_alias));
__device__ __forceinline__ u32x4 load16(const void* p) { return *static_cast<const u32x4_any*>(p); }
__device__ __forceinline__ void store16(void* p, u32x4 x) { *static_cast<u32x4_any*>(p) = x; }

// two float32 as a pair of bfloat16, each to nearest even
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    bf16x2 p;
    p[0] = static_cast<__bf16>(a);
    p[1] = static_cast<__bf16>(b);
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

template <typename E> struct Vec { static constexpr int N = 16 / sizeof(E); };

// the n < N first elements of a row, zeros behind them
template <typename E> __device__ __forceinline__ u32x4 load_few(const E* p, int n)
{
    constexpr int PER = 4 / sizeof(E);
    u32x4 x = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < Vec<E>::N - 1; ++i)
        if (i < n) {
            uint32_t u = 0;
            memcpy(&u, p + i, sizeof(E));
            x[i / PER] |= u << (i % PER * 16);
        }
    return x;
}
template <typename E> __device__ __forceinline__ u32x4 load(const E* p, int n) { return n >= Vec<E>::N ? load16(p) : load_few(p, n); }
template <typename E> __device__ __forceinline__ void store(E* p, u32x4 x, int n)
{
    if (n >= Vec<E>::N) {
        store16(p, x);
        return;
    }
    constexpr int PER = 4 / sizeof(E);
#pragma unroll
    for (int i = 0; i < Vec<E>::N - 1; ++i)
        if (i < n) {
            const uint32_t u = x[i / PER] >> (i % PER * 16);
            memcpy(p + i, &u, sizeof(E));
        }
}

template <typename E> __device__ __forceinline__ void unpack(float (&f)[Vec<E>::N], u32x4 x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 2) {
            f[2 * i] = lo_f32(x[i]);
            f[2 * i + 1] = hi_f32(x[i]);
        } else {
            f[i] = __uint_as_float(x[i]);
        }
    }
}
template <typename E> __device__ __forceinline__ u32x4 pack(const float (&f)[Vec<E>::N])
{
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 2) x[i] = pack2(f[2 * i], f[2 * i + 1]);
        else x[i] = __float_as_uint(f[i]);
    }
    return x;
}

}  // namespace vec
}  // namespace sfda
