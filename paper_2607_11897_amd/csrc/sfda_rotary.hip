// Rotary positions (gfx950): pairs of channels (a, b) of a token at position p turned by the angle of
// their row of the tables, (a c - b s, a s + b c) with c, s = cos, sin[p, i]; the inverse turn is the gradient.
// Memory-bound: every element read and written once.  A thread keeps its position's cosines and
// sines in registers over HPT heads, so that the float32 tables cost an eighth of the bfloat16 elements' traffic and
// not as much as these.
#include "sfda_device.h"
#include "sfda_layer.h"

#include <string.h>

namespace sfda {
namespace {

constexpr int NT = 256;
constexpr int HPT = 4;      // heads of a thread

template <typename E> struct Vec;
template <> struct Vec<uint16_t> { static constexpr int N = 8; };
template <> struct Vec<float> { static constexpr int N = 4; };

// n of N elements from p (any alignment of the element type) as float32
template <typename E> __device__ __forceinline__ void get(float (&x)[Vec<E>::N], const E* p, int n)
{
    constexpr int N = Vec<E>::N;
    E e[N] = {};
    if (n >= N) {
        memcpy(e, p, 16);
    } else {
        for (int i = 0; i < N; ++i)
            if (i < n) e[i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = Elem<E>::load(e, i);
}
__device__ __forceinline__ void to(float& e, float x) { e = x; }
__device__ __forceinline__ void to(uint16_t& e, float x) { e = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }
template <typename E> __device__ __forceinline__ void put(E* p, const float (&x)[Vec<E>::N], int n)
{
    constexpr int N = Vec<E>::N;
    E e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) to(e[i], x[i]);
    if (n >= N) {
        memcpy(p, e, 16);
    } else {
        for (int i = 0; i < N; ++i)
            if (i < n) p[i] = e[i];
    }
}

// A unit of a row: INTER: N channels, of which those below `rot` are turned in pairs (2i, 2i + 1).
// Halves: N pairs (i, i + rot / 2), or, past the pairs' units, N channels that pass through.
template <typename E, bool INTER>
__global__ __launch_bounds__(NT) void rotary_kernel(RotaryLaunch L, int units, int groups)
{
    constexpr int N = Vec<E>::N;
    const long long id = static_cast<long long>(blockIdx.x) * NT + threadIdx.x;
    const int u = static_cast<int>(id % units);
    const long long rest = id / units;
    const int t = static_cast<int>(rest % L.T);
    const long long rest2 = rest / L.T;
    const int hg = static_cast<int>(rest2 % groups);
    const int b = static_cast<int>(rest2 / groups);
    if (b >= L.B) return;

    const int half = L.rot / 2, pair_units = (half + N - 1) / N;
    const bool through = INTER ? u * N >= L.rot : u >= pair_units;
    // first channel, its count; the second's for halves
    const int ch = INTER ? u * N : through ? L.rot + (u - pair_units) * N : u * N;
    const int n = INTER ? L.D - ch : through ? L.D - ch : half - ch;
    float c[N], s[N];       // of pair i
    if (!through) {
        long long pos = L.offset + t;
        if (L.positions != nullptr) {
            const long long at = b * L.pos_b + t;
            pos = L.pos64 ? static_cast<const long long*>(L.positions)[at] : static_cast<const int*>(L.positions)[at];
        }
        const int first = INTER ? ch / 2 : ch, pairs = INTER ? N / 2 : N;
        const bool there = pos >= 0 && pos < L.P;       // a position without a row of the tables gives NaN
        const long long row = there ? pos * half : 0;
#pragma unroll
        for (int i = 0; i < pairs; ++i) {
            const bool in = first + i < half;
            const long long at = row + (in ? first + i : 0);
            c[i] = L.cos[at];
            s[i] = L.inverse ? -L.sin[at] : L.sin[at];
            if (!there) c[i] = s[i] = __builtin_nanf("");
            if (!in) { c[i] = 1.f; s[i] = 0.f; }        // channels past the rotated ones in the last unit
        }
    }
    for (int i = 0; i < HPT; ++i) {
        const int hh = hg * HPT + i;
        if (hh >= L.Hq + L.Hk) break;
        const bool isk = hh >= L.Hq;
        const int h = isk ? hh - L.Hq : hh;
        const long long* ss = isk ? L.k_s : L.q_s;
        const long long* os = isk ? L.ko_s : L.qo_s;
        const E* src = static_cast<const E*>(isk ? L.k : L.q) + b * ss[0] + h * ss[1] + t * ss[2] + ch;
        E* dst = static_cast<E*>(isk ? L.ko : L.qo) + b * os[0] + h * os[1] + t * os[2] + ch;
        float x[N];
        get<E>(x, src, n);
        if (!through) {
            if (INTER) {
#pragma unroll
                for (int p = 0; p < N / 2; ++p) {
                    const float a = x[2 * p], d = x[2 * p + 1];
                    // (a pair past the rotated ones passes bit for bit, infinities too)
                    if (ch + 2 * p < L.rot) {
                        x[2 * p] = a * c[p] - d * s[p];
                        x[2 * p + 1] = a * s[p] + d * c[p];
                    }
                }
            } else {
                float y[N];
                get<E>(y, src + half, n);
#pragma unroll
                for (int p = 0; p < N; ++p) {
                    const float a = x[p], d = y[p];
                    x[p] = a * c[p] - d * s[p];
                    y[p] = a * s[p] + d * c[p];
                }
                put<E>(dst + half, y, n);
            }
        }
        put<E>(dst, x, n);
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryLaunch& L, hipStream_t st)
{
    const int N = L.bf16 ? 8 : 4;
    const int units = L.interleaved ? (L.D + N - 1) / N : (L.rot / 2 + N - 1) / N + (L.D - L.rot + N - 1) / N;
    const int groups = (L.Hq + L.Hk + HPT - 1) / HPT;
    const long long threads = static_cast<long long>(L.B) * groups * L.T * units;
    const dim3 grid(static_cast<unsigned>((threads + NT - 1) / NT)), block(NT);
    if (L.bf16) {
        if (L.interleaved) hipLaunchKernelGGL((rotary_kernel<uint16_t, true>), grid, block, 0, st, L, units, groups);
        else hipLaunchKernelGGL((rotary_kernel<uint16_t, false>), grid, block, 0, st, L, units, groups);
    } else {
        if (L.interleaved) hipLaunchKernelGGL((rotary_kernel<float, true>), grid, block, 0, st, L, units, groups);
        else hipLaunchKernelGGL((rotary_kernel<float, false>), grid, block, 0, st, L, units, groups);
    }
    return hipGetLastError();
}

}  // namespace sfda
