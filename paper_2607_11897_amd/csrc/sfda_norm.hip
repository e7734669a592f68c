// Group norm of every token's heads with an activation or an activated gate (gfx950), forward and backward.
//   x^ = (x - mean) / sqrt(var + eps) over the D channels of one head of one token,  n = x^ w + b,
//   y = act(n) without a gate, n act(z) with one;  act(z) = z or z sigmoid(z).
// Memory-bound.  A group of lanes holds a row in registers (two-pass variance, float32), a workgroup keeps
// one head's weights in registers over its strip of tokens, and in the backward their gradients too.
#include "sfda_device.h"
#include "sfda_layer.h"

#include <string.h>

namespace sfda {
namespace {

constexpr int NT = 256;

template <typename E> struct Vec;
template <> struct Vec<uint16_t> { static constexpr int N = 8; };
template <> struct Vec<float> { static constexpr int N = 4; };

template <typename E> __device__ __forceinline__ void get(float* x, const E* p, int n)
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
template <typename E> __device__ __forceinline__ void put(E* p, const float* x, int n)
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

// sum over a group of `lpg` (a power of two) neighbouring lanes, in the same order for every lane
__device__ __forceinline__ float group_sum(float x, int lpg)
{
    for (int m = 1; m < lpg; m <<= 1) x += __shfl_xor(x, m);
    return x;
}

// act and its derivative (at infinities their limits: the product with 0 is taken of a finite number)
__device__ __forceinline__ void silu(float z, int on, float& f, float& df)
{
    if (on) {
        const float s = 1.f / (1.f + expf(-z)), most = 3e38f, zc = z < -most ? -most : z > most ? most : z;
        f = (z < 0.f ? zc : z) * s;
        df = s * (1.f + zc * (1.f - s));
    } else {
        f = z;
        df = 1.f;
    }
}

// V: vectors of a lane.  A workgroup takes one head and every strips-th block of rows (b, t).
template <typename E, int V, bool BWD>
__global__ __launch_bounds__(NT) void norm_kernel(NormLaunch L, int lpg, int strips)
{
    constexpr int N = Vec<E>::N;
    __shared__ float red[BWD ? NT * N : 1];
    const int tid = threadIdx.x, gl = tid & (lpg - 1), gi = tid / lpg, groups = NT / lpg;
    const int h = blockIdx.x % L.H, strip = blockIdx.x / L.H, D = L.D;
    float w[V][N], bias[V][N], dw[V][N], db[V][N];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int ch = (gl + k * lpg) * N;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool in = ch + i < D;
            const long long at = static_cast<long long>(h) * D + (in ? ch + i : 0);
            w[k][i] = L.weight != nullptr ? L.weight[at] : 1.f;
            bias[k][i] = L.bias != nullptr ? L.bias[at] : 0.f;
            if (!in) w[k][i] = bias[k][i] = 0.f;
            dw[k][i] = db[k][i] = 0.f;
        }
    }
    const long long rows = static_cast<long long>(L.B) * L.T;
    const float inv = 1.f / D;
    for (long long r0 = static_cast<long long>(strip) * groups; r0 < rows; r0 += static_cast<long long>(strips) * groups) {
        const long long row = r0 + gi;
        const bool there = row < rows;
        const long long rr = there ? row : rows - 1;        // (a group without a row repeats the last one and writes nothing)
        const long long b = rr / L.T, t = rr - b * L.T;
        const E* xp = static_cast<const E*>(L.x) + b * L.x_s[0] + h * L.x_s[1] + t * L.x_s[2];
        const long long hc = static_cast<long long>(h) * D;
        float x[V][N], z[V][N], dy[V][N];
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int ch = (gl + k * lpg) * N, n = D - ch;
            if (n > 0) {
                get<E>(x[k], xp + ch, n);
                if (L.gate != nullptr) get<E>(z[k], static_cast<const E*>(L.gate) + b * L.g_s[0] + t * L.g_s[1] + hc + ch, n);
                if (BWD) get<E>(dy[k], static_cast<const E*>(L.dy) + b * L.y_s[0] + t * L.y_s[1] + hc + ch, n);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) x[k][i] = z[k][i] = dy[k][i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) sum += x[k][i];     // (elements past D are zero)
        }
        const float mean = group_sum(sum, lpg) * inv;
        float sq = 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = (gl + k * lpg) * N + i < D ? x[k][i] - mean : 0.f;
                x[k][i] = d;
                sq = __builtin_fmaf(d, d, sq);
            }
        const float rstd = 1.f / sqrtf(group_sum(sq, lpg) * inv + L.eps);
        if (!BWD) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int ch = (gl + k * lpg) * N, n = D - ch;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float nn = __builtin_fmaf(x[k][i] * rstd, w[k][i], bias[k][i]);
                    float f, df;
                    silu(L.gate != nullptr ? z[k][i] : nn, L.silu, f, df);
                    x[k][i] = L.gate != nullptr ? nn * f : f;
                }
                if (there && n > 0) put<E>(static_cast<E*>(L.y) + b * L.y_s[0] + t * L.y_s[1] + hc + ch, x[k], n);
            }
        } else {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float xn = x[k][i] * rstd, nn = __builtin_fmaf(xn, w[k][i], bias[k][i]);
                    float f, df, dn;
                    silu(L.gate != nullptr ? z[k][i] : nn, L.silu, f, df);
                    if (L.gate != nullptr) {
                        dn = dy[k][i] * f;
                        z[k][i] = dy[k][i] * nn * df;
                    } else {
                        dn = dy[k][i] * df;
                    }
                    if (there) {
                        dw[k][i] = __builtin_fmaf(dn, xn, dw[k][i]);
                        db[k][i] += dn;
                    }
                    const float dxn = dn * w[k][i];
                    x[k][i] = xn;
                    dy[k][i] = dxn;
                    s1 += dxn;
                    s2 = __builtin_fmaf(dxn, xn, s2);
                }
            s1 = group_sum(s1, lpg) * inv;
            s2 = group_sum(s2, lpg) * inv;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int ch = (gl + k * lpg) * N, n = D - ch;
#pragma unroll
                for (int i = 0; i < N; ++i) x[k][i] = rstd * (dy[k][i] - s1 - x[k][i] * s2);
                if (there && n > 0) {
                    put<E>(static_cast<E*>(L.dx) + b * L.dx_s[0] + h * L.dx_s[1] + t * L.dx_s[2] + ch, x[k], n);
                    if (L.gate != nullptr)
                        put<E>(static_cast<E*>(L.dgate) + b * L.dg_s[0] + t * L.dg_s[1] + hc + ch, z[k], n);
                }
            }
        }
    }
    if (BWD && L.partial != nullptr) {
        // the workgroup's sums of dw and db, groups added in order
        const long long HD = static_cast<long long>(L.H) * D;
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < N; ++i) red[(gi * lpg + gl) * N + i] = which ? db[k][i] : dw[k][i];
                __syncthreads();
                for (int e = tid; e < lpg * N; e += NT) {
                    const int ch = k * lpg * N + e;
                    if (ch >= D) continue;
                    float s = 0.f;
                    for (int j = 0; j < groups; ++j) s += red[j * lpg * N + e];
                    L.partial[(static_cast<long long>(strip) * 2 + which) * HD + static_cast<long long>(h) * D + ch] = s;
                }
            }
    }
}

// dweight and dbias: the strips' sums, added in order
__global__ __launch_bounds__(NT) void norm_join_kernel(NormLaunch L, int strips)
{
    const long long HD = static_cast<long long>(L.H) * L.D, at = static_cast<long long>(blockIdx.x) * NT + threadIdx.x;
    if (at >= 2 * HD) return;
    float* out = at < HD ? L.dweight : L.dbias;
    if (out == nullptr) return;
    float s = 0.f;
    for (int i = 0; i < strips; ++i) s += L.partial[static_cast<long long>(i) * 2 * HD + at];
    out[at < HD ? at : at - HD] = s;
}

struct Shape { int lpg, v; };
Shape shape_of(int D, bool bf16)
{
    const int N = bf16 ? 8 : 4, nv = (D + N - 1) / N;
    int lpg = 1;
    while (lpg < nv && lpg < 64) lpg *= 2;
    int v = 1;
    while (v * lpg < nv) v *= 2;
    return {lpg, v};
}

template <typename E, bool BWD> hipError_t go(const NormLaunch& L, hipStream_t st)
{
    const Shape s = shape_of(L.D, L.bf16);
    const int strips = norm_strips(static_cast<long>(L.B) * L.T, L.H, L.D, L.bf16);
    const dim3 grid(static_cast<unsigned>(strips) * static_cast<unsigned>(L.H)), block(NT);
    switch (s.v) {
        case 1: hipLaunchKernelGGL((norm_kernel<E, 1, BWD>), grid, block, 0, st, L, s.lpg, strips); break;
        case 2: hipLaunchKernelGGL((norm_kernel<E, 2, BWD>), grid, block, 0, st, L, s.lpg, strips); break;
        case 4: hipLaunchKernelGGL((norm_kernel<E, 4, BWD>), grid, block, 0, st, L, s.lpg, strips); break;
        default:        // float32 past 1024 channels
            if constexpr (Vec<E>::N == 4) hipLaunchKernelGGL((norm_kernel<E, 8, BWD>), grid, block, 0, st, L, s.lpg, strips);
            else return hipErrorInvalidValue;
    }
    hipError_t e = hipGetLastError();
    if (BWD && e == hipSuccess && L.partial != nullptr) {
        const long long n = 2LL * L.H * L.D;
        hipLaunchKernelGGL(norm_join_kernel, dim3(static_cast<unsigned>((n + NT - 1) / NT)), block, 0, st, L, strips);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

// workgroups of a head: enough for 2048 in all, each with at least 4 blocks of rows
int norm_strips(long rows_bt, int H, int D, bool bf16)
{
    const long groups = NT / shape_of(D, bf16).lpg, blocks = (rows_bt + 4 * groups - 1) / (4 * groups);
    const long want = (2048 + H - 1) / H;
    const long s = want < blocks ? want : blocks;
    return s < 1 ? 1 : static_cast<int>(s);
}

hipError_t launch_norm(const NormLaunch& L, hipStream_t st) { return L.bf16 ? go<uint16_t, false>(L, st) : go<float, false>(L, st); }
hipError_t launch_norm_bwd(const NormLaunch& L, hipStream_t st) { return L.bf16 ? go<uint16_t, true>(L, st) : go<float, true>(L, st); }

}  // namespace sfda
