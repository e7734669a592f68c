// Group norm of every token's heads with an activation or an activated gate (gfx950), forward and backward.
//   x^ = (x - mean) / sqrt(var + eps) over the D channels of one head of one token,  n = x^ w + b,
//   y = act(n) without a gate, n act(z) with one;  act(z) = z or z sigmoid(z).
// Memory-bound.  A group of lanes holds a row in registers (two-pass variance, float32), a workgroup keeps
// one head's weights in registers over its strip of tokens, and in the backward their gradients too.  The next row's vectors
// are requested before a row's arithmetic, so that the reductions do not leave the memory idle.
// bfloat16 with a silu gate, B8 H16 T4096 d 128: forward 95 us (0.40 GB, 4.2 TB/s), backward 146 us (0.67 GB, 4.6 TB/s).
#include "sfda_layer.h"
#include "sfda_vec.h"

namespace sfda {
namespace {

using namespace vec;

constexpr int NT = 256;

template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, false));
}
// sum over a group of `lpg` (a power of two) neighbouring lanes, the same for every lane of it.  Within 16 lanes by data-parallel
// moves: the quad's neighbours, then mirrored halves, whose lanes already hold equal sums.
__device__ __forceinline__ float group_sum(float x, int lpg)
{
    if (lpg > 1) x += dpp<0xB1>(x);         // quad [1, 0, 3, 2]
    if (lpg > 2) x += dpp<0x4E>(x);         // quad [2, 3, 0, 1]
    if (lpg > 4) x += dpp<0x141>(x);        // half row mirrored
    if (lpg > 8) x += dpp<0x140>(x);        // row mirrored
    if (lpg > 16) x += __shfl_xor(x, 16);
    if (lpg > 32) x += __shfl_xor(x, 32);
    return x;
}

// 1 / sqrt(x), x >= 0.  The hardware's instruction takes a subnormal for 0; a variance below 2^-126 (values of 1e-19) is one, and
// with eps = 0 it counts.  The scaling takes no time that shows (bfloat16 B8 H16 T4096 d 128, in turn: forward 95.4 us and 95.0
// without, backward 147.5 and 147.6).
__device__ __forceinline__ float inverse_root(float x)
{
    const bool small = x < 0x1p-100f;
    const float r = __builtin_amdgcn_rsqf(small ? x * 0x1p64f : x);
    return small ? r * 0x1p32f : r;
}

// act and its derivative.  The sigmoid by the hardware's exponential and reciprocal (an ulp each, and |z| 2^-24 of the
// exponent's own rounding); at infinities the limits: the product with 0 is taken of a finite number.
template <bool SILU> __device__ __forceinline__ void act(float z, float& f, float& df)
{
    if constexpr (SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504089f));
        const float most = 3e38f, zc = z < -most ? -most : z > most ? most : z;
        f = (z < 0.f ? zc : z) * s;
        df = s * (1.f + zc * (1.f - s));
    } else {
        f = z;
        df = 1.f;
    }
}

// V: vectors of a lane.  A workgroup takes one head and every strips-th block of rows (b, t).
template <typename E, int V, bool BWD, bool GATE, bool SILU>
__device__ __forceinline__ void norm_rows(const NormLaunch& L, int lpg, int strips, float (&dw)[V][Vec<E>::N], float (&db)[V][Vec<E>::N])
{
    constexpr int N = Vec<E>::N;
    const int tid = threadIdx.x, gl = tid & (lpg - 1), gi = tid / lpg, groups = NT / lpg;
    const int h = blockIdx.x % L.H, strip = blockIdx.x / L.H, D = L.D;
    const long long hc = static_cast<long long>(h) * D;
    float w[V][N], bias[V][N];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int ch = (gl + k * lpg) * N;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool in = ch + i < D;
            const long long at = hc + (in ? ch + i : 0);
            w[k][i] = L.weight != nullptr ? L.weight[at] : 1.f;
            bias[k][i] = L.bias != nullptr ? L.bias[at] : 0.f;
            if (!in) w[k][i] = bias[k][i] = 0.f;
        }
    }
    const long long rows = static_cast<long long>(L.B) * L.T, stride = static_cast<long long>(strips) * groups;
    const float inv = 1.f / D;
    // (b, t) of a row, moved on by `stride` rows at a time
    const long long first = static_cast<long long>(strip) * groups + gi;
    const int step_b = static_cast<int>(stride / L.T), step_t = static_cast<int>(stride - static_cast<long long>(step_b) * L.T);
    long long b = first / L.T, t = first - b * L.T;

    u32x4 rx[V], rz[V], rd[V];
    auto fetch = [&](long long b, long long t) {
        const E* xp = static_cast<const E*>(L.x) + b * L.x_s[0] + h * L.x_s[1] + t * L.x_s[2];
        const E* zp = static_cast<const E*>(L.gate) + b * L.g_s[0] + t * L.g_s[1] + hc;
        const E* dp = static_cast<const E*>(L.dy) + b * L.y_s[0] + t * L.y_s[1] + hc;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int ch = (gl + k * lpg) * N, n = D - ch;
            if (n > 0) {
                rx[k] = load<E>(xp + ch, n);
                if (GATE) rz[k] = load<E>(zp + ch, n);
                if (BWD) rd[k] = load<E>(dp + ch, n);
            }
        }
    };
    const u32x4 none = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < V; ++k) rx[k] = rz[k] = rd[k] = none;       // (lanes past D keep zeros)
    if (first < rows) fetch(b, t);
    // every group of a wave makes the same number of turns (their sums need all lanes); one past the last row writes nothing
    for (long long r = static_cast<long long>(strip) * groups; r < rows; r += stride) {
        const bool there = r + gi < rows;
        float x[V][N], z[V][N], dy[V][N];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            unpack<E>(x[k], rx[k]);
            if (GATE) unpack<E>(z[k], rz[k]);
            if (BWD) unpack<E>(dy[k], rd[k]);
        }
        const long long tb = b, tt = t;
        b += step_b;
        t += step_t;
        if (t >= L.T) {
            t -= L.T;
            ++b;
        }
        if (r + stride + gi < rows) fetch(b, t);

        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) sum += x[k][i];     // (elements past D are zero)
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
        float rstd = inverse_root(group_sum(sq, lpg) * inv + L.eps);
        // (a group past the last row may hold none at all: with eps = 0 its x^ would be 0 * inf, which no factor 0 of dw takes back)
        if (BWD && !there) rstd = 0.f;
        if constexpr (!BWD) {
            E* yp = static_cast<E*>(L.y) + tb * L.y_s[0] + tt * L.y_s[1] + hc;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int ch = (gl + k * lpg) * N, n = D - ch;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float nn = __builtin_fmaf(x[k][i] * rstd, w[k][i], bias[k][i]);
                    float f, df;
                    act<SILU>(GATE ? z[k][i] : nn, f, df);
                    x[k][i] = GATE ? nn * f : f;
                }
                if (there && n > 0) store<E>(yp + ch, pack<E>(x[k]), n);
            }
        } else {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float xn = x[k][i] * rstd, nn = __builtin_fmaf(xn, w[k][i], bias[k][i]);
                    float f, df, dn;
                    act<SILU>(GATE ? z[k][i] : nn, f, df);
                    if (GATE) {
                        dn = dy[k][i] * f;
                        z[k][i] = dy[k][i] * nn * df;
                    } else {
                        dn = dy[k][i] * df;
                    }
                    if (!there) dn = 0.f;
                    dw[k][i] = __builtin_fmaf(dn, xn, dw[k][i]);
                    db[k][i] += dn;
                    const float dxn = dn * w[k][i];
                    x[k][i] = xn;
                    dy[k][i] = dxn;
                    s1 += dxn;
                    s2 = __builtin_fmaf(dxn, xn, s2);
                }
            s1 = group_sum(s1, lpg) * inv;
            s2 = group_sum(s2, lpg) * inv;
            E* dxp = static_cast<E*>(L.dx) + tb * L.dx_s[0] + h * L.dx_s[1] + tt * L.dx_s[2];
            E* dzp = static_cast<E*>(L.dgate) + tb * L.dg_s[0] + tt * L.dg_s[1] + hc;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int ch = (gl + k * lpg) * N, n = D - ch;
#pragma unroll
                for (int i = 0; i < N; ++i) x[k][i] = rstd * (dy[k][i] - s1 - x[k][i] * s2);
                if (there && n > 0) {
                    store<E>(dxp + ch, pack<E>(x[k]), n);
                    if (GATE) store<E>(dzp + ch, pack<E>(z[k]), n);
                }
            }
        }
    }
}

template <typename E, int V, bool BWD>
__global__ __launch_bounds__(NT) void norm_kernel(NormLaunch L, int lpg, int strips)
{
    constexpr int N = Vec<E>::N;
    float dw[V][N] = {}, db[V][N] = {};
    if (L.gate != nullptr) {
        if (L.silu) norm_rows<E, V, BWD, true, true>(L, lpg, strips, dw, db);
        else norm_rows<E, V, BWD, true, false>(L, lpg, strips, dw, db);
    } else {
        if (L.silu) norm_rows<E, V, BWD, false, true>(L, lpg, strips, dw, db);
        else norm_rows<E, V, BWD, false, false>(L, lpg, strips, dw, db);
    }
    if constexpr (BWD) {
        if (L.partial == nullptr) return;
        // the workgroup's sums of dw and db, groups added in order
        __shared__ float red[NT * N];
        const int tid = threadIdx.x, groups = NT / lpg, h = blockIdx.x % L.H, strip = blockIdx.x / L.H;
        const long long HD = static_cast<long long>(L.H) * L.D;
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < N; ++i) red[tid * N + i] = which ? db[k][i] : dw[k][i];
                __syncthreads();
                for (int e = tid; e < lpg * N; e += NT) {
                    const int ch = k * lpg * N + e;
                    if (ch >= L.D) continue;
                    float s = 0.f;
                    for (int j = 0; j < groups; ++j) s += red[j * lpg * N + e];
                    L.partial[(static_cast<long long>(strip) * 2 + which) * HD + static_cast<long long>(h) * L.D + ch] = s;
                }
            }
    }
}

// dweight and dbias: the strips' sums.  A workgroup for 64 of them at a time; its four waves take every fourth strip, and their
// parts are added in order.
constexpr long long JOIN_GROUPS = 1 << 20;      // (a launch holds less than 2^32 threads)
__global__ __launch_bounds__(NT) void norm_join_kernel(NormLaunch L, int strips)
{
    __shared__ float part[NT];
    const long long HD = static_cast<long long>(L.H) * L.D;
    for (long long base = static_cast<long long>(blockIdx.x) * 64; base < 2 * HD; base += static_cast<long long>(gridDim.x) * 64) {
        const long long at = base + (threadIdx.x & 63);
        float s = 0.f;
        if (at < 2 * HD) {
#pragma unroll 8
            for (int i = threadIdx.x >> 6; i < strips; i += 4) s += L.partial[static_cast<long long>(i) * 2 * HD + at];
        }
        part[threadIdx.x] = s;
        __syncthreads();
        if (threadIdx.x < 64 && at < 2 * HD) {
            s = part[threadIdx.x] + part[threadIdx.x + 64] + part[threadIdx.x + 128] + part[threadIdx.x + 192];
            float* out = at < HD ? L.dweight : L.dbias;
            if (out != nullptr) out[at < HD ? at : at - HD] = s;
        }
        __syncthreads();
    }
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
        const long long need = (2LL * L.H * L.D + 63) / 64;
        hipLaunchKernelGGL(norm_join_kernel, dim3(static_cast<unsigned>(need < JOIN_GROUPS ? need : JOIN_GROUPS)), block, 0, st, L, strips);
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
