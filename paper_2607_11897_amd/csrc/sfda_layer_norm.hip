// Layer norm with the residual sum before it (gfx950), forward and backward.
//   t = x + r (rounded to the type: the stream goes on as t),  x^ = (t - mean) / sqrt(var + eps) over the D channels,  y = x^ w + b
//   dx = (g - mean(g) - x^ mean(g x^)) / sqrt(var + eps) + dt,  g = dy w;   dw = sum dy x^,  db = sum dy over the rows.
// Memory-bound.  The lanes of a row hold it in registers (two-pass variance, float32): up to a wave of them by lane moves alone, more
// waves through LDS.  A workgroup keeps its lanes' weights, and in the backward their gradients, in registers over its strip of rows;
// the next row's vectors are requested before a row's arithmetic.  bfloat16, B8 T4096 of 2048 channels: with the residual sum 112 us, 4.8 TB/s, a
// large copy's rate; the backward with dtotal 128 us, 4.2 TB/s, 7 of it the join.
#include "sfda_layer.h"
#include "sfda_rows.h"
#include "sfda_vec.h"

namespace sfda {
namespace {

using namespace rows;
using namespace vec;

constexpr int FEW = 256, MANY = 1024;       // threads of a workgroup: as many as keep the row's vectors in registers

// sum over the `lpr` (a power of two) neighbouring threads of a row, the same for each of them
__device__ __forceinline__ float row_sum(float x, int lpr, float* red)
{
    x = group_sum(x, lpr < 64 ? lpr : 64);
    if (lpr <= 64) return x;
    const int w = threadIdx.x >> 6, per = lpr >> 6, w0 = w & ~(per - 1);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[w] = x;
    __syncthreads();
    x = 0.f;
    for (int i = 0; i < per; ++i) x += red[w0 + i];
    return x;
}

// V: vectors of a lane
template <typename E, int NT, int V, bool BWD, bool MORE> __global__ __launch_bounds__(NT) void layer_norm_kernel(LayerNormLaunch L, int lpr)
{
    constexpr int N = Vec<E>::N;
    extern __shared__ __align__(16) float red[];
    const int tid = threadIdx.x, gl = tid & (lpr - 1), gi = tid / lpr, groups = NT / lpr, D = L.D;
    float w[V][N], bias[BWD ? 1 : V][N], dw[BWD ? V : 1][N] = {}, db[BWD ? V : 1][N] = {};
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int ch = (gl + k * lpr) * N;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool in = ch + i < D;
            w[k][i] = L.weight != nullptr ? L.weight[in ? ch + i : 0] : 1.f;
            if (!in) w[k][i] = 0.f;
            if constexpr (!BWD) {
                bias[k][i] = L.bias != nullptr ? L.bias[in ? ch + i : 0] : 0.f;
                if (!in) bias[k][i] = 0.f;
            }
        }
    }
    const long long rows = static_cast<long long>(L.B) * L.T, stride = static_cast<long long>(gridDim.x) * groups;
    const float inv = 1.f / D;
    // (b, t) of a row, moved on by `stride` rows at a time
    const long long first = static_cast<long long>(blockIdx.x) * groups + gi;
    const int step_b = static_cast<int>(stride / L.T), step_t = static_cast<int>(stride - static_cast<long long>(step_b) * L.T);
    long long b = first / L.T, t = first - b * L.T;

    u32x4 rx[V], rd[V], rr[V];
    auto fetch = [&](long long b, long long t) {
        const E* xp = static_cast<const E*>(L.x) + b * L.x_s[0] + t * L.x_s[1];
        const E* dp = BWD ? static_cast<const E*>(L.dy) + b * L.dy_s[0] + t * L.dy_s[1] : nullptr;
        const E* rp = !MORE ? nullptr : BWD ? static_cast<const E*>(L.dtotal) + b * L.dt_s[0] + t * L.dt_s[1]
                                            : static_cast<const E*>(L.residual) + b * L.r_s[0] + t * L.r_s[1];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int ch = (gl + k * lpr) * N, n = D - ch;
            if (n > 0) {
                rx[k] = load<E>(xp + ch, n);
                if (BWD) rd[k] = load<E>(dp + ch, n);
                if (MORE) rr[k] = load<E>(rp + ch, n);
            }
        }
    };
    const u32x4 none = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < V; ++k) rx[k] = rd[k] = rr[k] = none;       // (lanes past D keep zeros)
    if (first < rows) fetch(b, t);
    // every group of the workgroup makes the same number of turns; one past the last row writes nothing
    for (long long r = static_cast<long long>(blockIdx.x) * groups; r < rows; r += stride) {
        const bool there = r + gi < rows;
        float x[V][N], dy[BWD ? V : 1][N], more[MORE ? V : 1][N];
        const long long tb = b, tt = t;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            unpack<E>(x[k], rx[k]);
            if constexpr (BWD) unpack<E>(dy[k], rd[k]);
            if constexpr (MORE) unpack<E>(more[k], rr[k]);
        }
        b += step_b;
        t += step_t;
        if (t >= L.T) {
            t -= L.T;
            ++b;
        }
        if (r + stride + gi < rows) fetch(b, t);
        if constexpr (MORE && !BWD) {
            E* tp = static_cast<E*>(L.total) + tb * L.t_s[0] + tt * L.t_s[1];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int ch = (gl + k * lpr) * N, n = D - ch;
#pragma unroll
                for (int i = 0; i < N; ++i) x[k][i] += more[k][i];
                const u32x4 sum = pack<E>(x[k]);
                if (there && n > 0) store<E>(tp + ch, sum, n);
                unpack<E>(x[k], sum);
            }
        }
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) sum += x[k][i];     // (elements past D are zero)
        const float mean = row_sum(sum, lpr, red) * inv;
        float sq = 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = (gl + k * lpr) * N + i < D ? x[k][i] - mean : 0.f;
                x[k][i] = d;
                sq = __builtin_fmaf(d, d, sq);
            }
        float rstd = inverse_root(row_sum(sq, lpr, red) * inv + L.eps);
        if constexpr (!BWD) {
            E* yp = static_cast<E*>(L.y) + tb * L.y_s[0] + tt * L.y_s[1];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int ch = (gl + k * lpr) * N, n = D - ch;
#pragma unroll
                for (int i = 0; i < N; ++i) x[k][i] = __builtin_fmaf(x[k][i] * rstd, w[k][i], bias[k][i]);
                if (there && n > 0) store<E>(yp + ch, pack<E>(x[k]), n);
            }
        } else {
            // (a group past the last row may hold none at all: with eps = 0 its x^ would be 0 * inf, which no factor 0 of dw takes back)
            if (!there) rstd = 0.f;
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float xn = x[k][i] * rstd, d = there ? dy[k][i] : 0.f;
                    dw[k][i] = __builtin_fmaf(d, xn, dw[k][i]);
                    db[k][i] += d;
                    const float gg = d * w[k][i];
                    x[k][i] = xn;
                    dy[k][i] = gg;
                    s1 += gg;
                    s2 = __builtin_fmaf(gg, xn, s2);
                }
            s1 = row_sum(s1, lpr, red) * inv;
            s2 = row_sum(s2, lpr, red) * inv;
            E* dxp = static_cast<E*>(L.dx) + tb * L.dx_s[0] + tt * L.dx_s[1];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int ch = (gl + k * lpr) * N, n = D - ch;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    x[k][i] = rstd * (dy[k][i] - s1 - x[k][i] * s2);
                    if constexpr (MORE) x[k][i] += more[k][i];
                }
                if (there && n > 0) store<E>(dxp + ch, pack<E>(x[k]), n);
            }
        }
    }
    if constexpr (BWD) {
        if (L.partial == nullptr) return;
        // the workgroup's sums of dw and db, groups added in order
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < N; ++i) red[tid * N + i] = which ? db[k][i] : dw[k][i];
                __syncthreads();
                for (int e = tid; e < lpr * N; e += NT) {
                    const int ch = k * lpr * N + e;
                    if (ch >= D) continue;
                    float s = 0.f;
                    for (int j = 0; j < groups; ++j) s += red[j * lpr * N + e];
                    L.partial[(static_cast<long long>(blockIdx.x) * 2 + which) * D + ch] = s;
                }
            }
    }
}

// dweight and dbias: the workgroups' sums.  16 threads for a channel take every 16th part, and their sums are added in order.
constexpr int JOIN_NT = 256, JOIN_PARTS = 16, JOIN_CH = JOIN_NT / JOIN_PARTS;
__global__ __launch_bounds__(JOIN_NT) void layer_norm_join_kernel(LayerNormLaunch L, int strips)
{
    __shared__ float part[JOIN_PARTS][JOIN_CH + 1];
    const int c = threadIdx.x % JOIN_CH, p = threadIdx.x / JOIN_CH;
    const long long at = static_cast<long long>(blockIdx.x) * JOIN_CH + c, size = 2LL * L.D;
    float s = 0.f;
    if (at < size) {
#pragma unroll 4
        for (int i = p; i < strips; i += JOIN_PARTS) s += L.partial[i * size + at];
    }
    part[p][c] = s;
    __syncthreads();
    if (p == 0 && at < size) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < JOIN_PARTS; ++i) s += part[i][c];
        float* out = at < L.D ? L.dweight : L.dbias;
        if (out != nullptr) out[at < L.D ? at : at - L.D] = s;
    }
}

// Vectors of a lane, then lanes, then vectors.  The backward starts with two: in bfloat16 four take 256 registers and leave a SIMD one
// wave, and in float32 one has too few loads on their way.  One / two / four, us: bfloat16 with dtotal, 32768 rows of 2048 130 / 131 / 153,
// 16384 of 4096 141 / 141 / 180, 32768 of 1024 68 / 66 / 66; float32, 32768 rows of 1024 without dtotal 104 / 93 / 91, with it 115 / 119 / 113,
// 32768 of 512 57 / 55 / 55.  Past 8192 channels 1024 threads have 128 registers each, too few for the backward, which spills (144
// bytes a lane in bfloat16, 284 in float32): 4096 rows of 12288 with dtotal 304 and 560 us, where a copy takes 83 and 165.
struct Shape { int lpr, v, nt; };
Shape shape_of(int D, bool bf16, bool bwd)
{
    const int N = bf16 ? 8 : 4, nv = (D + N - 1) / N;
    int lpr = 1;
    while (lpr < nv && lpr < 64) lpr *= 2;
    int v = 1;
    while (v * lpr < nv && v < (bwd ? 2 : 4)) v *= 2;
    while (v * lpr < nv && lpr < FEW) lpr *= 2;
    while (v * lpr < nv && v < 4) v *= 2;
    if (v * lpr >= nv) return {lpr, v, FEW};
    for (lpr = MANY, v = 1; v * lpr < nv;) v *= 2;
    return {lpr, v, MANY};
}

template <typename E, bool BWD, bool MORE> hipError_t go(const LayerNormLaunch& L, hipStream_t st)
{
    const Shape s = shape_of(L.D, L.bf16, BWD);
    const int strips = layer_norm_strips(static_cast<long long>(L.B) * L.T, L.D, L.bf16, BWD);
    const dim3 grid(strips), block(s.nt);
    const size_t lds = BWD ? sizeof(float) * s.nt * Vec<E>::N : sizeof(float) * (MANY / 64);
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, lds, st, L, s.lpr); };
    if (s.nt == FEW) {
        if (s.v == 1) run(layer_norm_kernel<E, FEW, 1, BWD, MORE>);
        else if (s.v == 2) run(layer_norm_kernel<E, FEW, 2, BWD, MORE>);
        else run(layer_norm_kernel<E, FEW, 4, BWD, MORE>);
    } else if (s.v <= 2) {
        run(layer_norm_kernel<E, MANY, 2, BWD, MORE>);
    } else {
        if constexpr (Vec<E>::N == 4) run(layer_norm_kernel<E, MANY, 4, BWD, MORE>);       // float32 past 8192 channels
        else return hipErrorInvalidValue;
    }
    hipError_t e = hipGetLastError();
    if (BWD && e == hipSuccess && L.partial != nullptr) {
        hipLaunchKernelGGL(layer_norm_join_kernel, dim3((2 * L.D + JOIN_CH - 1) / JOIN_CH), dim3(JOIN_NT), 0, st, L, strips);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int layer_norm_strips(long long rows, int D, bool bf16, bool bwd)
{
    const Shape s = shape_of(D, bf16, bwd);
    const long long groups = s.nt / s.lpr, blocks = (rows + groups - 1) / groups, most = 1024 * FEW / s.nt;
    return static_cast<int>(blocks < 1 ? 1 : blocks < most ? blocks : most);
}

hipError_t launch_layer_norm(const LayerNormLaunch& L, hipStream_t st)
{
    if (L.bf16) return L.residual != nullptr ? go<uint16_t, false, true>(L, st) : go<uint16_t, false, false>(L, st);
    return L.residual != nullptr ? go<float, false, true>(L, st) : go<float, false, false>(L, st);
}
hipError_t launch_layer_norm_bwd(const LayerNormLaunch& L, hipStream_t st)
{
    if (L.bf16) return L.dtotal != nullptr ? go<uint16_t, true, true>(L, st) : go<uint16_t, true, false>(L, st);
    return L.dtotal != nullptr ? go<float, true, true>(L, st) : go<float, true, false>(L, st);
}

}  // namespace sfda
