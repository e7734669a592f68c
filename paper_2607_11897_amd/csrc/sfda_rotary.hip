// Rotary positions (gfx950): pairs of channels (a, b) of a token at position p turned by the angle of
// their row of the tables, (a c - b s, a s + b c) with c, s = cos, sin[p, i]; the inverse turn is the gradient.
// Memory-bound: every element read and written once, the tables from the caches.  Lanes run along the memory: over a row's
// units, then over the inner one of the heads and tokens; a thread takes IPT rows of the outer one, their
// loads before their arithmetic.  bfloat16 q and k of B8 H16 T4096 d 128: 106 us, 5.1 TB/s (a large copy: 4.8); one token of 32 x 16
// rows: 4 us, a launch's.
#include "sfda_layer.h"
#include "sfda_vec.h"

namespace sfda {
namespace {

using namespace vec;

constexpr int NT = 256;
constexpr int IPT = 4;      // rows of a thread

struct RotarySide {
    const void* x;
    void* y;
    long long x_s[3], y_s[3];
    int H, inner, outer_groups;         // inner: rows along the inner axis
    unsigned threads;
};

// A unit of a row.  INTER: N channels, of which those below `rot` are turned in pairs (2i, 2i + 1).
// Halves: N pairs (i, i + rot / 2), or, past the pairs' units, N channels that pass through.
// HIN: heads are the inner axis and a thread's rows are tokens; else the other way round (and its rows share their angles).
template <typename E, bool INTER, bool HIN>
__device__ __forceinline__ void turn(const RotaryLaunch& L, const RotarySide& S, unsigned id, unsigned units)
{
    constexpr int N = Vec<E>::N, PAIRS = INTER ? N / 2 : N;
    const unsigned rest = id / units, u = id - rest * units;
    const unsigned rest2 = rest / static_cast<unsigned>(S.inner), in = rest - rest2 * static_cast<unsigned>(S.inner);
    const unsigned b = rest2 / static_cast<unsigned>(S.outer_groups), og = rest2 - b * static_cast<unsigned>(S.outer_groups);
    const int outer = HIN ? L.T : S.H;

    const int half = L.rot / 2, pair_units = (half + N - 1) / N;
    const bool through = INTER ? static_cast<int>(u) * N >= L.rot : static_cast<int>(u) >= pair_units;
    const int ch = INTER ? u * N : through ? L.rot + (static_cast<int>(u) - pair_units) * N : static_cast<int>(u) * N;
    const int n = INTER || through ? L.D - ch : half - ch;      // channels from ch on (halves: pairs)
    const int first = INTER ? ch / 2 : ch;                      // pair
    const bool pairs = !through;

    u32x4 xa[IPT], xb[IPT];
    const E* src[IPT];
    E* dst[IPT];
    int tok[IPT];
    bool live[IPT];
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
        const int o = static_cast<int>(og) * IPT + i;
        live[i] = o < outer;
        const long long h = HIN ? static_cast<long long>(in) : o, t = HIN ? o : static_cast<long long>(in);
        tok[i] = static_cast<int>(t);
        src[i] = static_cast<const E*>(S.x) + b * S.x_s[0] + h * S.x_s[1] + t * S.x_s[2] + ch;
        dst[i] = static_cast<E*>(S.y) + b * S.y_s[0] + h * S.y_s[1] + t * S.y_s[2] + ch;
        if (live[i]) {
            xa[i] = load<E>(src[i], n);
            if (!INTER && pairs) xb[i] = load<E>(src[i] + half, n);
        }
    }
    float c[PAIRS], s[PAIRS];
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
        if (!live[i]) break;
        if (pairs) {
            if (HIN || i == 0) {
                long long pos = L.offset + tok[i];
                if (L.positions != nullptr) {
                    const long long at = b * L.pos_b + tok[i];
                    pos = L.pos64 ? static_cast<const long long*>(L.positions)[at] : static_cast<const int*>(L.positions)[at];
                }
                const bool there = pos >= 0 && pos < L.P;       // a position without a row of the tables gives NaN
                const float *cp = L.cos + (there ? pos * half : 0) + first, *sp = L.sin + (there ? pos * half : 0) + first;
#pragma unroll
                for (int v = 0; v < PAIRS; v += 4) {
                    if (first + v + 4 <= half) {
                        const u32x4 cv = load16(cp + v), sv = load16(sp + v);
#pragma unroll
                        for (int e = 0; e < 4 && v + e < PAIRS; ++e) {
                            c[v + e] = __uint_as_float(cv[e]);
                            s[v + e] = __uint_as_float(sv[e]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4 && v + e < PAIRS; ++e) {
                            const bool is = first + v + e < half;
                            c[v + e] = is ? cp[v + e] : 0.f;
                            s[v + e] = is ? sp[v + e] : 0.f;
                        }
                    }
                }
#pragma unroll
                for (int p = 0; p < PAIRS; ++p) {
                    s[p] = L.inverse ? -s[p] : s[p];
                    if (!there) c[p] = s[p] = __builtin_nanf("");
                }
            }
            float x[N];
            unpack<E>(x, xa[i]);
            if constexpr (INTER) {
#pragma unroll
                for (int p = 0; p < N / 2; ++p) {
                    const float a = x[2 * p], d = x[2 * p + 1];
                    // (a pair past the rotated ones passes as it is, infinities too)
                    if (ch + 2 * p < L.rot) {
                        x[2 * p] = a * c[p] - d * s[p];
                        x[2 * p + 1] = a * s[p] + d * c[p];
                    }
                }
            } else {
                float y[N];
                unpack<E>(y, xb[i]);
#pragma unroll
                for (int p = 0; p < N; ++p) {
                    const float a = x[p], d = y[p];
                    x[p] = a * c[p] - d * s[p];
                    y[p] = a * s[p] + d * c[p];
                }
                store<E>(dst[i] + half, pack<E>(y), n);
            }
            xa[i] = pack<E>(x);
        }
        store<E>(dst[i], xa[i], n);
    }
}

// (queries first, then keys; each may have either order of axes)
template <typename E, bool INTER>
__global__ __launch_bounds__(NT) void rotary_kernel(RotaryLaunch L, RotarySide Q, RotarySide K, unsigned units, int q_heads_in, int k_heads_in)
{
    const unsigned blocks = (Q.threads + NT - 1) / NT;
    if (blockIdx.x < blocks) {
        const unsigned id = blockIdx.x * NT + threadIdx.x;
        if (id >= Q.threads) return;
        if (q_heads_in) turn<E, INTER, true>(L, Q, id, units);
        else turn<E, INTER, false>(L, Q, id, units);
    } else {
        const unsigned id = (blockIdx.x - blocks) * NT + threadIdx.x;
        if (id >= K.threads) return;
        if (k_heads_in) turn<E, INTER, true>(L, K, id, units);
        else turn<E, INTER, false>(L, K, id, units);
    }
}

RotarySide side(const RotaryLaunch& L, const void* x, void* y, const long long (&xs)[3], const long long (&ys)[3], int H, unsigned units, bool& heads_in)
{
    RotarySide s{};
    s.x = x;
    s.y = y;
    for (int i = 0; i < 3; ++i) {
        s.x_s[i] = xs[i];
        s.y_s[i] = ys[i];
    }
    s.H = H;
    // heads inside where they are closer than the tokens, and where there is but one token (a decode step)
    heads_in = L.T == 1 ? false : xs[1] < xs[2] && H > 1;
    const int outer = heads_in ? L.T : H;
    s.inner = heads_in ? H : L.T;
    s.outer_groups = (outer + IPT - 1) / IPT;
    s.threads = static_cast<unsigned>(static_cast<long long>(L.B) * s.outer_groups * s.inner * units);
    return s;
}

}  // namespace

hipError_t launch_rotary(const RotaryLaunch& L, hipStream_t st)
{
    const int N = L.bf16 ? 8 : 4;
    const unsigned units = L.interleaved ? (L.D + N - 1) / N : (L.rot / 2 + N - 1) / N + (L.D - L.rot + N - 1) / N;
    bool qin = false, kin = false;
    const RotarySide Q = side(L, L.q, L.qo, L.q_s, L.qo_s, L.Hq, units, qin), K = side(L, L.k, L.ko, L.k_s, L.ko_s, L.Hk, units, kin);
    const unsigned blocks = (Q.threads + NT - 1) / NT + (K.threads + NT - 1) / NT;
    const dim3 grid(blocks), block(NT);
    if (L.bf16) {
        if (L.interleaved) hipLaunchKernelGGL((rotary_kernel<uint16_t, true>), grid, block, 0, st, L, Q, K, units, qin, kin);
        else hipLaunchKernelGGL((rotary_kernel<uint16_t, false>), grid, block, 0, st, L, Q, K, units, qin, kin);
    } else {
        if (L.interleaved) hipLaunchKernelGGL((rotary_kernel<float, true>), grid, block, 0, st, L, Q, K, units, qin, kin);
        else hipLaunchKernelGGL((rotary_kernel<float, false>), grid, block, 0, st, L, Q, K, units, qin, kin);
    }
    return hipGetLastError();
}

}  // namespace sfda
