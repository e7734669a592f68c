// Rotary positions (gfx950): pairs of channels (a, b) of a token at position p turned by the angle of
// their row of the tables, (a c - b s, a s + b c) with c, s = cos, sin[p, i]; the inverse turn is the gradient.
// Memory-bound: every element read and written once, the tables from the caches.  Lanes run along the memory: over a row's
// units, then over the inner one of the heads and tokens; a thread takes IPT rows of the outer one, their
// loads before their arithmetic.  With several axes a pair's row is that of its axis' position: a lane reads the rows of the axes that its own
// pairs follow, most often one, and selects.  bfloat16 q and k of B8 H16 T4096 d 128: 106 us, 5.1 TB/s (a large copy: 4.8); one token of 32 x 16
// rows: 4 us, a launch's.  Three axes in runs, the same size: 112 us (141 by a loop over the axes, each waited for alone).
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

// cos and sin of a position's pairs from `first` on, zeros past them
template <int PAIRS> __device__ __forceinline__ void angles(const RotaryLaunch& L, long long pos, int first, int half, float (&c)[PAIRS], float (&s)[PAIRS])
{
    const float *cp = L.cos + pos * half + first, *sp = L.sin + pos * half + first;
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
}

// A unit of a row.  INTER: N channels, of which those below `rot` are turned in pairs (2i, 2i + 1).
// Halves: N pairs (i, i + rot / 2), or, past the pairs' units, N channels that pass through.
// HIN: heads are the inner axis and a thread's rows are tokens; else the other way round (and its rows share their angles).
template <typename E, bool INTER, bool HIN, bool AXES>
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
                bool there = true;
                if constexpr (AXES) {
                    // 2 bits for each of the lane's pairs.  The axis of its first pair is every lane's first, so that lanes with one axis, as in
                    // runs, wait for their angles once; then those of lanes that have more.
                    constexpr unsigned ALL = (1u << 2 * PAIRS) - 1;
                    const unsigned axes = L.axis[first >> 4] >> (2 * (first & 15)) & ALL;
                    unsigned left = 0x5555u & ALL;
                    if (half - first < PAIRS) left &= (1u << 2 * (half - first)) - 1;
                    auto angles_of = [&](unsigned a, unsigned mine) {
                        const long long at = a * L.pos_a + b * L.pos_b + tok[i];
                        const long long pos = L.pos64 ? static_cast<const long long*>(L.positions)[at] : static_cast<const int*>(L.positions)[at];
                        const bool ok = pos >= 0 && pos < L.P;
                        float ca[PAIRS], sa[PAIRS];
                        angles<PAIRS>(L, ok ? pos : 0, first, half, ca, sa);
#pragma unroll
                        for (int p = 0; p < PAIRS; ++p) {
                            const bool set = mine >> 2 * p & 1;
                            c[p] = set ? ok ? ca[p] : __builtin_nanf("") : c[p];
                            s[p] = set ? ok ? sa[p] : __builtin_nanf("") : s[p];
                        }
                    };
                    auto pairs_of = [&](unsigned a) {
                        const unsigned other = axes ^ (a * 0x5555u & ALL);      // (00 where a pair follows this axis)
                        return ~(other | other >> 1) & left;
                    };
#pragma unroll
                    for (int p = 0; p < PAIRS; ++p) c[p] = s[p] = 0.f;
                    const unsigned a0 = axes & 3u, mine = pairs_of(a0);
                    angles_of(a0, mine);
                    left &= ~mine;
                    for (int a = 0; a < L.axes && left != 0; ++a) {
                        const unsigned more = pairs_of(a);
                        if (more == 0) continue;
                        angles_of(a, more);
                        left &= ~more;
                    }
                } else {
                    long long pos = L.offset + tok[i];
                    if (L.positions != nullptr) {
                        const long long at = b * L.pos_b + tok[i];
                        pos = L.pos64 ? static_cast<const long long*>(L.positions)[at] : static_cast<const int*>(L.positions)[at];
                    }
                    there = pos >= 0 && pos < L.P;              // a position without a row of the tables gives NaN
                    angles<PAIRS>(L, there ? pos : 0, first, half, c, s);
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
template <typename E, bool INTER, bool AXES>
__global__ __launch_bounds__(NT) void rotary_kernel(RotaryLaunch L, RotarySide Q, RotarySide K, unsigned units, int q_heads_in, int k_heads_in)
{
    const unsigned blocks = (Q.threads + NT - 1) / NT;
    if (blockIdx.x < blocks) {
        const unsigned id = blockIdx.x * NT + threadIdx.x;
        if (id >= Q.threads) return;
        if (q_heads_in) turn<E, INTER, true, AXES>(L, Q, id, units);
        else turn<E, INTER, false, AXES>(L, Q, id, units);
    } else {
        const unsigned id = (blockIdx.x - blocks) * NT + threadIdx.x;
        if (id >= K.threads) return;
        if (k_heads_in) turn<E, INTER, true, AXES>(L, K, id, units);
        else turn<E, INTER, false, AXES>(L, K, id, units);
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
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, L, Q, K, units, qin, kin); };
    if (L.axes == 0) {
        if (L.bf16) L.interleaved ? go(rotary_kernel<uint16_t, true, false>) : go(rotary_kernel<uint16_t, false, false>);
        else L.interleaved ? go(rotary_kernel<float, true, false>) : go(rotary_kernel<float, false, false>);
    } else {
        if (L.bf16) L.interleaved ? go(rotary_kernel<uint16_t, true, true>) : go(rotary_kernel<uint16_t, false, true>);
        else L.interleaved ? go(rotary_kernel<float, true, true>) : go(rotary_kernel<float, false, true>);
    }
    return hipGetLastError();
}

}  // namespace sfda
