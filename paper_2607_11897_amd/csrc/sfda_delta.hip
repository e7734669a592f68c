// Linear attention with the gated delta rule (gfx950): the blocks' inverses, the chunked forward and the decode step.
#include "sfda_delta.h"

#include <utility>

namespace sfda {
namespace delta {
namespace {

// ------------------------------------------------------------------ the blocks' inverses

// 8 channels of a row as a fragment; channels past the row and rows that are not there are zero
template <typename E> __device__ __forceinline__ u32x4 vector_at(const char* row, int col, int cols, bool there)
{
    constexpr int VE = Ops<E>::VE;
    const u32x4 none = {0, 0, 0, 0};
    if (cols < VE) {
        const u32x4 x = short_row<E>(row, cols);
        return there && col == 0 ? x : none;
    }
    const int past = col + VE - cols;
    const u32x4 x = load16(row + (past <= 0 ? col : cols - VE) * static_cast<int>(sizeof(E)));
    return !there || past >= VE ? none : past > 0 ? move_down<E>(x, past) : x;
}
template <typename E> __device__ __forceinline__ Op<Block<E>::P> key_frag(const char* row, int col, int cols, bool there)
{
    Op<Block<E>::P> o;
    if constexpr (sizeof(E) == 2) {
        o.p[0] = __builtin_bit_cast(bf16x8, vector_at<E>(row, col, cols, there));
    } else {
        float x[8];
        const u32x4 a = vector_at<E>(row, col, cols, there), b = vector_at<E>(row, col + 4, cols, there);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = __uint_as_float(a[i]);
            x[4 + i] = __uint_as_float(b[i]);
        }
        o = op_of<3>(x);
    }
    return o;
}

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// N = (I - X)^(-1) = I + X N for X strictly lower triangular, by forward substitution: lane (c, g) holds row c of X and columns 4 g + k of
// row c of N; a pivot row is lane s of the lane's own 16.
template <int S> __device__ __forceinline__ void pivot(float (&n)[4], const float (&x)[16])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) n[k] = __builtin_fmaf(x[S], row_bcast<S>(n[k]), n[k]);
}
template <int... S> __device__ __forceinline__ void pivots(float (&n)[4], const float (&x)[16], std::integer_sequence<int, S...>)
{
    (pivot<S>(n, x), ...);
}
// d += A B, 16 x 16 in float32: a holds row c of A, b column c of B, each at 4 g + r
__device__ __forceinline__ void mul16(f32x4& d, const f32x4& a, const f32x4& b)
{
#pragma unroll
    for (int r = 0; r < 4; ++r) d = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], d, 0, 0, 0);
}

constexpr int tile_at(int i, int j) { return i * (i + 1) / 2 + j; }

// What a block's scan needs apart from the state, one wave for a block and one of
//   0  (I + L diag(beta))^(-1), and the tokens' factors     1  c D . Q K^T diag(beta)
//   2  the transpose of (I + diag(beta) L)^(-1)              3  that of c D . Q K^T
// (0 and 1 for the forward scan, 2 and 3 for the adjoint one).  Inverses: diagonal tiles by substitution, then pairs of them joined,
// [A 0; X B]^(-1) having -B^(-1) X A^(-1) in its corner, all in float32 (on its matrix instructions), where the states' 24 bits
// come from.  The results go out as the bfloat16 parts that the scans multiply, tile by tile.  Bound by latencies: the rows' loads are
// all on their way first, and nothing waits for another wave.  128 registers, so that a SIMD has four waves: bfloat16, 8192 blocks of 64
// tokens and 128 channels 134 us for the forward's two kinds (155 with three waves), 250 for all four.
template <typename E, int DKP> __global__ __launch_bounds__(NT, 4) void sfda_delta_prep(DeltaLaunch L, unsigned units, int kinds)
{
    typedef Block<E> B;
    constexpr int C = B::C, CT = B::CT, P = B::P, TILES = B::TILES, ES = sizeof(E), ROW = 20;
    constexpr int AHEAD = 2;                // times 32 channels loaded at a time
    __shared__ __align__(16) float scratch[NW][16 * ROW];
    __shared__ __align__(16) float tok[NW][3][C];

    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int groups = (L.blocks + NW - 1) / NW;
    // what is formed of the same blocks runs on one XCD, whose L2 has their rows
    const unsigned eights = blockIdx.x / 8u, kind = eights % static_cast<unsigned>(kinds), unit = eights / static_cast<unsigned>(kinds) * 8u + blockIdx.x % 8u;
    if (unit >= units) return;
    const unsigned head = unit / static_cast<unsigned>(groups), first = (unit - head * groups) * NW;
    const long long bh = L.first + head;
    const int b = static_cast<int>(bh / L.H), h = static_cast<int>(bh - static_cast<long long>(b) * L.H), hk = h / (L.H / L.Hk);
    const int len = __builtin_amdgcn_readfirstlane(seq_length(L.lengths, b, L.T)), blocks = (len + C - 1) / C, blk = first + w;
    if (blk >= blocks) return;              // (no barriers below)
    const int what = static_cast<int>(kind), t0 = blk * C, cnt = len - t0 < C ? len - t0 : C;
    const bool by_row = what >= 2, inverse = (what & 1) == 0;
    float* const buf = scratch[w];

    // 8 channels of 16 tokens' rows for a lane, both operands of all tiles; a: rows of the first operand
    const char* const kp = static_cast<const char*>(L.k) + (b * L.k_s[0] + hk * L.k_s[1] + t0 * L.k_s[2]) * ES;
    const char* const qp = static_cast<const char*>(L.q) + (b * L.q_s[0] + hk * L.q_s[1] + t0 * L.q_s[2]) * ES;
    const uint32_t kst = static_cast<uint32_t>(L.k_s[2] * ES), qst = static_cast<uint32_t>(L.q_s[2] * ES);
    Op<P> kf[AHEAD][CT], qf[AHEAD][CT];
    auto fetch = [&](int f0) {
#pragma unroll
        for (int f = 0; f < AHEAD; ++f)
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const int r = 16 * t + c, rr = r < cnt ? r : cnt - 1;
                kf[f][t] = key_frag<E>(kp + static_cast<uint64_t>(rr * kst), 32 * (f0 + f) + 8 * g, L.dk, r < cnt);
                if (!inverse) qf[f][t] = key_frag<E>(qp + static_cast<uint64_t>(rr * qst), 32 * (f0 + f) + 8 * g, L.dk, r < cnt);
            }
    };
    const bool there = lane < cnt;
    const int token = t0 + (there ? lane : 0);
    float a = L.log_decay[b * L.l_s[0] + h * L.l_s[1] + token * L.l_s[2]];
    const float be = L.beta[b * L.b_s[0] + h * L.b_s[1] + token * L.b_s[2]];
    fetch(0);

    {   // sums of the log decays as hi + lo; past -128 a decay is 0 in any case, and sums of such stay finite
        if (a < -128.f) a = -128.f;
        double s = there ? a : 0.f;
#pragma unroll
        for (int d = 1; d < C; d *= 2) {
            const double o = __shfl_up(s, d);
            if (lane >= d) s += o;
        }
        const float hi = static_cast<float>(s), lo = static_cast<float>(s - hi);
        const float eh = __shfl(hi, C - 1), el = __shfl(lo, C - 1), bt = there ? be : 0.f;
        if (lane < C) {
            tok[w][0][lane] = hi;
            tok[w][1][lane] = lo;
            tok[w][2][lane] = bt;
            if (what == 0) {
                // the block's decay as hi + lo: a state that lives for thousands of blocks keeps its 24 bits
                const float x = eh + el, wt = expf((eh - hi) + (el - lo));
                const bool near = x > -0.5f && x < 0.5f;
                const float m = near ? expm1f(x) : 0.f, end = near ? 1.f + m : expf(x);
                float4* to = L.scalars + 2 * ((head * static_cast<long long>(L.blocks) + blk) * C + lane);
                to[0] = float4{hi, lo, bt, expf(hi + lo)};
                to[1] = float4{wt, wt * bt, end, near ? m - (end - 1.f) : 0.f};
            }
        }
    }

    // lane (c, g) of tile (i, j): row c, columns 4 g + r; of K K^T, of Q K^T, or of K Q^T (tile (j, i))
    f32x4 X[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) X[t] = zero4();
#pragma unroll
    for (int f0 = 0; f0 < DKP / 32; f0 += AHEAD) {
        if (f0 > 0) {
            if (32 * f0 >= L.dk) break;
            fetch(f0);
        }
#pragma unroll
        for (int f = 0; f < AHEAD; ++f)
#pragma unroll
            for (int i = 0; i < PAIRS<P, P>; ++i)
#pragma unroll
                for (int ti = 0; ti < CT; ++ti)
#pragma unroll
                    for (int tj = 0; tj <= ti; ++tj) {
                        f32x4& x = X[tile_at(ti, tj)];
                        if (inverse) mm<P, P>(i, x, kf[f][tj], kf[f][ti]);
                        else if (by_row) mm<P, P>(i, x, qf[f][ti], kf[f][tj]);
                        else mm<P, P>(i, x, kf[f][tj], qf[f][ti]);
                    }
    }
    wave_sync();
    // rows of 16 to memory as parts: part s of tile t at s * TILES + t
    auto put = [&](uint16_t* to, const f32x4& x, int parts) {
        float y[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int s = 0; s < 3; ++s) {
            if (s >= parts) break;
            uint32_t p[2] = {pack2(y[0], y[1]), pack2(y[2], y[3])};
            asm("" : "+v"(p[0]), "+v"(p[1]));
            *reinterpret_cast<u32x2*>(to + s * (TILES * 256) + c * 16 + 4 * g) = u32x2{p[0], p[1]};
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] -= i & 1 ? hi_f32(p[i / 2]) : lo_f32(p[i / 2]);
        }
    };
    const long long at = (head * static_cast<long long>(L.blocks) + blk) * (3 * TILES * 256);
#pragma unroll
    for (int ti = 0; ti < CT; ++ti)
#pragma unroll
        for (int tj = 0; tj <= ti; ++tj) {
            const bool back = by_row && !inverse;           // (rows are the earlier tokens)
            const int one = 16 * (back ? tj : ti) + c, four = 16 * (back ? ti : tj) + 4 * g;
            float d[4];
            decays(d, tok[w][0], tok[w][1], one, four, back);
            const f32x4 b4 = *reinterpret_cast<const f32x4*>(&tok[w][2][four]);
            const float b1 = tok[w][2][one];
            f32x4& x = X[tile_at(ti, tj)];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (inverse) x[r] = masked(four + r < one, -x[r] * (d[r] * (by_row ? b1 : b4[r])));
                else x[r] = masked(back ? one <= four + r : four + r <= one, x[r] * (L.scale * d[r] * (back ? 1.f : b4[r])));
            }
            if (!inverse) put((back ? L.scores_back : L.scores) + at + tile_at(ti, tj) * 256, x, back ? 3 : L.score_parts);
        }
    if (!inverse) return;

    // row c at 4 g .. to column c at 4 g .., and back
    auto turn = [&](const f32x4& x) {
        f32x4 y;
        wave_sync();
        *reinterpret_cast<f32x4*>(buf + c * ROW + 4 * g) = x;
        wave_sync();
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = buf[(4 * g + r) * ROW + c];
        return y;
    };
    f32x4 rows[CT], T[TILES];               // diagonal tiles by rows; all tiles by columns
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        wave_sync();
        *reinterpret_cast<f32x4*>(buf + c * ROW + 4 * g) = X[tile_at(t, t)];
        wave_sync();
        float x[16], n[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 y = *reinterpret_cast<const f32x4*>(buf + c * ROW + 4 * i);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[4 * i + r] = y[r];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) n[k] = 4 * g + k == c ? 1.f : 0.f;
        pivots(n, x, std::make_integer_sequence<int, 15>());
        rows[t] = f32x4{n[0], n[1], n[2], n[3]};
        T[tile_at(t, t)] = turn(rows[t]);
    }
#pragma unroll
    for (int t = 0; t < CT; t += 2) {
        f32x4 m = zero4(), n = zero4();
        mul16(m, X[tile_at(t + 1, t)], T[tile_at(t, t)]);
        mul16(n, rows[t + 1], m);
        T[tile_at(t + 1, t)] = n;
    }
    if constexpr (CT == 4) {
        const f32x4 r32 = turn(T[tile_at(3, 2)]);
        f32x4 m[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                m[i][j] = zero4();
#pragma unroll
                for (int k = j; k < 2; ++k) mul16(m[i][j], X[tile_at(2 + i, k)], T[tile_at(k, j)]);
            }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            f32x4 y = zero4(), d = zero4();
            mul16(y, rows[2], m[0][j]);
            mul16(d, r32, m[0][j]);
            mul16(d, rows[3], m[1][j]);
            T[tile_at(2, j)] = y;
            T[tile_at(3, j)] = d;
        }
    }
#pragma unroll
    for (int ti = 0; ti < CT; ++ti)
#pragma unroll
        for (int tj = 0; tj <= ti; ++tj) {
            f32x4 x = T[tile_at(ti, tj)];
            if (!by_row) x = ti == tj ? rows[ti] : turn(x);
            put((by_row ? L.inv_back : L.inv) + at + tile_at(ti, tj) * 256, x, 3);
        }
}

// ------------------------------------------------------------------ the forward scan

template <typename E, int DKP, int MODE> __global__ __launch_bounds__((Scan<E, DKP, MODE>::THREADS)) void sfda_delta_fwd(DeltaLaunch L, int slices)
{
    extern __shared__ __align__(16) unsigned char smem[];
    long head;
    int sl;
    head_slice(blockIdx.x, slices, L.heads, head, sl);
    head = static_cast<long>(same_for_all(static_cast<uint64_t>(head)));
    sl = __builtin_amdgcn_readfirstlane(sl);
    Scan<E, DKP, MODE>::run(L, head, sl, blockIdx.y, smem);
}

// The states that enter the segments, S <- N + M S one after the other.  One workgroup for a head and 16 value columns, a quarter of
// the state's rows in a wave; M's rows, which do not wait for the state, are a segment ahead, and the state goes round through
// LDS.  4.7 us a segment at 128 channels: a load of M and N, two waits for LDS.  S0 is kept behind the segments' states.
template <int DKP> __global__ __launch_bounds__(NT) void sfda_delta_join(DeltaLaunch L, int columns)
{
    constexpr int DT = DKP / 16, DF = DKP / 32, DW = DT / NW;
    __shared__ float state[2][DKP][17];
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long head = blockIdx.x / static_cast<unsigned>(columns);
    const int n = 16 * static_cast<int>(blockIdx.x - head * columns) + c, dk = L.dk, dv = L.dv;
    const bool in = n < dv;
    const long long cells = static_cast<long long>(dk) * dv;
    const float* const S0 = L.S0 == nullptr ? nullptr : L.S0 + (L.first + head) * cells;
    for (int i = threadIdx.x; i < DKP * 16; i += NT) {
        const int ch = i / 16, col = n - c + i % 16;
        const bool there = S0 != nullptr && ch < dk && col < dv;
        const float x = there ? S0[ch * dv + col] : 0.f;
        state[0][ch][i % 16] = x;
        if (there) L.seg_N[((L.segments - 1) * static_cast<long long>(L.heads) + head) * cells + ch * dv + col] = x;
    }
    float m[DW][DF][8], y[DW][4];           // the wave's rows of M (tile row c, 8 channels) and of N (rows 4 g + r, column c)
    auto fetch = [&](int seg) {
        const long long at = seg * static_cast<long long>(L.heads) + head;
        const float* const M = L.seg_M + at * dk * dk;
        const float* const N = L.seg_N + at * cells;
#pragma unroll
        for (int d = 0; d < DW; ++d) {
            const int row = 16 * (w * DW + d) + c;
#pragma unroll
            for (int f = 0; f < DF; ++f) {
                const int col = 32 * f + 8 * g;
                const float* const p = M + (row < dk ? row : 0) * dk;
                if (dk % 8 == 0) {
                    const u32x4 a = load16(p + (col < dk ? col : 0)), b = load16(p + (col < dk ? col : 0) + 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) m[d][f][i] = __uint_as_float(i < 4 ? a[i % 4] : b[i % 4]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) m[d][f][i] = p[col + i < dk ? col + i : 0];
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int ch = 16 * (w * DW + d) + 4 * g + r;
                y[d][r] = N[(ch < dk ? ch : 0) * dv + (in ? n : 0)];
            }
        }
    };
    if (L.segments > 1) fetch(0);
    for (int seg = 0; seg + 1 < L.segments; ++seg) {
        __syncthreads();                    // (the state is written; the other buffer's readers are past it)
        Op<3> s[DF];
#pragma unroll
        for (int f = 0; f < DF; ++f) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = state[seg & 1][32 * f + 8 * g + i][c];     // (rows past dk are zero)
            s[f] = op_of<3>(x);
        }
        f32x4 z[DW];
#pragma unroll
        for (int d = 0; d < DW; ++d) z[d] = f32x4{y[d][0], y[d][1], y[d][2], y[d][3]};
#pragma unroll
        for (int f = 0; f < DF; ++f) {
            Op<3> a[DW];
#pragma unroll
            for (int d = 0; d < DW; ++d) a[d] = op_of<3>(m[d][f]);
#pragma unroll
            for (int i = 0; i < 6; ++i)
#pragma unroll
                for (int d = 0; d < DW; ++d) mm<3, 3>(i, z[d], a[d], s[f]);
        }
        if (seg + 2 < L.segments) fetch(seg + 1);
        float* const N = L.seg_N + (seg * static_cast<long long>(L.heads) + head) * cells;
#pragma unroll
        for (int d = 0; d < DW; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int ch = 16 * (w * DW + d) + 4 * g + r;
                state[(seg & 1) ^ 1][ch][c] = ch < dk ? z[d][r] : 0.f;
                if (in && ch < dk) N[ch * dv + n] = z[d][r];
            }
    }
}

template <typename E, int DKP> hipError_t fwd(DeltaLaunch L, hipStream_t st)
{
    typedef Scan<E, DKP, FWD> Sc;
    L.slices = (L.dv + SLICE - 1) / SLICE;
    if constexpr (Sc::PAIR) {
        if (L.segments > 1) {
            typedef Scan<E, DKP, STATES> Ss;
            const int slices = L.slices + (L.dk + SLICE - 1) / SLICE;
            hipLaunchKernelGGL((sfda_delta_fwd<E, DKP, STATES>), dim3(static_cast<unsigned>(L.heads) * slices, L.segments - 1), dim3(Ss::THREADS), Ss::BYTES, st, L, slices);
            hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            hipLaunchKernelGGL((sfda_delta_join<DKP>), dim3(static_cast<unsigned>(L.heads) * ((L.dv + 15) / 16)), dim3(NT), 0, st, L, (L.dv + 15) / 16);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    } else if (L.segments > 1) {
        return hipErrorInvalidValue;
    }
    hipLaunchKernelGGL((sfda_delta_fwd<E, DKP, FWD>), dim3(static_cast<unsigned>(L.heads) * L.slices, L.segments), dim3(Sc::THREADS), Sc::BYTES, st, L, L.slices);
    return hipGetLastError();
}
template <typename E> hipError_t fwd_any(const DeltaLaunch& L, hipStream_t st)
{
    return L.dk <= 64 ? fwd<E, 64>(L, st) : L.dk <= 128 ? fwd<E, 128>(L, st) : fwd<E, 256>(L, st);
}

// ------------------------------------------------------------------ decode step
// S <- a S + k u^T, u = beta (v - a S^T k), o = scale S^T q = scale (a S^T q + (k . q) u), the state read and written once.  One workgroup for
// a head and 16 float4 columns, whose 16 row groups hold every 16th row of the state in registers; S^T k and S^T q are added over
// them through LDS.  Memory-bound: 16384 states of 128 x 128 (2.18 GB) 445 us, 4.9 TB/s, a large copy's rate; 64 states 11 us, the host's
// call (6 on the GPU).
template <typename E, int ROWS> __global__ __launch_bounds__(NT) void sfda_delta_step(DeltaStepLaunch L, int slices)
{
    constexpr int RG = NT / 16, SW = 64;
    __shared__ __align__(16) float part[2][RG][SW + 4];
    __shared__ float kqs[RG];
    const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4;
    const long long bh = blockIdx.x / static_cast<unsigned>(slices);
    const int sl = static_cast<int>(blockIdx.x - bh * slices), n = sl * SW + 4 * cg;
    const int b = static_cast<int>(bh / L.H), h = static_cast<int>(bh - static_cast<long long>(b) * L.H), hk = h / (L.H / L.Hk);
    const E* q = static_cast<const E*>(L.q) + b * L.q_s[0] + hk * L.q_s[1];
    const E* k = static_cast<const E*>(L.k) + b * L.k_s[0] + hk * L.k_s[1];
    const E* v = static_cast<const E*>(L.v) + b * L.v_s[0] + h * L.v_s[1];
    float* S = L.S + bh * L.dk * static_cast<long long>(L.dv);
    const float g = L.log_decay[b * L.l_s[0] + h * L.l_s[1]], beta = L.beta[b * L.b_s[0] + h * L.b_s[1]];
    const int m = L.dv - n < 4 ? L.dv - n : 4;

    f32x4 s[ROWS], p = zero4(), o = zero4();
    float kd[ROWS], qd[ROWS], kq = 0.f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int d = rg + i * RG;
        const bool there = d < L.dk;
        s[i] = zero4();
        kd[i] = there ? Elem<E>::load(k, d) : 0.f;
        qd[i] = there ? Elem<E>::load(q, d) : 0.f;
        if (there && m > 0) {
            const float* row = S + static_cast<long long>(d) * L.dv + n;
            if (m == 4) {
                memcpy(&s[i], row, 16);
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < m) s[i][e] = row[e];
            }
        }
    }
    float vv[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) vv[e] = e < m ? Elem<E>::load(v, n + e) : 0.f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        kq = __builtin_fmaf(kd[i], qd[i], kq);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            p[e] = __builtin_fmaf(kd[i], s[i][e], p[e]);
            o[e] = __builtin_fmaf(qd[i], s[i][e], o[e]);
        }
    }
    *reinterpret_cast<f32x4*>(&part[0][rg][4 * cg]) = p;
    *reinterpret_cast<f32x4*>(&part[1][rg][4 * cg]) = o;
    if (cg == 0) kqs[rg] = kq;
    __syncthreads();
    p = o = zero4();
    kq = 0.f;
#pragma unroll
    for (int i = 0; i < RG; ++i) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(&part[0][i][4 * cg]), d = *reinterpret_cast<const f32x4*>(&part[1][i][4 * cg]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            p[e] += a[e];
            o[e] += d[e];
        }
        kq += kqs[i];
    }
    // the decay as hi + lo, so that a state that keeps nearly all of itself for thousands of tokens keeps its 24 bits
    const bool near = g > -0.5f && g < 0.5f;
    const float em = near ? expm1f(g) : 0.f, hi = near ? 1.f + em : expf(g), lo = near ? em - (hi - 1.f) : 0.f;
    f32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = beta * (vv[e] - __builtin_fmaf(p[e], hi, p[e] * lo));
    if (m > 0) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int d = rg + i * RG;
            if (d >= L.dk) break;
            float* row = S + static_cast<long long>(d) * L.dv + n;
#pragma unroll
            for (int e = 0; e < 4; ++e) s[i][e] = __builtin_fmaf(kd[i], u[e], __builtin_fmaf(s[i][e], hi, s[i][e] * lo));
            if (m == 4) {
                memcpy(row, &s[i], 16);
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < m) row[e] = s[i][e];
            }
        }
        if (rg == 0) {
            E* to = static_cast<E*>(L.o) + b * L.o_s[0] + h * L.o_s[1] + n;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < m) Ops<E>::store1(to + e, L.scale * __builtin_fmaf(kq, u[e], __builtin_fmaf(o[e], hi, o[e] * lo)));
        }
    }
}

template <typename E> hipError_t step(const DeltaStepLaunch& L, hipStream_t st)
{
    const int slices = (L.dv + 63) / 64;
    const dim3 grid(static_cast<unsigned>(L.B) * L.H * slices), block(NT);
    if (L.dk <= 64) hipLaunchKernelGGL((sfda_delta_step<E, 4>), grid, block, 0, st, L, slices);
    else if (L.dk <= 128) hipLaunchKernelGGL((sfda_delta_step<E, 8>), grid, block, 0, st, L, slices);
    else hipLaunchKernelGGL((sfda_delta_step<E, 16>), grid, block, 0, st, L, slices);
    return hipGetLastError();
}

}  // namespace

hipError_t prep(const DeltaLaunch& L, int scans, hipStream_t st)
{
    if (L.blocks == 0) return hipSuccess;
    const unsigned units = static_cast<unsigned>(L.heads) * ((L.blocks + NW - 1) / NW);
    const dim3 grid((units + 7) / 8 * 8 * (2 * scans));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(NT), 0, st, L, units, 2 * scans); };
    if (L.bf16) L.dk <= 64 ? go(sfda_delta_prep<uint16_t, 64>) : L.dk <= 128 ? go(sfda_delta_prep<uint16_t, 128>) : go(sfda_delta_prep<uint16_t, 256>);
    else L.dk <= 64 ? go(sfda_delta_prep<float, 64>) : L.dk <= 128 ? go(sfda_delta_prep<float, 128>) : go(sfda_delta_prep<float, 256>);
    return hipGetLastError();
}

}  // namespace delta

hipError_t launch_delta_fwd(const DeltaLaunch& L, hipStream_t st)
{
    const hipError_t e = delta::prep(L, 1, st);
    if (e != hipSuccess) return e;
    return L.bf16 ? delta::fwd_any<uint16_t>(L, st) : delta::fwd_any<float>(L, st);
}

hipError_t launch_delta_step(const DeltaStepLaunch& L, hipStream_t st)
{
    return L.bf16 ? delta::step<uint16_t>(L, st) : delta::step<float>(L, st);
}

}  // namespace sfda
