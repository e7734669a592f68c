// The scan of the gated delta rule over blocks of tokens (gfx950), shared by the forward and the backward.
//
// For one head, with a_t = exp(log_decay_t):  S_t = a_t S_(t-1) + k_t (beta_t r_t)^T,  r_t = v_t - a_t S_(t-1)^T k_t,  o_t = c S_t^T q_t.
// In a block of C tokens let G_i be the sum of its log decays up to i, e_i = exp(G_i), w_i = exp(G_C - G_i), D_ij = exp(G_i - G_j) for
// j <= i, L_ij = D_ij k_i . k_j for j < i, S the state before the block and U the gradient of the state after it.  Then
//   R = (I + L diag(beta))^(-1) (V - e K S),      O = c (e Q S + P diag(beta) R),  P = D . Q K^T
//   S' = e_C S + K^T (w beta R)
// and backward, with du the gradient of the writes u_t = beta_t r_t,
//   du = (I + diag(beta) L)^(-T) (c P^T dO + w K U),   U' = e_C U + Q^T (c e dO) - K^T (e beta du).
// The inverses do not depend on the state: sfda_delta_prep forms them for all blocks at once.  What is left to be done block after
// block has the same form both ways, and is split over the value columns: a wave holds 16 columns of the state in accumulators,
// where they stay.  Every operand of the chain K S -> R -> K^T R comes out of an accumulator tile in the lane where the next product
// takes it, so that the chain needs no exchange between lanes, no LDS and no barrier; K, Q, the inverse and P are read from LDS.
//
// Lane l of a fragment has index c = l % 16 of the free axis and 8 neighbours of the contraction, for its group g = l / 16: 8 g ..
// 8 g + 7 of 32.  An accumulator tile has column c and rows 4 g .. 4 g + 3 in a lane.  So that two tiles make such a fragment, tile
// (f, h) holds the rows 32 f + 8 g + 4 h + r of channels or tokens, h = 0, 1.
#pragma once

#include "sfda_layer.h"
#include "sfda_mma.h"

#include <stddef.h>

namespace sfda {
namespace delta {

using namespace mx;

constexpr int NT = 256, NW = 4, SLICE = 16 * NW;        // threads, waves and value columns of a workgroup

// C tokens of a block: float32 operands are three planes in LDS, so that its blocks are half as long
template <typename E> struct Block {
    static constexpr int C = sizeof(E) == 2 ? 64 : 32, CT = C / 16, CF = C / 32, P = Ops<E>::PL, TILES = CT * (CT + 1) / 2;
};
static_assert(Block<uint16_t>::C == delta_block(true) && Block<float>::C == delta_block(false), "blocks");

// an operand as a sum of P bfloat16 parts
template <int P> struct Op { bf16x8 p[P]; };

template <int P> __device__ __forceinline__ Op<P> op_of(const float (&x)[8])
{
    Op<P> o;
    u32x4 w[P];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a = x[2 * e], b = x[2 * e + 1];
#pragma unroll
        for (int s = 0; s < P; ++s) {
            uint32_t p = pack2(a, b);
            asm("" : "+v"(p));          // (or the halves are converted once more, one by one)
            w[s][e] = p;
            if (s + 1 < P) {
                a -= lo_f32(p);
                b -= hi_f32(p);
            }
        }
    }
#pragma unroll
    for (int s = 0; s < P; ++s) o.p[s] = __builtin_bit_cast(bf16x8, w[s]);
    return o;
}
// of the tiles (f, 0), (f, 1)
template <int P> __device__ __forceinline__ Op<P> op_of(const f32x4& t0, const f32x4& t1)
{
    const float x[8] = {t0[0], t0[1], t0[2], t0[3], t1[0], t1[1], t1[2], t1[3]};
    return op_of<P>(x);
}
// row-major [free][contraction] in LDS: p is the lane's row and 8 neighbours
template <int P> __device__ __forceinline__ Op<P> op_rows(const uint16_t* p, int plane)
{
    Op<P> o;
#pragma unroll
    for (int s = 0; s < P; ++s) o.p[s] = plane_rows(p + s * plane);
    return o;
}
// row-major [contraction][free]: by the transposing read, which takes 4 rows of 16 from a group of lanes (lane l: row l / 4, 4
// elements) and gives lane l column l.  p: the lane's own 4 elements in row 8 g + c / 4
template <int P> __device__ __forceinline__ Op<P> op_cols(const uint16_t* p, int stride, int plane)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    Op<P> o;
#pragma unroll
    for (int s = 0; s < P; ++s) {
        u32x4 w;
        w.lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + s * plane)));
        w.hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + s * plane + 4 * stride)));
        o.p[s] = __builtin_bit_cast(bf16x8, w);
    }
    return o;
}
// the products of parts that reach 2^-22 of the whole, the small ones first; a loop over tiles inside one over these has no product
// wait for the last
template <int PA, int PB> constexpr int PAIRS = PA * PB < 9 ? PA * PB : 6;
template <int PA, int PB> __device__ __forceinline__ void mm(int i, f32x4& d, const Op<PA>& a, const Op<PB>& b)
{
    static_assert(PA == 1 || PB == 1 || (PA == 3 && PB == 3), "parts");
    if constexpr (PA == 3 && PB == 3) {
        constexpr int A[6] = {2, 0, 1, 1, 0, 0}, B[6] = {0, 2, 1, 0, 1, 0};
        mfma(d, a.p[A[i]], b.p[B[i]]);
    } else {
        mfma(d, a.p[PA > 1 ? PA - 1 - i : 0], b.p[PB > 1 ? PB - 1 - i : 0]);
    }
}

// 4 neighbours as P planes
template <int P> __device__ __forceinline__ void put_parts(uint16_t* to, int plane, const f32x4& x)
{
    float a[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int s = 0; s < P; ++s) {
        uint32_t p[2] = {pack2(a[0], a[1]), pack2(a[2], a[3])};
        asm("" : "+v"(p[0]), "+v"(p[1]));
        *reinterpret_cast<u32x2*>(to + s * plane) = u32x2{p[0], p[1]};
        if (s + 1 < P)
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] -= i & 1 ? hi_f32(p[i / 2]) : lo_f32(p[i / 2]);
    }
}
__device__ __forceinline__ int row_of(int f, int h, int c) { return 32 * f + 8 * (c >> 2) + 4 * h + (c & 3); }     // of a tile's row c

// A block's rows of one tensor on their way to LDS: C tokens x COLS channels (padded), 16-byte vectors held in registers between the
// load and the write.  The vector that would cross a row's end is moved back to end with it and into place when it is written; rows
// shorter than a vector are read by elements.  Rows past the n that are there are read as the last one and written as zeros; the
// padding's zeros in LDS are never written.
template <typename E, int COLS, int C, int STRIDE, int THREADS = NT> struct RowTile {
    static constexpr int VE = Ops<E>::VE, ES = sizeof(E), VPR = COLS / VE, RPP = THREADS / VPR, N = C / RPP, PLANE = C * STRIDE;
    static_assert(THREADS % VPR == 0 && C % RPP == 0 && N >= 1, "whole passes");
    u32x4 x[N];

    __device__ __forceinline__ void load(const char* base, uint32_t st, int n, int cols, int tid)
    {
        const int col = (tid % VPR) * VE, r0 = tid / VPR;
        if (cols < VE) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int r = r0 + u * RPP;
                x[u] = u32x4{0, 0, 0, 0};
                if (col == 0) x[u] = short_row<E>(base + static_cast<uint64_t>(r < n ? r : n - 1) * st, cols);
            }
            return;
        }
        const uint32_t at = (col + VE <= cols ? col : col >= cols ? 0 : cols - VE) * ES;
        if (n == C) {
            const uint32_t lane = r0 * st + at;
#pragma unroll
            for (int u = 0; u < N; ++u) x[u] = load16(base + static_cast<uint64_t>(u * RPP) * st + lane);
        } else {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int r = r0 + u * RPP;
                x[u] = load16(base + ((r < n ? r : n - 1) * st + at));
            }
        }
    }
    __device__ __forceinline__ void store(uint16_t* lds, int n, int cols, int tid) const
    {
        const int col = (tid % VPR) * VE, past = cols < VE ? 0 : col + VE - cols;
        if (col >= cols) return;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int r = tid / VPR + u * RPP;
            u32x4 w = r < n ? x[u] : u32x4{0, 0, 0, 0};
            if (cols % VE != 0 && past > 0) w = move_down<E>(w, past);
            Ops<E>::put(lds + r * STRIDE + col, PLANE, w);
        }
    }
};

template <typename E> __device__ __forceinline__ float value(const char* p)
{
    E x;
    memcpy(&x, p, sizeof(E));
    if constexpr (sizeof(E) == 2) return bf16_bits_to_f32(x);
    else return x;
}

// Elements [token][column] of a block in a lane: column c, tokens first(i) + 8 g, as they lie in memory (a conversion beside the load
// would wait for it).  Tokens past the n that are there are copies of the last one: their keys, queries and strengths are zero.
// base: the block's row 0; col: the lane's own (clamped) column in bytes.
template <typename E> __device__ __forceinline__ uint32_t bits(const char* p)
{
    E x;
    memcpy(&x, p, sizeof(E));
    if constexpr (sizeof(E) == 2) return x;
    else return __float_as_uint(x);
}
template <typename E> __device__ __forceinline__ float float_of(uint32_t x) { return __uint_as_float(sizeof(E) == 2 ? x << 16 : x); }
template <typename E, int COUNT, typename First>
__device__ __forceinline__ void column(uint32_t (&x)[COUNT], const char* base, uint32_t col, uint32_t st, int n, int whole, int g, First first)
{
    if (n == whole) {
        const uint32_t lane = 8 * g * st + col;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) x[i] = bits<E>(base + static_cast<uint64_t>(first(i)) * st + lane);
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int t = first(i) + 8 * g;
            x[i] = bits<E>(base + ((t < n ? t : n - 1) * st + col));
        }
    }
}

enum Mode { FWD, RECORD, ADJOINT };

template <typename E, int DKP, int MODE> struct Mem {
    typedef Block<E> B;
    static constexpr int C = B::C, P = B::P, PP = MODE == FWD ? P : 3, SK = DKP + 8, ST = C + 8;
    static constexpr int KPL = C * SK, TPL = C * ST;        // planes
    uint16_t k[P * KPL], q[P * KPL], t[3 * TPL], p[PP * TPL];
    float e[C], w[C], beta[C], gh[C], gl[C], end[4];
};

// One workgroup scans one head for 64 value columns, 16 in a wave.
template <typename E, int DKP, int MODE> __device__ __forceinline__ void scan(const DeltaLaunch& L, long head, int sl, unsigned char* smem)
{
    typedef Block<E> B;
    typedef Mem<E, DKP, MODE> M_;
    constexpr int C = B::C, CT = B::CT, CF = B::CF, P = B::P, PP = M_::PP, TILES = B::TILES, ES = sizeof(E);
    constexpr int DT = DKP / 16, DF = DKP / 32, SK = M_::SK, ST = M_::ST, KPL = M_::KPL, TPL = M_::TPL;
    constexpr bool BACK = MODE == ADJOINT;
    constexpr int OP = MODE == FWD ? P : 3;         // parts of the state and of R as operands of the outputs
    M_& M = *reinterpret_cast<M_*>(smem);

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long bh = L.first + head;
    const int b = __builtin_amdgcn_readfirstlane(static_cast<int>(bh / L.H)), h = __builtin_amdgcn_readfirstlane(static_cast<int>(bh - static_cast<long long>(b) * L.H));
    const int hk = h / (L.H / L.Hk), dk = L.dk, dv = L.dv;
    const int len = __builtin_amdgcn_readfirstlane(seq_length(L.lengths, b, L.T));
    const int blocks = (len + C - 1) / C;
    const int n0 = sl * SLICE + 16 * w, n = n0 + c;         // the wave's columns, the lane's
    const bool on = n0 < dv, in = n < dv;

    const char* const kp = static_cast<const char*>(L.k) + (b * L.k_s[0] + hk * L.k_s[1]) * ES;
    const char* const qp = static_cast<const char*>(L.q) + (b * L.q_s[0] + hk * L.q_s[1]) * ES;
    const char* const vp = static_cast<const char*>(L.v) + (b * L.v_s[0] + h * L.v_s[1]) * ES;
    const char* const gp = MODE == FWD ? nullptr : static_cast<const char*>(L.dO) + (b * L.g_s[0] + h * L.g_s[1]) * ES;
    const uint32_t kst = static_cast<uint32_t>(L.k_s[2] * ES), qst = static_cast<uint32_t>(L.q_s[2] * ES), vst = static_cast<uint32_t>(L.v_s[2] * ES);
    const uint32_t gst = MODE == FWD ? 0 : static_cast<uint32_t>(L.g_s[2] * ES);
    const uint32_t col = (in ? n : dv - 1) * ES;
    const float* const tmat = (BACK ? L.inv_back : L.inv) + head * L.blocks * static_cast<long long>(TILES * 256);
    const float4* const scal = L.scalars + head * L.blocks * static_cast<long long>(C);

    RowTile<E, DKP, C, SK> tk, tq;
    f32x4 tt[(TILES * 64 + NT - 1) / NT];
    float4 sc = {0.f, 0.f, 0.f, 0.f};
    uint32_t vr[CT * 4];                    // V, or dO
    auto fetch = [&](int blk) {
        const int t0 = blk * C, cnt = len - t0 < C ? len - t0 : C;
        tk.load(kp + static_cast<long long>(t0) * kst, kst, cnt, dk, tid);
        tq.load(qp + static_cast<long long>(t0) * qst, qst, cnt, dk, tid);
#pragma unroll
        for (int u = 0; u < (TILES * 64 + NT - 1) / NT; ++u) {
            const int at = tid + u * NT < TILES * 64 ? tid + u * NT : 0;
            tt[u] = *reinterpret_cast<const f32x4*>(tmat + static_cast<long long>(blk) * TILES * 256 + 4 * at);
        }
        if (tid < C) sc = scal[static_cast<long long>(blk) * C + tid];
        if (on) {
            if constexpr (BACK) column<E>(vr, gp + static_cast<long long>(t0) * gst, col, gst, cnt, C, g, [](int i) { return 32 * (i / 8) + i % 8; });
            else column<E>(vr, vp + static_cast<long long>(t0) * vst, col, vst, cnt, C, g, [](int i) { return 32 * (i / 8) + i % 8; });
        }
    };
    // (tile (f, h) row 4 g + r is token 32 f + 8 g + 4 h + r: the 8 neighbours of a lane are i = 4 h + r of both tiles)
    if (blocks > 0) fetch(BACK ? blocks - 1 : 0);

#ifdef SFDA_LDS_POISON
    lds_poison(&M, sizeof(M_), tid, NT);
    __syncthreads();
#endif
    {   // padding, and the tiles of the triangles that are never written, stay zero
        u32x4* z = reinterpret_cast<u32x4*>(smem);
        const u32x4 zero = {0, 0, 0, 0};
        for (int i = tid; i < static_cast<int>(offsetof(M_, e)) / 16; i += NT) z[i] = zero;
    }

    f32x4 S[DT];                            // tile 2 f + h: channels 32 f + 8 g + 4 h + r, column n
    const long long cells = static_cast<long long>(dk) * dv;
    auto channel = [&](int d, int r) { return 32 * (d / 2) + 8 * g + 4 * (d & 1) + r; };
    {
        const float* src = BACK ? L.dS_T : L.S0;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            S[d] = zero4();
            if (src != nullptr) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (in && channel(d, r) < dk) S[d][r] = src[bh * cells + static_cast<long long>(channel(d, r)) * dv + n];
            }
        }
    }
    auto record = [&](float* to) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (in && channel(d, r) < dk) to[static_cast<long long>(channel(d, r)) * dv + n] = S[d][r];
    };

#pragma clang loop unroll(disable)
    for (int it = 0; it < blocks; ++it) {
        const int blk = BACK ? blocks - 1 - it : it, t0 = blk * C, cnt = len - t0 < C ? len - t0 : C;
        __syncthreads();                    // (the last block's operands are read)
        tk.store(M.k, cnt, dk, tid);
        tq.store(M.q, cnt, dk, tid);
#pragma unroll
        for (int u = 0; u < (TILES * 64 + NT - 1) / NT; ++u) {
            const int at = tid + u * NT, tile = at >> 6, row = (at & 63) >> 2, c4 = 4 * (at & 3);
            const int ti = tile < 1 ? 0 : tile < 3 ? 1 : tile < 6 ? 2 : 3, tj = tile - ti * (ti + 1) / 2;
            if (tile < TILES) Ops<float>::put4(M.t + (16 * (BACK ? tj : ti) + row) * ST + 16 * (BACK ? ti : tj) + c4, TPL, tt[u]);
        }
        if (tid < C) {
            const float eh = __shfl(sc.x, C - 1), el = __shfl(sc.y, C - 1);
            M.gh[tid] = sc.x;
            M.gl[tid] = sc.y;
            M.beta[tid] = sc.z;
            M.e[tid] = expf(sc.x + sc.y);
            M.w[tid] = expf((eh - sc.x) + (el - sc.y));
            if (tid == 0) {
                // the block's decay as hi + lo: a state that lives for thousands of blocks keeps its 24 bits
                const float x = eh + el;
                const bool near = x > -0.5f && x < 0.5f;
                const float m = near ? expm1f(x) : 0.f, hi = near ? 1.f + m : expf(x);
                M.end[0] = hi;
                M.end[1] = near ? m - (hi - 1.f) : 0.f;
            }
        }
        __syncthreads();
        float vv[CT * 4];
#pragma unroll
        for (int i = 0; i < CT * 4; ++i) vv[i] = on ? float_of<E>(vr[i]) : 0.f;
        if (it + 1 < blocks) fetch(BACK ? blk - 1 : blk + 1);

        // P [i][j] (forward: times c beta_j), or its transpose: a tile of 16 x 16 for a wave at a time
        for (int tile = w; tile < TILES; tile += NW) {
            const int ti = tile < 1 ? 0 : tile < 3 ? 1 : tile < 6 ? 2 : 3, tj = tile - ti * (ti + 1) / 2;
            const uint16_t *pa = BACK ? M.q + (16 * ti + c) * SK : M.k + (16 * tj + c) * SK;
            const uint16_t *pb = BACK ? M.k + (16 * tj + c) * SK : M.q + (16 * ti + c) * SK;
            f32x4 s = zero4();
#pragma unroll
            for (int f = 0; f < DF; ++f) {
                const Op<P> a = op_rows<P>(pa + 32 * f + 8 * g, KPL), bb = op_rows<P>(pb + 32 * f + 8 * g, KPL);
#pragma unroll
                for (int i = 0; i < PAIRS<P, P>; ++i) mm<P, P>(i, s, a, bb);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * ti + (BACK ? 4 * g + r : c), j = 16 * tj + (BACK ? c : 4 * g + r);
                const float d = expf((M.gh[i] - M.gh[j]) + (M.gl[i] - M.gl[j]));
                s[r] = j <= i ? s[r] * (d * (BACK ? L.scale : L.scale * M.beta[j])) : 0.f;
            }
            uint16_t* to = BACK ? M.p + (16 * tj + c) * ST + 16 * ti + 4 * g : M.p + (16 * ti + c) * ST + 16 * tj + 4 * g;
            if constexpr (PP == 1) Ops<uint16_t>::put4(to, 0, s);
            else Ops<float>::put4(to, TPL, s);
        }

        f32x4 z[CT], x[BACK ? 1 : CT];
        if (on) {
            if constexpr (MODE == RECORD) record(L.rec_S + (head * (L.blocks + 1) + blk) * cells);
            if constexpr (MODE == ADJOINT) record(L.rec_U + (head * L.blocks + blk) * cells);
#pragma unroll
            for (int t = 0; t < CT; ++t) z[t] = zero4();
            if constexpr (!BACK) {
#pragma unroll
                for (int t = 0; t < CT; ++t) x[t] = zero4();
            }
            // K S (tokens x columns), and Q S (columns x tokens)
#pragma unroll
            for (int f = 0; f < DF; ++f) {
                const Op<3> s3 = op_of<3>(S[2 * f], S[2 * f + 1]);
                Op<P> kr[CT];
#pragma unroll
                for (int t = 0; t < CT; ++t) kr[t] = op_rows<P>(M.k + row_of(t / 2, t & 1, c) * SK + 32 * f + 8 * g, KPL);
#pragma unroll
                for (int i = 0; i < PAIRS<P, 3>; ++i)
#pragma unroll
                    for (int t = 0; t < CT; ++t) mm<P, 3>(i, z[t], kr[t], s3);
                if constexpr (!BACK) {
                    Op<OP> so;
#pragma unroll
                    for (int s = 0; s < OP; ++s) so.p[s] = s3.p[s];
#pragma unroll
                    for (int t = 0; t < CT; ++t) kr[t] = op_rows<P>(M.q + (16 * t + c) * SK + 32 * f + 8 * g, KPL);
#pragma unroll
                    for (int i = 0; i < PAIRS<OP, P>; ++i)
#pragma unroll
                        for (int t = 0; t < CT; ++t) mm<OP, P>(i, x[t], so, kr[t]);
                }
            }
        }
        __syncthreads();                    // (P is written)
        if (!on) continue;

        // e, w, beta of the lane's tokens
        f32x4 te[CT], tw[CT], tb[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const int at = 32 * (t / 2) + 8 * g + 4 * (t & 1);
            te[t] = *reinterpret_cast<const f32x4*>(M.e + at);
            tw[t] = *reinterpret_cast<const f32x4*>(M.w + at);
            tb[t] = *reinterpret_cast<const f32x4*>(M.beta + at);
        }
        const float ghi = M.end[0], glo = M.end[1];
        if constexpr (!BACK) {
            // R = (I + L beta)^(-1) (V - e K S)
            Op<3> zo[CF];
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) z[t][r] = vv[4 * t + r] - te[t][r] * z[t][r];
#pragma unroll
            for (int f = 0; f < CF; ++f) zo[f] = op_of<3>(z[2 * f], z[2 * f + 1]);
            f32x4 R[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                R[t] = zero4();
#pragma unroll
                for (int f = 0; f <= t / 2; ++f) {
                    const Op<3> a = op_rows<3>(M.t + row_of(t / 2, t & 1, c) * ST + 32 * f + 8 * g, TPL);
#pragma unroll
                    for (int i = 0; i < 6; ++i) mm<3, 3>(i, R[t], a, zo[f]);
                }
            }
            // the outputs, columns x tokens
            Op<OP> ro[CF];
#pragma unroll
            for (int f = 0; f < CF; ++f) ro[f] = op_of<OP>(R[2 * f], R[2 * f + 1]);
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const float et = L.scale * M.e[16 * t + c];
#pragma unroll
                for (int r = 0; r < 4; ++r) x[t][r] *= et;
#pragma unroll
                for (int f = 0; f <= t / 2; ++f) {
                    const Op<PP> p = op_rows<PP>(M.p + (16 * t + c) * ST + 32 * f + 8 * g, TPL);
#pragma unroll
                    for (int i = 0; i < PAIRS<OP, PP>; ++i) mm<OP, PP>(i, x[t], ro[f], p);
                }
            }
            if constexpr (MODE == FWD) {
                char* const op = static_cast<char*>(L.o) + (b * L.o_s[0] + h * L.o_s[1] + n0 + 4 * g) * ES;
                const int left = dv - n0 - 4 * g;
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    if (16 * t + c >= cnt) continue;
                    char* to = op + static_cast<long long>(t0 + 16 * t + c) * (L.o_s[2] * ES);
                    if (left >= 4) {
                        if constexpr (ES == 2) {
                            const u32x2 y = {pack2(x[t][0], x[t][1]), pack2(x[t][2], x[t][3])};
                            memcpy(to, &y, 8);
                        } else {
                            store16(to, __builtin_bit_cast(u32x4, x[t]));
                        }
                    } else {
#pragma unroll
                        for (int r = 0; r < 3; ++r)
                            if (r < left) Ops<E>::store1(reinterpret_cast<E*>(to) + r, x[t][r]);
                    }
                }
            } else {
                // o . dO over the wave's columns
                const int left = dv - n0 - 4 * g;
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const int tok = 16 * t + c;
                    const char* from = gp + static_cast<long long>(t0 + (tok < cnt ? tok : cnt - 1)) * gst + (n0 + 4 * g) * ES;
                    float s = 0.f;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (r < left) s = __builtin_fmaf(x[t][r], value<E>(from + r * ES), s);
                    s += __shfl_xor(s, 16);
                    s += __shfl_xor(s, 32);
                    if (g == 0 && tok < cnt) L.odo[(head * L.parts + n0 / 16) * (static_cast<long long>(L.blocks) * C) + t0 + tok] = s;
                }
#pragma unroll
                for (int t = 0; t < CT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int tok = 32 * (t / 2) + 8 * g + 4 * (t & 1) + r;
                        if (in && tok < cnt) L.rec_R[(head * (static_cast<long long>(L.blocks) * C) + t0 + tok) * dv + n] = R[t][r];
                    }
            }
            // the state: w beta R from the tokens
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) R[t][r] *= tw[t][r] * tb[t][r];
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[d][r] = __builtin_fmaf(S[d][r], ghi, S[d][r] * glo);
#pragma unroll
            for (int f = 0; f < CF; ++f) {
                const Op<3> u = op_of<3>(R[2 * f], R[2 * f + 1]);
                const uint16_t* at = M.k + (32 * f + 8 * g + (c >> 2)) * SK + 8 * (c & 3);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const Op<P> kc = op_cols<P>(at + 32 * (d / 2) + 4 * (d & 1), SK, KPL);
#pragma unroll
                    for (int i = 0; i < PAIRS<P, 3>; ++i) mm<P, 3>(i, S[d], kc, u);
                }
            }
        } else {
            // du = (I + beta L)^(-T) (c P^T dO + w K U)
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) z[t][r] *= tw[t][r];
            Op<P> go[CF];
#pragma unroll
            for (int f = 0; f < CF; ++f) {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = vv[8 * f + i];
                go[f] = op_of<P>(y);
            }
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int f = t / 2; f < CF; ++f) {
                    const Op<3> a = op_rows<3>(M.p + row_of(t / 2, t & 1, c) * ST + 32 * f + 8 * g, TPL);
#pragma unroll
                    for (int i = 0; i < PAIRS<3, P>; ++i) mm<3, P>(i, z[t], a, go[f]);
                }
            Op<3> zo[CF];
#pragma unroll
            for (int f = 0; f < CF; ++f) zo[f] = op_of<3>(z[2 * f], z[2 * f + 1]);
            f32x4 du[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                du[t] = zero4();
#pragma unroll
                for (int f = t / 2; f < CF; ++f) {
                    const Op<3> a = op_rows<3>(M.t + row_of(t / 2, t & 1, c) * ST + 32 * f + 8 * g, TPL);
#pragma unroll
                    for (int i = 0; i < 6; ++i) mm<3, 3>(i, du[t], a, zo[f]);
                }
            }
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int tok = 32 * (t / 2) + 8 * g + 4 * (t & 1) + r;
                    if (in && tok < cnt) L.rec_du[(head * (static_cast<long long>(L.blocks) * C) + t0 + tok) * dv + n] = du[t][r];
                    du[t][r] *= -te[t][r] * tb[t][r];
                    vv[4 * t + r] *= L.scale * te[t][r];
                }
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[d][r] = __builtin_fmaf(S[d][r], ghi, S[d][r] * glo);
#pragma unroll
            for (int f = 0; f < CF; ++f) {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = vv[8 * f + i];
                const Op<3> u = op_of<3>(du[2 * f], du[2 * f + 1]), o3 = op_of<3>(y);
                const int at = (32 * f + 8 * g + (c >> 2)) * SK + 8 * (c & 3);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const Op<P> kc = op_cols<P>(M.k + at + 32 * (d / 2) + 4 * (d & 1), SK, KPL);
                    const Op<P> qc = op_cols<P>(M.q + at + 32 * (d / 2) + 4 * (d & 1), SK, KPL);
#pragma unroll
                    for (int i = 0; i < PAIRS<P, 3>; ++i) {
                        mm<P, 3>(i, S[d], kc, u);
                        mm<P, 3>(i, S[d], qc, o3);
                    }
                }
            }
        }
    }

    if (on) {
        float* dst = BACK ? L.dS0 : L.S_T;
        if (dst != nullptr) record(dst + bh * cells);
        if constexpr (MODE == RECORD) record(L.rec_S + (head * (L.blocks + 1) + blocks) * cells);
    }
    if constexpr (MODE == FWD) {            // tokens past the sequence's length
        E* const op = static_cast<E*>(L.o) + b * L.o_s[0] + h * L.o_s[1] + sl * SLICE;
        if (lane < dv - sl * SLICE)
            for (long long t = len + w; t < L.T; t += NW) Ops<E>::store1(op + t * L.o_s[2] + lane, 0.f);
    }
}

// ------------------------------------------------------------------ the scan by two kinds of waves
// The same scan with eight waves: four hold the state and run the chain alone, four help.  Forward, the helpers form P and the
// outputs, a block behind the chain, from the state and R as operands that the chain's waves leave in LDS fragment by fragment (as
// the lane has them: 16 bytes a lane, no two on one bank).  Backward, they form P^T and Q^T (c e dO), which do not depend on the state.

// rows of a triangular matrix in LDS: 32 rows of a block row are as long as the block columns that they have
template <int C, bool UPPER> struct Tri {
    static constexpr int S0 = (C == 64 && UPPER ? 64 : 32) + 8, S1 = (UPPER ? 32 : 64) + 8, SIZE = 32 * S0 + (C == 64 ? 32 * S1 : 0);
    // row 32 f + r, column 0
    static __device__ __forceinline__ int at(int f, int r) { return f == 0 ? r * S0 : 32 * S0 + r * S1 - (UPPER ? 32 : 0); }
    static __device__ __forceinline__ int row(int i) { return at(i >> 5, i & 31); }
};

template <typename E, int DKP, int MODE> struct PairMem {
    typedef Block<E> B;
    static constexpr bool BACK = MODE == ADJOINT;
    // parts of the state and of R as operands of the outputs, and of P.  bfloat16 outputs: one part each leaves an error of 0.0027 of the
    // results (0.0017 their own rounding), P in two 0.0024
    static constexpr int C = B::C, P = B::P, OP = MODE == FWD ? P : 3, PP = MODE == FWD && P == 1 ? 2 : 3;
    typedef Tri<C, BACK> T;
    static constexpr int SK = DKP + 8, KPL = C * SK, TPL = T::SIZE, DF = DKP / 32, DT = DKP / 16;
    uint16_t k[P * KPL], q[P * KPL], t[3 * TPL], p[PP * TPL];
    union {
        struct { u32x4 s[NW][DF * OP][64], r[NW][B::CF * OP][64]; } fwd;        // the state and R
        f32x4 add[NW][BACK ? DT : 1][64];                                       // Q^T (c e dO)
    };
    float e[C], w[C], beta[C], gh[C], gl[C], end[4];
};

constexpr int PAIR_NT = 2 * NT;

// chain: the wave holds the state.  (Each kind of wave runs a copy of its own, with the other kind's registers free; all have the same
// barriers.)
template <typename E, int DKP, int MODE, bool chain> __device__ __forceinline__ void pair_scan(const DeltaLaunch& L, long head, int sl, unsigned char* smem)
{
    typedef Block<E> B;
    typedef PairMem<E, DKP, MODE> M_;
    typedef typename M_::T Tr;
    constexpr int C = B::C, CT = B::CT, CF = B::CF, P = B::P, PP = M_::PP, OP = M_::OP, TILES = B::TILES, ES = sizeof(E);
    constexpr int DT = DKP / 16, DF = DKP / 32, SK = M_::SK, KPL = M_::KPL, TPL = M_::TPL, NTT = (TILES * 64 + PAIR_NT - 1) / PAIR_NT;
    constexpr int NSC = (TILES + NW - 1) / NW;      // tiles of P of a helper
    constexpr bool BACK = MODE == ADJOINT;
    M_& M = *reinterpret_cast<M_*>(smem);

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int w = wave & (NW - 1);
    const long long bh = L.first + head;
    const int b = __builtin_amdgcn_readfirstlane(static_cast<int>(bh / L.H)), h = __builtin_amdgcn_readfirstlane(static_cast<int>(bh - static_cast<long long>(b) * L.H));
    const int hk = h / (L.H / L.Hk), dk = L.dk, dv = L.dv;
    const int len = __builtin_amdgcn_readfirstlane(seq_length(L.lengths, b, L.T));
    const int blocks = (len + C - 1) / C;
    const int n0 = sl * SLICE + 16 * w, n = n0 + c;         // the wave's columns, the lane's
    const bool on = n0 < dv, in = n < dv;

    const char* const kp = static_cast<const char*>(L.k) + (b * L.k_s[0] + hk * L.k_s[1]) * ES;
    const char* const qp = static_cast<const char*>(L.q) + (b * L.q_s[0] + hk * L.q_s[1]) * ES;
    const char* const vp = static_cast<const char*>(L.v) + (b * L.v_s[0] + h * L.v_s[1]) * ES;
    const char* const gp = MODE == FWD ? nullptr : static_cast<const char*>(L.dO) + (b * L.g_s[0] + h * L.g_s[1]) * ES;
    const uint32_t kst = static_cast<uint32_t>(L.k_s[2] * ES), qst = static_cast<uint32_t>(L.q_s[2] * ES), vst = static_cast<uint32_t>(L.v_s[2] * ES);
    const uint32_t gst = MODE == FWD ? 0 : static_cast<uint32_t>(L.g_s[2] * ES);
    const uint32_t col = (in ? n : dv - 1) * ES;
    const float* const tmat = (BACK ? L.inv_back : L.inv) + head * L.blocks * static_cast<long long>(TILES * 256);
    const float4* const scal = L.scalars + head * L.blocks * static_cast<long long>(C);

    RowTile<E, DKP, C, SK, PAIR_NT> tk, tq;
    f32x4 tt[NTT];
    float4 sc = {0.f, 0.f, 0.f, 0.f};
    uint32_t vr[CT * 4];                    // V, or dO
    auto fetch = [&](int blk) {
        const int t0 = blk * C, cnt = len - t0 < C ? len - t0 : C;
        tk.load(kp + static_cast<long long>(t0) * kst, kst, cnt, dk, tid);
        tq.load(qp + static_cast<long long>(t0) * qst, qst, cnt, dk, tid);
#pragma unroll
        for (int u = 0; u < NTT; ++u) {
            const int at = tid + u * PAIR_NT < TILES * 64 ? tid + u * PAIR_NT : 0;
            tt[u] = *reinterpret_cast<const f32x4*>(tmat + static_cast<long long>(blk) * TILES * 256 + 4 * at);
        }
        if (tid < C) sc = scal[static_cast<long long>(blk) * C + tid];
        if (!on) return;
        // tile (f, h) row 4 g + r is token 32 f + 8 g + 4 h + r: the 8 neighbours of a lane are i = 4 h + r of both tiles
        if constexpr (BACK) {
            column<E>(vr, gp + static_cast<long long>(t0) * gst, col, gst, cnt, C, g, [](int i) { return 32 * (i / 8) + i % 8; });
        } else if (chain) {
            column<E>(vr, vp + static_cast<long long>(t0) * vst, col, vst, cnt, C, g, [](int i) { return 32 * (i / 8) + i % 8; });
        }
    };
    if (blocks > 0) fetch(BACK ? blocks - 1 : 0);

#ifdef SFDA_LDS_POISON
    lds_poison(&M, sizeof(M_), tid, PAIR_NT);
    __syncthreads();
#endif
    {   // padding, and the tiles of the triangles that are never written, stay zero
        u32x4* z = reinterpret_cast<u32x4*>(smem);
        const u32x4 zero = {0, 0, 0, 0};
        for (int i = tid; i < static_cast<int>(offsetof(M_, fwd)) / 16; i += PAIR_NT) z[i] = zero;
    }

    f32x4 S[DT];                            // tile 2 f + h: channels 32 f + 8 g + 4 h + r, column n
    const long long cells = static_cast<long long>(dk) * dv;
    auto channel = [&](int d, int r) { return 32 * (d / 2) + 8 * g + 4 * (d & 1) + r; };
#pragma unroll
    for (int d = 0; d < DT; ++d) S[d] = zero4();
    if (chain && (BACK ? L.dS_T : L.S0) != nullptr) {
        const float* const src = (BACK ? L.dS_T : L.S0) + bh * cells;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (in && channel(d, r) < dk) S[d][r] = src[channel(d, r) * dv + n];
    }
    auto record = [&](float* to) {
        float* const at = to + (8 * g) * dv + n;
        if (dk == DKP) {
            if (in)
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) at[(32 * (d / 2) + 4 * (d & 1) + r) * dv] = S[d][r];
        } else {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (in && channel(d, r) < dk) at[(32 * (d / 2) + 4 * (d & 1) + r) * dv] = S[d][r];
        }
    };
    // P's tile `x` of the helper: row and column tile
    auto tile_row = [](int tile) { return tile < 1 ? 0 : tile < 3 ? 1 : tile < 6 ? 2 : 3; };

    Op<OP> ro[BACK ? 1 : CF];               // R, of the chain's waves
    f32x4 x[BACK ? 1 : CT], ps[NSC];        // outputs and tiles of P, of the helpers
    float et[BACK ? 1 : CT];

#pragma clang loop unroll(disable)
    for (int it = 0; it <= blocks; ++it) {
        const bool work = it < blocks;
        const int blk = BACK ? blocks - 1 - it : it, t0 = blk * C, cnt = len - t0 < C ? len - t0 : C;
        __syncthreads();                    // (the last block's operands are read)
        if (work) {
            tk.store(M.k, cnt, dk, tid);
            tq.store(M.q, cnt, dk, tid);
#pragma unroll
            for (int u = 0; u < NTT; ++u) {
                const int at = tid + u * PAIR_NT, tile = at >> 6, row = (at & 63) >> 2, c4 = 4 * (at & 3);
                const int ti = tile_row(tile), tj = tile - ti * (ti + 1) / 2;
                if (tile < TILES) put_parts<3>(M.t + Tr::row(16 * (BACK ? tj : ti) + row) + 16 * (BACK ? ti : tj) + c4, TPL, tt[u]);
            }
            if (tid < C) {
                const float eh = __shfl(sc.x, C - 1), el = __shfl(sc.y, C - 1);
                M.gh[tid] = sc.x;
                M.gl[tid] = sc.y;
                M.beta[tid] = sc.z;
                M.e[tid] = expf(sc.x + sc.y);
                M.w[tid] = expf((eh - sc.x) + (el - sc.y));
                if (tid == 0) {
                    // the block's decay as hi + lo: a state that lives for thousands of blocks keeps its 24 bits
                    const float s = eh + el;
                    const bool near = s > -0.5f && s < 0.5f;
                    const float m = near ? expm1f(s) : 0.f, hi = near ? 1.f + m : expf(s);
                    M.end[0] = hi;
                    M.end[1] = near ? m - (hi - 1.f) : 0.f;
                }
            }
        }
        Op<3> s3[DF];
        if (chain && on) {
            if constexpr (BACK) {
                if (it > 0) {
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const f32x4 y = M.add[w][d][lane];
#pragma unroll
                        for (int r = 0; r < 4; ++r) S[d][r] += y[r];
                    }
                }
            } else if (it > 0) {
#pragma unroll
                for (int f = 0; f < CF; ++f)
#pragma unroll
                    for (int s = 0; s < OP; ++s) M.fwd.r[w][f * OP + s][lane] = __builtin_bit_cast(u32x4, ro[f].p[s]);
            }
            if (work) {
#pragma unroll
                for (int f = 0; f < DF; ++f) {
                    s3[f] = op_of<3>(S[2 * f], S[2 * f + 1]);
                    if constexpr (!BACK) {
#pragma unroll
                        for (int s = 0; s < OP; ++s) M.fwd.s[w][f * OP + s][lane] = __builtin_bit_cast(u32x4, s3[f].p[s]);
                    }
                }
                if constexpr (MODE == RECORD) record(L.rec_S + (head * (L.blocks + 1) + blk) * cells);
                if constexpr (MODE == ADJOINT) record(L.rec_U + (head * L.blocks + blk) * cells);
            }
        }
        if constexpr (!BACK) {
            if (!chain && it > 0) {
#pragma unroll
                for (int i = 0; i < NSC; ++i) {
                    const int tile = w + NW * i, ti = tile_row(tile), tj = tile - ti * (ti + 1) / 2;
                    if (tile < TILES) put_parts<PP>(M.p + Tr::row(16 * ti + c) + 16 * tj + 4 * g, TPL, ps[i]);
                }
            }
        }
        if (BACK && !work) break;
        __syncthreads();
        uint32_t vv[CT * 4];
#pragma unroll
        for (int i = 0; i < CT * 4; ++i) vv[i] = vr[i];
        if (it + 1 < blocks) fetch(BACK ? blk - 1 : blk + 1);

        // tiles of P [i][j] times c beta_j, or of P^T times c
        auto scores = [&] {
#pragma unroll
            for (int x = 0; x < NSC; ++x) {
                const int tile = w + NW * x, ti = tile_row(tile), tj = tile - ti * (ti + 1) / 2;
                if (tile >= TILES) break;
                const uint16_t *pa = BACK ? M.q + (16 * ti + c) * SK : M.k + (16 * tj + c) * SK;
                const uint16_t *pb = BACK ? M.k + (16 * tj + c) * SK : M.q + (16 * ti + c) * SK;
                f32x4 s = zero4();
#pragma unroll
                for (int f = 0; f < DF; ++f) {
                    const Op<P> a = op_rows<P>(pa + 32 * f + 8 * g, KPL), bb = op_rows<P>(pb + 32 * f + 8 * g, KPL);
#pragma unroll
                    for (int i = 0; i < PAIRS<P, P>; ++i) mm<P, P>(i, s, a, bb);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * ti + (BACK ? 4 * g + r : c), j = 16 * tj + (BACK ? c : 4 * g + r);
                    const float d = expf((M.gh[i] - M.gh[j]) + (M.gl[i] - M.gl[j]));
                    s[r] = j <= i ? s[r] * (d * (BACK ? L.scale : L.scale * M.beta[j])) : 0.f;
                }
                ps[x] = s;
                if constexpr (BACK) put_parts<3>(M.p + Tr::row(16 * tj + c) + 16 * ti + 4 * g, TPL, s);
            }
        };
        // K S, tokens x columns
        f32x4 z[CT];
        auto held = [&] {
#pragma unroll
            for (int t = 0; t < CT; ++t) z[t] = zero4();
#pragma unroll
            for (int f = 0; f < DF; ++f) {
                Op<P> kr[CT];
#pragma unroll
                for (int t = 0; t < CT; ++t) kr[t] = op_rows<P>(M.k + row_of(t / 2, t & 1, c) * SK + 32 * f + 8 * g, KPL);
#pragma unroll
                for (int i = 0; i < PAIRS<P, 3>; ++i)
#pragma unroll
                    for (int t = 0; t < CT; ++t) mm<P, 3>(i, z[t], kr[t], s3[f]);
            }
        };
        // what the lane's tokens have in `from`
        auto factors = [&](const float* from, int t) { return *reinterpret_cast<const f32x4*>(from + 32 * (t / 2) + 8 * g + 4 * (t & 1)); };
        // the inverse (or its transpose) times Z
        auto solve = [&](f32x4 (&R)[CT]) {
            Op<3> zo[CF];
#pragma unroll
            for (int f = 0; f < CF; ++f) zo[f] = op_of<3>(z[2 * f], z[2 * f + 1]);
#pragma unroll
            for (int t = 0; t < CT; ++t) R[t] = zero4();
#pragma unroll
            for (int t2 = 0; t2 < CT; t2 += 2)
#pragma unroll
                for (int f = BACK ? t2 / 2 : 0; f <= (BACK ? CF - 1 : t2 / 2); ++f) {
                    Op<3> a[2];
#pragma unroll
                    for (int t = 0; t < 2; ++t) a[t] = op_rows<3>(M.t + Tr::at(t2 / 2, row_of(0, t, c)) + 32 * f + 8 * g, TPL);
#pragma unroll
                    for (int i = 0; i < 6; ++i)
#pragma unroll
                        for (int t = 0; t < 2; ++t) mm<3, 3>(i, R[t2 + t], a[t], zo[f]);
                }
        };
        // S <- e_C S + K^T y
        auto update = [&](const f32x4 (&y)[CT]) {
            const float ghi = M.end[0], glo = M.end[1];
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[d][r] = __builtin_fmaf(S[d][r], ghi, S[d][r] * glo);
#pragma unroll
            for (int f = 0; f < CF; ++f) {
                const Op<3> u = op_of<3>(y[2 * f], y[2 * f + 1]);
                const uint16_t* at = M.k + (32 * f + 8 * g + (c >> 2)) * SK + 8 * (c & 3);
#pragma unroll
                for (int d2 = 0; d2 < DT; d2 += 4) {
                    Op<P> kc[4];
#pragma unroll
                    for (int d = 0; d < 4; ++d) kc[d] = op_cols<P>(at + 32 * ((d2 + d) / 2) + 4 * (d & 1), SK, KPL);
#pragma unroll
                    for (int i = 0; i < PAIRS<P, 3>; ++i)
#pragma unroll
                        for (int d = 0; d < 4; ++d) mm<P, 3>(i, S[d2 + d], kc[d], u);
                }
            }
        };

        if constexpr (!BACK) {
            if (chain && work && on) {
                held();
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const f32x4 te = factors(M.e, t);
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[t][r] = float_of<E>(vv[4 * t + r]) - te[r] * z[t][r];
                }
                f32x4 R[CT];
                solve(R);
#pragma unroll
                for (int f = 0; f < CF; ++f) ro[f] = op_of<OP>(R[2 * f], R[2 * f + 1]);
                if constexpr (MODE == RECORD) {
#pragma unroll
                    for (int t = 0; t < CT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int tok = 32 * (t / 2) + 8 * g + 4 * (t & 1) + r;
                            if (in && tok < cnt) L.rec_R[(head * (static_cast<long long>(L.blocks) * C) + t0 + tok) * dv + n] = R[t][r];
                        }
                }
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const f32x4 tw = factors(M.w, t), tb = factors(M.beta, t);
#pragma unroll
                    for (int r = 0; r < 4; ++r) R[t][r] *= tw[r] * tb[r];
                }
                update(R);
            } else if (!chain) {
                if (it > 0 && on) {         // the block before: x += P R
                    const int tb = t0 - C, left = dv - n0 - 4 * g, last = len - tb < C ? len - tb : C;
                    Op<OP> rr[CF];
#pragma unroll
                    for (int f = 0; f < CF; ++f)
#pragma unroll
                        for (int s = 0; s < OP; ++s) rr[f].p[s] = __builtin_bit_cast(bf16x8, M.fwd.r[w][f * OP + s][lane]);
#pragma unroll
                    for (int t = 0; t < CT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[t][r] *= et[t];
#pragma unroll
                    for (int f = 0; f < CF; ++f) {
                        Op<PP> p[CT];
#pragma unroll
                        for (int t = 2 * f; t < CT; ++t) p[t] = op_rows<PP>(M.p + Tr::at(t / 2, 16 * (t & 1) + c) + 32 * f + 8 * g, TPL);
#pragma unroll
                        for (int i = 0; i < PAIRS<OP, PP>; ++i)
#pragma unroll
                            for (int t = 2 * f; t < CT; ++t) mm<OP, PP>(i, x[t], rr[f], p[t]);
                    }
                    if constexpr (MODE == FWD) {
                        char* const op = static_cast<char*>(L.o) + (b * L.o_s[0] + h * L.o_s[1] + tb * L.o_s[2] + n0 + 4 * g) * ES;
#pragma unroll
                        for (int t = 0; t < CT; ++t) {
                            if (16 * t + c >= last) continue;
                            char* to = op + (16 * t + c) * (L.o_s[2] * ES);
                            if (left >= 4) {
                                if constexpr (ES == 2) {
                                    const u32x2 y = {pack2(x[t][0], x[t][1]), pack2(x[t][2], x[t][3])};
                                    memcpy(to, &y, 8);
                                } else {
                                    store16(to, __builtin_bit_cast(u32x4, x[t]));
                                }
                            } else {
#pragma unroll
                                for (int r = 0; r < 3; ++r)
                                    if (r < left) Ops<E>::store1(reinterpret_cast<E*>(to) + r, x[t][r]);
                            }
                        }
                    } else {
                        // o . dO over the wave's columns
#pragma unroll
                        for (int t = 0; t < CT; ++t) {
                            const int tok = 16 * t + c;
                            float s = 0.f;
#pragma unroll
                            for (int r = 0; r < 4; ++r) s = __builtin_fmaf(r < left ? x[t][r] : 0.f, float_of<E>(vr[4 * t + r]), s);
                            s += __shfl_xor(s, 16);
                            s += __shfl_xor(s, 32);
                            if (g == 0 && tok < last) L.odo[(head * L.parts + n0 / 16) * (static_cast<long long>(L.blocks) * C) + tb + tok] = s;
                        }
                    }
                }
                if (work) {
                    if constexpr (MODE == RECORD) {         // this block's dO, for its outputs
#pragma unroll
                        for (int t = 0; t < CT; ++t) {
                            const int tok = 16 * t + c < cnt ? 16 * t + c : cnt - 1;
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int at = n0 + 4 * g + r < dv ? n0 + 4 * g + r : dv - 1;
                                vr[4 * t + r] = bits<E>(gp + static_cast<long long>(t0) * gst + (tok * gst + at * ES));
                            }
                        }
                    }
                    scores();
                    if (on) {
#pragma unroll
                        for (int t = 0; t < CT; ++t) {
                            x[t] = zero4();
                            et[t] = L.scale * M.e[16 * t + c];
                        }
#pragma unroll
                        for (int f = 0; f < DF; ++f) {      // Q S, columns x tokens
                            Op<OP> so;
                            Op<P> qr[CT];
#pragma unroll
                            for (int s = 0; s < OP; ++s) so.p[s] = __builtin_bit_cast(bf16x8, M.fwd.s[w][f * OP + s][lane]);
#pragma unroll
                            for (int t = 0; t < CT; ++t) qr[t] = op_rows<P>(M.q + (16 * t + c) * SK + 32 * f + 8 * g, KPL);
#pragma unroll
                            for (int i = 0; i < PAIRS<OP, P>; ++i)
#pragma unroll
                                for (int t = 0; t < CT; ++t) mm<OP, P>(i, x[t], so, qr[t]);
                        }
                    }
                }
            }
        } else {
            if (chain && on) held();
            if (!chain) scores();
            __syncthreads();                // (P^T is written)
            if (!on) continue;
            if (chain) {
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const f32x4 tw = factors(M.w, t);
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[t][r] *= tw[r];
                }
#pragma unroll
                for (int f = 0; f < CF; ++f) {
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = float_of<E>(vv[8 * f + i]);
                    const Op<P> go = op_of<P>(y);
                    Op<3> a[CT];
#pragma unroll
                    for (int t = 0; t < 2 * f + 2; ++t) a[t] = op_rows<3>(M.p + Tr::at(t / 2, row_of(0, t & 1, c)) + 32 * f + 8 * g, TPL);
#pragma unroll
                    for (int i = 0; i < PAIRS<3, P>; ++i)
#pragma unroll
                        for (int t = 0; t < 2 * f + 2; ++t) mm<3, P>(i, z[t], a[t], go);
                }
                f32x4 du[CT];
                solve(du);
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const f32x4 te = factors(M.e, t), tb = factors(M.beta, t);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int tok = 32 * (t / 2) + 8 * g + 4 * (t & 1) + r;
                        if (in && tok < cnt) L.rec_du[(head * (static_cast<long long>(L.blocks) * C) + t0 + tok) * dv + n] = du[t][r];
                        du[t][r] *= -te[r] * tb[r];
                    }
                }
                update(du);
            } else {
                f32x4 add[DT];
#pragma unroll
                for (int d = 0; d < DT; ++d) add[d] = zero4();
#pragma unroll
                for (int f = 0; f < CF; ++f) {
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = float_of<E>(vv[8 * f + i]) * (L.scale * M.e[32 * f + 8 * g + i]);
                    const Op<3> o3 = op_of<3>(y);
                    const uint16_t* at = M.q + (32 * f + 8 * g + (c >> 2)) * SK + 8 * (c & 3);
#pragma unroll
                    for (int d2 = 0; d2 < DT; d2 += 4) {
                        Op<P> qc[4];
#pragma unroll
                        for (int d = 0; d < 4; ++d) qc[d] = op_cols<P>(at + 32 * ((d2 + d) / 2) + 4 * (d & 1), SK, KPL);
#pragma unroll
                        for (int i = 0; i < PAIRS<P, 3>; ++i)
#pragma unroll
                            for (int d = 0; d < 4; ++d) mm<P, 3>(i, add[d2 + d], qc[d], o3);
                    }
                }
#pragma unroll
                for (int d = 0; d < DT; ++d) M.add[w][d][lane] = add[d];
            }
        }
    }

    if (chain && on) {
        float* dst = BACK ? L.dS0 : L.S_T;
        if (dst != nullptr) record(dst + bh * cells);
        if constexpr (MODE == RECORD) record(L.rec_S + (head * (L.blocks + 1) + blocks) * cells);
    }
    if constexpr (MODE == FWD) {            // tokens past the sequence's length
        E* const op = static_cast<E*>(L.o) + b * L.o_s[0] + h * L.o_s[1] + sl * SLICE;
        if (lane < dv - sl * SLICE)
            for (long long t = len + wave; t < L.T; t += 2 * NW) Ops<E>::store1(op + t * L.o_s[2] + lane, 0.f);
    }
}

// the scan for a type, padded channels and direction: by two kinds of waves where the LDS holds what they pass on
template <typename E, int DKP, int MODE> struct Scan {
    static constexpr bool PAIR = sizeof(PairMem<E, DKP, MODE>) <= 160 * 1024;
    static constexpr int THREADS = PAIR ? PAIR_NT : NT;
    static constexpr size_t BYTES = PAIR ? sizeof(PairMem<E, DKP, MODE>) : sizeof(Mem<E, DKP, MODE>);
    static_assert(BYTES <= 160 * 1024, "one compute unit's LDS");
    static __device__ __forceinline__ void run(const DeltaLaunch& L, long head, int sl, unsigned char* smem)
    {
        if constexpr (PAIR) {
            if (__builtin_amdgcn_readfirstlane(threadIdx.x) < NT) pair_scan<E, DKP, MODE, true>(L, head, sl, smem);
            else pair_scan<E, DKP, MODE, false>(L, head, sl, smem);
        } else scan<E, DKP, MODE>(L, head, sl, smem);
    }
};

}  // namespace delta
}  // namespace sfda
