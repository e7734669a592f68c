// The scan of the gated delta rule over blocks of tokens (gfx950), shared by the forward and the backward.
//
// For one head, with a_t = exp(log_decay_t):  S_t = a_t S_(t-1) + k_t (beta_t r_t)^T,  r_t = v_t - a_t S_(t-1)^T k_t,  o_t = c S_t^T q_t.
// In a block of C tokens let G_i be the sum of its log decays up to i, e_i = exp(G_i), w_i = exp(G_C - G_i), D_ij = exp(G_i - G_j) for
// j <= i, L_ij = D_ij k_i . k_j for j < i, S the state before the block and U the gradient of the state after it.  Then
//   R = (I + L diag(beta))^(-1) (V - e K S),      O = c (e Q S + P diag(beta) R),  P = D . Q K^T
//   S' = e_C S + K^T (w beta R)
// and backward, with du the gradient of the writes u_t = beta_t r_t,
//   du = (I + diag(beta) L)^(-T) (c P^T dO + w K U),   U' = e_C U + Q^T (c e dO) - K^T (e beta du).
// The inverses and P do not depend on the state: sfda_delta_prep forms them for all blocks at once.  What is left to be done block after
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

#include <type_traits>

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
// the same with the lane's rows 8 g + c / 4 and 4 further given apart
template <int P> __device__ __forceinline__ Op<P> op_cols2(const uint16_t* p, const uint16_t* q, int plane)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    Op<P> o;
#pragma unroll
    for (int s = 0; s < P; ++s) {
        u32x4 w;
        w.lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + s * plane)));
        w.hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(q + s * plane)));
        o.p[s] = __builtin_bit_cast(bf16x8, w);
    }
    return o;
}
// the products of parts that reach 2^-22 of the whole (of two parts 2^-16), the small ones first; a loop over tiles inside one over these has no product
// wait for the last
template <int PA, int PB> constexpr int PAIRS = PA == 2 && PB == 2 ? 3 : PA * PB < 9 ? PA * PB : 6;
template <int PA, int PB> __device__ __forceinline__ void mm(int i, f32x4& d, const Op<PA>& a, const Op<PB>& b)
{
    static_assert(PA == 1 || PB == 1 || PA == PB, "parts");
    if constexpr (PA == 3 && PB == 3) {
        constexpr int A[6] = {2, 0, 1, 1, 0, 0}, B[6] = {0, 2, 1, 0, 1, 0};
        mfma(d, a.p[A[i]], b.p[B[i]]);
    } else if constexpr (PA == 2 && PB == 2) {
        mfma(d, a.p[i == 0], b.p[i == 1]);
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
// exp(x) by the hardware's power of 2: off by an ulp and by |x| 2^-24 of itself, x negative
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504089f); }
// The decays between token `one` and tokens four .. four + 3 of a block, from the sums of the log decays: of those that come later
// (earlier, if `back`) the reciprocals.  Without branches: the compiler makes a branch of a masked result's every load and exponential
// (12 of them took 2 us of a block).
__device__ __forceinline__ void decays(float (&d)[4], const float* hi, const float* lo, int one, int four, bool back)
{
    const f32x4 h4 = *reinterpret_cast<const f32x4*>(hi + four), l4 = *reinterpret_cast<const f32x4*>(lo + four);
    const float h1 = hi[one], l1 = lo[one];
#pragma unroll
    for (int r = 0; r < 4; ++r) d[r] = pin(exp_of(back ? (h4[r] - h1) + (l4[r] - l1) : (h1 - h4[r]) + (l1 - l4[r])));
}
// Lanes (c, g) hold rows 4 g + r of column c; then they hold columns 4 (c / 4) + r of row 4 g + c % 4: 4 x 4 in each four lanes.
__device__ __forceinline__ void turn4(f32x4& a, int c)
{
    auto from = [](float x, auto ctrl) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, false)); };
    const bool odd = c & 1, two = c & 2;
#pragma unroll
    for (int x = 0; x < 4; x += 2) {
        const float got = from(odd ? a[x] : a[x + 1], std::integral_constant<int, 0xB1>());        // quad [1, 0, 3, 2]
        a[x] = odd ? got : a[x];
        a[x + 1] = odd ? a[x + 1] : got;
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const float got = from(two ? a[x] : a[x + 2], std::integral_constant<int, 0x4E>());        // quad [2, 3, 0, 1]
        a[x] = two ? got : a[x];
        a[x + 2] = two ? a[x + 2] : got;
    }
}
__device__ __forceinline__ int row_of(int f, int h, int c) { return 32 * f + 8 * (c >> 2) + 4 * h + (c & 3); }     // of a tile's row c

// Rows of keys and queries in LDS, DKP channels each: the 16-byte units of row i change places by x(i) = 4 (i % 4) + i / 4 % 4, so that what
// is read at a time lies on different banks: one unit of 8 rows (i .. i + 7, or two fours 8 apart), or four neighbouring
// units of 4 rows (of 64 channels, whose rows are 8 units long, by x(i) / 2).  An index of channel 32 f of a row is that of
// channel 0 with 32 f in exclusive or.
template <int DKP> struct KeyRows {
    static constexpr int SHIFT = DKP >= 128 ? 0 : 1;
    static __device__ __forceinline__ int at(int row, int unit) { return row * DKP + 8 * (unit ^ ((4 * (row & 3) + (row >> 2 & 3)) >> SHIFT)); }
};

// A value that the compiler takes for another one at each call: what is computed from it is not kept over a loop (and spilled; a
// reload waits for all loads before it)
__device__ __forceinline__ int anew(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// A block's rows of one tensor on their way to LDS: C tokens x COLS channels (padded), 16-byte vectors held in registers between the
// load and the write.  The vector that would cross a row's end is moved back to end with it and into place when it is written; rows
// shorter than a vector are read by elements.  Rows past the n that are there are read as the last one and written as zeros; the
// padding's zeros in LDS are never written.
template <typename E, int COLS, int C, int STRIDE, int THREADS = NT, bool SWAPPED = false> struct RowTile {
    static constexpr int VE = Ops<E>::VE, ES = sizeof(E), VPR = COLS / VE, RPP = THREADS / VPR, N = C / RPP, PLANE = C * STRIDE;
    static_assert(THREADS % VPR == 0 && C % RPP == 0 && N >= 1, "whole passes");
    u32x4 x[N];

    __device__ __forceinline__ void load(const char* base, uint32_t st, int n, int cols, int thread)
    {
        const int tid = anew(thread), col = (tid % VPR) * VE, r0 = tid / VPR;
        const uint32_t at = (col + VE <= cols ? col : col >= cols || cols < VE ? 0 : cols - VE) * ES;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int r = r0 + u * RPP;
            const uint32_t off = (r < n ? r : n - 1) * st + at;
            if (cols >= VE) x[u] = load16(base + off);
            else x[u] = col == 0 ? short_row<E>(base + off, cols) : u32x4{0, 0, 0, 0};
        }
    }
    // as they lie in memory, rows STRIDE elements apart, zeros past the columns too
    __device__ __forceinline__ void store_raw(E* lds, int n, int cols, int tid) const
    {
        const int col = (tid % VPR) * VE, past = cols < VE ? 0 : col + VE - cols;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int r = tid / VPR + u * RPP;
            u32x4 w = r < n && col < cols ? x[u] : u32x4{0, 0, 0, 0};
            if (cols % VE != 0 && past > 0 && past < VE) w = move_down<E>(w, past);
            *reinterpret_cast<u32x4*>(lds + r * STRIDE + col) = w;
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
            uint16_t* to = lds + (SWAPPED ? KeyRows<COLS>::at(r, col / 8) + col % 8 : r * STRIDE + col);
            Ops<E>::put(to, PLANE, w);
        }
    }
};

// The parts of a block's triangular matrices on their way to LDS: 16 bytes are half a tile's row.  HALVES of a part for THREADS
// threads; the first `parts` of them are there.
template <int TILES, int PARTS, int THREADS> struct Matrix {
    static constexpr int HALVES = TILES * 32, N = (PARTS * HALVES + THREADS - 1) / THREADS;
    u32x4 x[N];
    __device__ __forceinline__ void load(const uint16_t* from, int thread)
    {
        const int tid = anew(thread);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int i = tid + u * THREADS;
            x[u] = *reinterpret_cast<const u32x4*>(from + static_cast<uint32_t>(8 * (i < PARTS * HALVES ? i : 0)));
        }
    }
    // place(part, row tile, column tile, row, column) of 8 neighbours; UPPER: tile (i, j) of the triangle has column tile i
    template <bool UPPER, typename Place> __device__ __forceinline__ void store(int thread, Place place) const
    {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int i = thread + u * THREADS, part = i / HALVES, j = i - part * HALVES, tile = j >> 5;
            const int ti = tile < 1 ? 0 : tile < 3 ? 1 : tile < 6 ? 2 : 3, tj = tile - ti * (ti + 1) / 2;
            if (i < PARTS * HALVES) *reinterpret_cast<u32x4*>(place(part, 16 * (UPPER ? tj : ti) + (j >> 1 & 15), 16 * (UPPER ? ti : tj) + 8 * (j & 1))) = x[u];
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
        const uint32_t lane = 8 * anew(g) * st + col;
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

enum Mode { FWD, RECORD, ADJOINT, STATES };      // STATES: a segment's end state alone, and what it makes of its start state

// Parts of the state, of R and of P as operands of the outputs, for inputs of P parts.  A bfloat16 output's terms may cancel (keys that
// are alike, strengths past 1), so that one part of 8 bits each leaves an error of up to 0.017 of the results; two leave their own rounding,
// 0.0017.  The rows of R and the sums of outputs that the backward records are float32.
template <int P, int MODE> constexpr int OUT_PARTS = MODE == FWD && P == 1 ? 2 : 3;

template <typename E, int DKP, int MODE> struct Mem {
    typedef Block<E> B;
    static constexpr int C = B::C, P = B::P, PP = OUT_PARTS<P, MODE>, SK = DKP + 8, ST = C + 8;
    static constexpr int KPL = C * SK, TPL = C * ST;        // planes
    uint16_t k[P * KPL], q[P * KPL], t[3 * TPL], p[PP * TPL];
    float e[C], w[C], beta[C], end[4];
};

// One workgroup scans one head for 64 value columns, 16 in a wave.  (For float32 of more than 128 channels, and the bfloat16 backward
// of more: their operands and what two kinds of waves pass on do not fit the LDS together.)
template <typename E, int DKP, int MODE> __device__ __forceinline__ void scan(const DeltaLaunch& L, long head, int sl, unsigned char* smem)
{
    typedef Block<E> B;
    typedef Mem<E, DKP, MODE> M_;
    constexpr int C = B::C, CT = B::CT, CF = B::CF, P = B::P, PP = M_::PP, TILES = B::TILES, ES = sizeof(E);
    constexpr int DT = DKP / 16, DF = DKP / 32, SK = M_::SK, ST = M_::ST, KPL = M_::KPL, TPL = M_::TPL;
    constexpr bool BACK = MODE == ADJOINT;
    constexpr int OP = PP;
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
    const uint16_t* const tmat = (BACK ? L.inv_back : L.inv) + head * L.blocks * static_cast<long long>(3 * TILES * 256);
    const uint16_t* const pmat = (BACK ? L.scores_back : L.scores) + head * L.blocks * static_cast<long long>(3 * TILES * 256);
    const float4* const scal = L.scalars + 2 * (head * L.blocks * static_cast<long long>(C));

    RowTile<E, DKP, C, SK> tk, tq;
    Matrix<TILES, 3, NT> tt;
    Matrix<TILES, PP, NT> pp;
    float4 sc[2];
    uint32_t vr[CT * 4];                    // V, or dO
    auto fetch = [&](int blk) {
        const int t0 = blk * C, cnt = len - t0 < C ? len - t0 : C;
        tk.load(kp + static_cast<long long>(t0) * kst, kst, cnt, dk, tid);
        tq.load(qp + static_cast<long long>(t0) * qst, qst, cnt, dk, tid);
        tt.load(tmat + static_cast<long long>(blk) * (3 * TILES * 256), tid);
        pp.load(pmat + static_cast<long long>(blk) * (3 * TILES * 256), tid);
        const int tok = tid < C ? tid : 0;
        sc[0] = scal[2 * (static_cast<long long>(blk) * C + tok)];
        sc[1] = scal[2 * (static_cast<long long>(blk) * C + tok) + 1];
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
        tt.template store<BACK>(tid, [&](int s, int row, int col) { return M.t + s * TPL + row * ST + col; });
        pp.template store<BACK>(tid, [&](int s, int row, int col) { return M.p + s * TPL + row * ST + col; });
        if (tid < C) {
            M.beta[tid] = sc[0].z;
            M.e[tid] = sc[0].w;
            M.w[tid] = sc[1].x;
            if (tid == 0) {
                M.end[0] = sc[1].z;
                M.end[1] = sc[1].w;
            }
        }
        __syncthreads();
        float vv[CT * 4];
#pragma unroll
        for (int i = 0; i < CT * 4; ++i) vv[i] = on ? float_of<E>(vr[i]) : 0.f;
        if (it + 1 < blocks) fetch(BACK ? blk - 1 : blk + 1);

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
// The same scan with eight waves: four hold the state and run the chain alone, four help.  Forward, the helpers form the
// outputs, a block behind the chain, from the state and R as operands that the chain's waves leave in LDS fragment by fragment (as
// the lane has them: 16 bytes a lane, no two on one bank).  Backward, they form Q^T (c e dO), which does not depend on the state.
// Bound by the chain: bfloat16, 128 channels, 8300 to 11000 cycles for 64 tokens, of which K S takes 800, the solve 1900, the update 2000, and
// waits for operands most of the rest: for rows from memory (20 bytes a cycle on a compute unit) and for the LDS.  B8 H16 T4096: forward 345 us
// (with outputs of one part 320, and 545 by four waves for all of it), the two scans of the backward 900 (1689).

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
    static constexpr int C = B::C, P = B::P, OP = MODE == STATES ? 1 : OUT_PARTS<P, MODE>, PP = OP;
    typedef Tri<C, BACK> T;
    static constexpr int KPL = C * DKP, TPL = T::SIZE, DF = DKP / 32, DT = DKP / 16;
    // fragments of the state that the helpers have at a time: of more than 128 bfloat16 channels one half, then the other
    static constexpr int SF = MODE == FWD && P == 1 && DKP > 128 ? DF / 2 : DF;
    static constexpr int SV = SLICE + (sizeof(E) == 2 ? 16 : 4);
    uint16_t k[P * KPL], q[P * KPL], t[3 * TPL], p[PP * TPL];
    E v[C * SV];                // V, or dO, of the slice
    union {
        struct { u32x4 s[NW][SF * OP][64], r[NW][B::CF * OP][64]; } fwd;        // the state and R
        f32x4 add[NW][BACK ? DT : 1][64];                                       // Q^T (c e dO)
    };
    float e[C], w[C], beta[C], end[4];
};

constexpr int PAIR_NT = 2 * NT;

// chain: the wave holds the state.  (Each kind of wave runs a copy of its own, with the other kind's registers free; all have the same
// barriers.)
template <typename E, int DKP, int MODE, bool chain, bool whole> __device__ __forceinline__ void pair_scan(const DeltaLaunch& L, long head, int sl, int seg, unsigned char* smem)
{
    typedef Block<E> B;
    typedef PairMem<E, DKP, MODE> M_;
    typedef typename M_::T Tr;
    typedef KeyRows<DKP> Key;
    constexpr int C = B::C, CT = B::CT, CF = B::CF, P = B::P, PP = M_::PP, OP = M_::OP, TILES = B::TILES, ES = sizeof(E);
    constexpr int DT = DKP / 16, DF = DKP / 32, SF = M_::SF, KPL = M_::KPL, TPL = M_::TPL;
    constexpr bool BACK = MODE == ADJOINT;
    M_& M = *reinterpret_cast<M_*>(smem);

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int w = wave & (NW - 1);
    const long long bh = L.first + head;
    const int b = __builtin_amdgcn_readfirstlane(static_cast<int>(bh / L.H)), h = __builtin_amdgcn_readfirstlane(static_cast<int>(bh - static_cast<long long>(b) * L.H));
    const int hk = h / (L.H / L.Hk), dk = L.dk, dv = L.dv;
    const int len = __builtin_amdgcn_readfirstlane(seq_length(L.lengths, b, L.T));
    // the segment's blocks
    const int all = (len + C - 1) / C, begin = BACK || MODE == RECORD ? 0 : min(seg * L.seg_blocks, all);
    const int end = BACK || MODE == RECORD ? all : min(begin + L.seg_blocks, all), blocks = end - begin;
    // a segment's state after it is what it makes of the state before it, M S, plus what its tokens write, N.  Slices past those of the
    // value columns take M's: the same scan from the unit matrix with values of zero.
    const bool unit = MODE == STATES && sl >= L.slices;
    if (unit) sl -= L.slices;
    const int width = unit ? dk : dv;
    const int n0 = sl * SLICE + 16 * w, n = n0 + c;         // the wave's columns, the lane's
    const bool on = n0 < width, in = n < width;

    const char* const kp = static_cast<const char*>(L.k) + (b * L.k_s[0] + hk * L.k_s[1]) * ES;
    const char* const qp = static_cast<const char*>(L.q) + (b * L.q_s[0] + hk * L.q_s[1]) * ES;
    const char* const vp = static_cast<const char*>(L.v) + (b * L.v_s[0] + h * L.v_s[1]) * ES;
    const char* const gp = MODE == FWD ? nullptr : static_cast<const char*>(L.dO) + (b * L.g_s[0] + h * L.g_s[1]) * ES;
    const uint32_t kst = static_cast<uint32_t>(L.k_s[2] * ES), qst = static_cast<uint32_t>(L.q_s[2] * ES), vst = static_cast<uint32_t>(L.v_s[2] * ES);
    const uint32_t gst = MODE == FWD ? 0 : static_cast<uint32_t>(L.g_s[2] * ES);
    const uint16_t* const tmat = (BACK ? L.inv_back : L.inv) + head * L.blocks * static_cast<long long>(3 * TILES * 256);
    const uint16_t* const pmat = (BACK ? L.scores_back : L.scores) + head * L.blocks * static_cast<long long>(3 * TILES * 256);
    const float4* const scal = L.scalars + 2 * (head * L.blocks * static_cast<long long>(C));

    RowTile<E, DKP, C, DKP, PAIR_NT, true> tk, tq;
    Matrix<TILES, 3, NT> tt;                // the inverse and P, by the helpers
    Matrix<TILES, PP, NT> pp;
    float4 sc[2];
    RowTile<E, SLICE, C, M_::SV, NT> tv;    // V, or dO, by the helpers
    const int cols = width - sl * SLICE < SLICE ? width - sl * SLICE : SLICE;
    const char* const wp = (BACK ? gp : vp) + sl * SLICE * ES;
    const uint32_t wst = BACK ? gst : vst;
    // A block's loads.  A compute unit takes in some 20 bytes a cycle, and a wave whose loads find no room stands still: forward,
    // where they are due sooner, all go out first; backward, the matrices' and values' after the helpers' products.
    auto fetch_keys = [&](int blk) {
        const int t0 = blk * C, cnt = len - t0 < C ? len - t0 : C;
        tk.load(kp + static_cast<long long>(t0) * kst, kst, cnt, dk, tid);
        if (MODE != STATES) tq.load(qp + static_cast<long long>(t0) * qst, qst, cnt, dk, tid);
    };
    auto fetch_matrices = [&](int blk) {        // (by the helpers; forward, P is that of the block before)
        if (blk < end) tt.load(tmat + static_cast<long long>(blk) * (3 * TILES * 256), tid - NT);
        if (MODE != STATES && (BACK || blk > begin)) pp.load(pmat + static_cast<long long>(BACK ? blk : blk - 1) * (3 * TILES * 256), tid - NT);
    };
    auto fetch_values = [&](int blk) {          // (by the helpers)
        const int t0 = blk * C, cnt = len - t0 < C ? len - t0 : C, tok = tid - NT < C ? tid - NT : 0;
        sc[0] = scal[2 * (static_cast<long long>(blk) * C + tok)];
        sc[1] = scal[2 * (static_cast<long long>(blk) * C + tok) + 1];
        if (!unit) tv.load(wp + static_cast<long long>(t0) * wst, wst, cnt, cols, tid - NT);
    };
    if (blocks > 0) {
        fetch_keys(BACK ? end - 1 : begin);
        if constexpr (!chain) {
            fetch_matrices(BACK ? end - 1 : begin);
            fetch_values(BACK ? end - 1 : begin);
        }
    }

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
    if (chain && MODE == STATES) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[d][r] = unit && channel(d, r) == n ? 1.f : 0.f;
    } else if (chain) {
        const float* src = BACK ? L.dS_T : L.S0;
        if (src != nullptr) src += bh * cells;
        // the state that enters a segment lies where N of the one before it lay; a copy of S0, which the last segment may write (as S_T)
        // before the first one reads it, lies behind them
        if (MODE == FWD && L.segments > 1 && (seg > 0 || src != nullptr)) src = L.seg_N + (((seg > 0 ? seg : L.segments) - 1) * static_cast<long long>(L.heads) + head) * cells;
        if (src != nullptr) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (in && channel(d, r) < dk) S[d][r] = src[channel(d, r) * dv + n];
        }
    }
    // Rows of 4 g + r neighbours to memory: with `whole` columns by 16 bytes (a lane's four rows, each in another line, take four
    // times as many stores, which bound the scans that record).  Stores past the resource's range are dropped: a store that a branch
    // skips would make the waits for loads before it waits for all stores too.
    constexpr uint32_t NOWHERE = 0x80000000u;
    auto put = [&](float* to, int row, int most, f32x4 x) {     // row: the first of four
        const From<true> out(reinterpret_cast<const char*>(to));
        if constexpr (whole) {
            const int r = row + (c & 3), at = anew(r * width + n0 + 4 * (c >> 2));
            turn4(x, c);
            out.store(r < most && n0 + 4 * (c >> 2) < width ? static_cast<uint32_t>(4 * at) : NOWHERE, 0, __builtin_bit_cast(u32x4, x));
        } else {
            const int at = anew(row * width + n);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x[r]), out.r, in && row + r < most ? static_cast<uint32_t>(4 * (at + r * width)) : NOWHERE, 0, 0);
        }
    };
    auto record = [&](float* to) {
#pragma unroll
        for (int d = 0; d < DT; ++d) put(to, channel(d, 0), dk, S[d]);
    };
    Op<OP> ro[BACK ? 1 : CF];               // R, of the chain's waves
    f32x4 x[BACK ? 1 : CT];                 // outputs, of the helpers
    float et[BACK ? 1 : CT];
    uint32_t dr[MODE == RECORD ? CT : 1][ES];       // their dO: 4 neighbours

    Op<3> s3[chain ? DF : 1];               // the state as an operand
    auto split = [&](int f) { s3[f] = op_of<3>(S[2 * f], S[2 * f + 1]); };
    if constexpr (chain) {
#pragma unroll
        for (int f = 0; f < DF; ++f) split(f);
    }
    auto give = [&](int first) {            // the state's fragments from `first` on to the helpers
#pragma unroll
        for (int f = 0; f < SF; ++f)
#pragma unroll
            for (int s = 0; s < OP; ++s) M.fwd.s[w][f * OP + s][lane] = __builtin_bit_cast(u32x4, s3[first + f].p[s]);
    };

#pragma clang loop unroll(disable)
    for (int it = 0; it < (BACK || MODE == STATES ? blocks : blocks + 1); ++it) {
        const bool work = it < blocks;
        const int blk = BACK ? end - 1 - it : begin + it, t0 = blk * C, cnt = len - t0 < C ? len - t0 : C;
        // a lane's elements of keys and queries: by columns, rows 8 g + c / 4 and 4 further; by rows, of a tile's h = 0 and 1 and of 16 rows in
        // their order.  (Given anew for each block, or their places for all channels are kept over the blocks, and spilled.)
        int at0 = Key::at(8 * g + (c >> 2), c & 3), at1 = Key::at(8 * g + 4 + (c >> 2), c & 3);
        int row0 = Key::at(row_of(0, 0, c), g), row1 = Key::at(row_of(0, 1, c), g), rown = Key::at(c, g);
        asm volatile("" : "+v"(at0), "+v"(at1), "+v"(row0), "+v"(row1), "+v"(rown));
        __syncthreads();                    // (the last block's operands are read)
        if (work) {
            tk.store(M.k, cnt, dk, tid);
            if (MODE != STATES) tq.store(M.q, cnt, dk, tid);
        }
        if constexpr (chain) {
            if (on) {
                if constexpr (!BACK && MODE != STATES) {
                    if (it > 0) {
#pragma unroll
                        for (int f = 0; f < CF; ++f)
#pragma unroll
                            for (int s = 0; s < OP; ++s) M.fwd.r[w][f * OP + s][lane] = __builtin_bit_cast(u32x4, ro[f].p[s]);
                    }
                    if (work) give(0);
                }
                if constexpr (MODE == RECORD) {
                    if (work) record(L.rec_S + (head * (L.blocks + 1) + blk) * cells);
                }
                if constexpr (MODE == ADJOINT) record(L.rec_U + (head * L.blocks + blk) * cells);
            }
        } else {
            if (work) {
                const int htid = tid - NT;
                tv.store_raw(M.v, unit ? 0 : cnt, cols, htid);
                tt.template store<BACK>(htid, [&](int s, int row, int col) { return M.t + s * TPL + Tr::row(row) + col; });
                if (htid < C) {
                    M.beta[htid] = sc[0].z;
                    M.e[htid] = sc[0].w;
                    M.w[htid] = BACK ? sc[1].x : sc[1].y;       // (forward: w beta)
                    if (htid == 0) {
                        M.end[0] = sc[1].z;
                        M.end[1] = sc[1].w;
                    }
                }
            }
            // (forward: of the block before)
            if (MODE != STATES && (BACK || it > 0)) pp.template store<BACK>(tid - NT, [&](int s, int row, int col) { return M.p + s * TPL + Tr::row(row) + col; });
        }
        __syncthreads();
        const bool more = it + 1 < blocks;
        const int next = BACK ? blk - 1 : blk + 1;

        // the wave's column c of V or dO: 8 neighbouring tokens
        auto tokens8 = [&](float (&y)[8], int f) {
            if constexpr (ES == 2) {
                const Op<1> o = op_cols<1>(M.v + (32 * f + 8 * g + (c >> 2)) * M_::SV + 16 * w + 4 * (c & 3), M_::SV, 0);
                const u32x4 x = __builtin_bit_cast(u32x4, o.p[0]);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = i & 1 ? hi_f32(x[i / 2]) : lo_f32(x[i / 2]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = M.v[(32 * f + 8 * g + i) * M_::SV + 16 * w + c];
            }
        };
        // The chain's products, each one's operands on their way from LDS before the product before it: the compiler leaves them where
        // they are used, and a wave waits 130 cycles and more for each.  Barriers for the scheduler alone keep them apart; between two, vector
        // instructions fill the matrix instructions' time.
        typedef Op<P> KeyOp[4];
        typedef Op<3> InvOp[2];
        f32x4 z[CT], R[CT];
        auto key_rows = [&](KeyOp& k, int f) {
#pragma unroll
            for (int t = 0; t < CT; ++t) k[t] = op_rows<P>(M.k + (t / 2) * 32 * DKP + ((t & 1 ? row1 : row0) ^ 32 * f), KPL);
        };
        auto key_cols = [&](const uint16_t* from, KeyOp& k, int f, int d2) {
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const int x = 32 * ((d2 + d) / 2);
                k[d] = op_cols2<P>(from + 32 * f * DKP + (at0 ^ x) + 4 * (d & 1), from + 32 * f * DKP + (at1 ^ x) + 4 * (d & 1), KPL);
            }
        };
        auto inverse = [&](InvOp& a, int t2, int f) {
#pragma unroll
            for (int t = 0; t < 2; ++t) a[t] = op_rows<3>(M.t + Tr::at(t2 / 2, row_of(0, t, c)) + 32 * f + 8 * g, TPL);
        };
        auto solve = [&](const InvOp& a, int t2, const Op<3>& y) {
#pragma unroll
            for (int i = 0; i < 6; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t) mm<3, 3>(i, R[t2 + t], a[t], y);
        };
        // R or du of 32 tokens
        auto record_rows = [&](float* rec, int f) {
            float* const to = rec + (head * (static_cast<long long>(L.blocks) * C) + t0) * dv;
            put(to, 32 * f + 8 * g, cnt, R[2 * f]);
            put(to, 32 * f + 8 * g + 4, cnt, R[2 * f + 1]);
        };
        // what the lane's tokens have in `from`
        auto factors = [&](const float* from, int t) { return *reinterpret_cast<const f32x4*>(from + 32 * (t / 2) + 8 * g + 4 * (t & 1)); };
        // K S, tokens x columns; the state decays meanwhile
        auto held = [&] {
            KeyOp k[2];
            key_rows(k[0], 0);
#pragma unroll
            for (int t = 0; t < CT; ++t) z[t] = R[t] = zero4();
            const float ghi = M.end[0], glo = M.end[1];
#pragma unroll
            for (int f = 0; f < DF; ++f) {
                if (f + 1 < DF) key_rows(k[(f + 1) & 1], f + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < PAIRS<P, 3>; ++i)
#pragma unroll
                    for (int t = 0; t < CT; ++t) mm<P, 3>(i, z[t], k[f & 1][t], s3[f]);
#pragma unroll
                for (int d = 2 * f; d < 2 * f + 2; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[d][r] = __builtin_fmaf(S[d][r], ghi, S[d][r] * glo);
            }
        };
        // S += K^T y, y the operands of the tokens' blocks of 32 in the order that they come in; the state's next operand on the way
        auto update = [&](KeyOp (&k)[2], int first, const Op<3>& y, bool last, int f) {
#pragma unroll
            for (int d2 = 0; d2 < DT; d2 += 4) {
                const int x = first + d2 / 4;
                if (d2 + 4 < DT) key_cols(M.k, k[(x + 1) & 1], f, d2 + 4);
                else if (!last) key_cols(M.k, k[(x + 1) & 1], BACK ? f - 1 : f + 1, 0);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < PAIRS<P, 3>; ++i)
#pragma unroll
                    for (int d = 0; d < 4; ++d) mm<P, 3>(i, S[d2 + d], k[x & 1][d], y);
                if (last && d2 > 0) {
                    split(d2 / 2 - 2);
                    split(d2 / 2 - 1);
                }
            }
            if (last) {
                split(DF - 2);
                split(DF - 1);
            }
        };

        if constexpr (!BACK) {
            if constexpr (chain) {
                if (!work) continue;
                if (more) fetch_keys(next);
                if (on) held();
                if constexpr (SF < DF) {
                    __syncthreads();        // (the first half is read)
                    if (on) give(SF);
                    __syncthreads();
                }
                if (!on) continue;
                InvOp a[2];
                inverse(a[0], 0, 0);
                f32x4 fe[CT], fw[CT];
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    fe[t] = factors(M.e, t);
                    fw[t] = factors(M.w, t);
                }
                float val[CF][8];
#pragma unroll
                for (int f = 0; f < CF; ++f) tokens8(val[f], f);
                auto lack = [&](int f) {
#pragma unroll
                    for (int t = 2 * f; t < 2 * f + 2; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) z[t][r] = val[f][4 * (t & 1) + r] - fe[t][r] * z[t][r];
                    return op_of<3>(z[2 * f], z[2 * f + 1]);
                };
                // R's tokens of a block of 32: the outputs' operand and the state's
                auto written = [&](int f) {
                    if constexpr (MODE != STATES) ro[f] = op_of<OP>(R[2 * f], R[2 * f + 1]);
                    if constexpr (MODE == RECORD) record_rows(L.rec_R, f);
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int t = 2 * f + i / 4, r = i % 4;
                        y[i] = R[t][r] * fw[t][r];
                    }
                    return op_of<3>(y);
                };
                KeyOp k[2];
                if constexpr (CF == 2) {
                    inverse(a[1], 2, 0);
                    const Op<3> z0 = lack(0);
                    __builtin_amdgcn_sched_barrier(0);
                    solve(a[0], 0, z0);
                    const Op<3> z1 = lack(1);
                    inverse(a[0], 2, 1);
                    __builtin_amdgcn_sched_barrier(0);
                    solve(a[1], 2, z0);
                    const Op<3> u0 = written(0);
                    key_cols(M.k, k[0], 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    solve(a[0], 2, z1);
                    update(k, 0, u0, false, 0);
                    const Op<3> u1 = written(1);
                    __builtin_amdgcn_sched_barrier(0);
                    update(k, DT / 4, u1, true, 1);
                } else {
                    const Op<3> z0 = lack(0);
                    key_cols(M.k, k[0], 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    solve(a[0], 0, z0);
                    const Op<3> u0 = written(0);
                    __builtin_amdgcn_sched_barrier(0);
                    update(k, 0, u0, true, 0);
                }
            } else {
                if (more) fetch_keys(next);
                if (work) fetch_matrices(next);
                if (more) fetch_values(next);
                if (MODE == STATES) continue;
                if (it > 0 && on) {         // the block before: x += P R
                    const int tb = t0 - C, left = dv - n0 - 4 * g, last = len - tb < C ? len - tb : C;
                    Op<OP> rr[CF];
                    Op<PP> ps[CF][CT];
#pragma unroll
                    for (int f = 0; f < CF; ++f) {
#pragma unroll
                        for (int s = 0; s < OP; ++s) rr[f].p[s] = __builtin_bit_cast(bf16x8, M.fwd.r[w][f * OP + s][lane]);
#pragma unroll
                        for (int t = 2 * f; t < CT; ++t) ps[f][t] = op_rows<PP>(M.p + Tr::at(t / 2, 16 * (t & 1) + c) + 32 * f + 8 * g, TPL);
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int t = 0; t < CT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[t][r] *= et[t];
#pragma unroll
                    for (int f = 0; f < CF; ++f)
#pragma unroll
                        for (int i = 0; i < PAIRS<OP, PP>; ++i)
#pragma unroll
                            for (int t = 2 * f; t < CT; ++t) mm<OP, PP>(i, x[t], rr[f], ps[f][t]);
                    if constexpr (MODE == FWD) {
                        char* const op = static_cast<char*>(L.o) + (b * L.o_s[0] + h * L.o_s[1] + tb * L.o_s[2] + n0) * ES;
                        const From<true> out(op);
                        const uint32_t ost = static_cast<uint32_t>(L.o_s[2] * ES);
#pragma unroll
                        for (int t = 0; t < CT; ++t) {
                            if constexpr (whole) {
                                const uint32_t off = 16 * t + c < last && left > 0 ? anew(16 * t + c) * ost + 4 * g * ES : NOWHERE;
                                if constexpr (ES == 2) __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack2(x[t][0], x[t][1]), pack2(x[t][2], x[t][3])}, out.r, off, 0, 0);
                                else out.store(off, 0, __builtin_bit_cast(u32x4, x[t]));
                                continue;
                            }
                            if (16 * t + c >= last) continue;
                            char* to = op + 4 * g * ES + static_cast<uint64_t>((16 * t + c) * ost);
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
                        const From<true> sums(reinterpret_cast<const char*>(L.odo + (head * L.parts + n0 / 16) * (static_cast<long long>(L.blocks) * C) + tb));
#pragma unroll
                        for (int t = 0; t < CT; ++t) {
                            const int tok = 16 * t + c;
                            float s = 0.f;
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const uint32_t y = dr[t][r * ES / 4];
                                s = __builtin_fmaf(r < left ? x[t][r] : 0.f, ES == 4 ? __uint_as_float(y) : r & 1 ? hi_f32(y) : lo_f32(y), s);
                            }
                            s += __shfl_xor(s, 16);
                            s += __shfl_xor(s, 32);
                            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(s), sums.r, g == 0 && tok < last ? 4u * tok : NOWHERE, 0, 0);
                        }
                    }
                }
                if (work) {
                    if constexpr (MODE == RECORD) {         // this block's dO, for its outputs
#pragma unroll
                        for (int t = 0; t < CT; ++t) {
                            const int tok = 16 * t + c < cnt ? 16 * t + c : cnt - 1;
                            const char* const from = gp + static_cast<long long>(t0) * gst;
                            if constexpr (whole) {
                                memcpy(&dr[t], from + (tok * gst + (n0 + 4 * g < dv ? n0 + 4 * g : 0) * ES), 4 * ES);
                            } else {
#pragma unroll
                                for (int r = 0; r < 4; ++r)
                                    dr[t][r * ES / 4] = (r * ES % 4 ? dr[t][r * ES / 4] : 0) | bits<E>(from + (tok * gst + (n0 + 4 * g + r < dv ? n0 + 4 * g + r : dv - 1) * ES)) << (r * ES % 4 * 8);
                            }
                        }
                    }
                    auto times = [&](int first) {           // Q S, columns x tokens
#pragma unroll
                        for (int f = 0; f < SF; ++f) {
                            Op<OP> so;
                            Op<P> qr[CT];
#pragma unroll
                            for (int s = 0; s < OP; ++s) so.p[s] = __builtin_bit_cast(bf16x8, M.fwd.s[w][f * OP + s][lane]);
#pragma unroll
                            for (int t = 0; t < CT; ++t) qr[t] = op_rows<P>(M.q + 16 * t * DKP + (rown ^ 32 * (first + f)), KPL);
#pragma unroll
                            for (int i = 0; i < PAIRS<OP, P>; ++i)
#pragma unroll
                                for (int t = 0; t < CT; ++t) mm<OP, P>(i, x[t], so, qr[t]);
                        }
                    };
                    if (on) {
#pragma unroll
                        for (int t = 0; t < CT; ++t) {
                            x[t] = zero4();
                            et[t] = L.scale * M.e[16 * t + c];
                        }
                        times(0);
                    }
                    if constexpr (SF < DF) {
                        __syncthreads();
                        __syncthreads();    // (the second half is there)
                        if (on) times(SF);
                    }
                }
            }
        } else {
            if constexpr (!chain) {
                if (more) fetch_keys(next);
                if (on) {                   // Q^T (c e dO)
                    f32x4 add[DT];
#pragma unroll
                    for (int d = 0; d < DT; ++d) add[d] = zero4();
                    KeyOp k[2];
                    key_cols(M.q, k[0], 0, 0);
#pragma unroll
                    for (int f = 0; f < CF; ++f) {
                        float y[8];
                        tokens8(y, f);
                        const f32x4 e0 = *reinterpret_cast<const f32x4*>(M.e + 32 * f + 8 * g), e1 = *reinterpret_cast<const f32x4*>(M.e + 32 * f + 8 * g + 4);
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] *= L.scale * (i < 4 ? e0[i % 4] : e1[i % 4]);
                        const Op<3> o3 = op_of<3>(y);
#pragma unroll
                        for (int d2 = 0; d2 < DT; d2 += 4) {
                            const int x = f * (DT / 4) + d2 / 4;
                            if (d2 + 4 < DT) key_cols(M.q, k[(x + 1) & 1], f, d2 + 4);
                            else if (f + 1 < CF) key_cols(M.q, k[(x + 1) & 1], f + 1, 0);
                            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                            for (int i = 0; i < PAIRS<P, 3>; ++i)
#pragma unroll
                                for (int d = 0; d < 4; ++d) mm<P, 3>(i, add[d2 + d], k[x & 1][d], o3);
                        }
                    }
#pragma unroll
                    for (int d = 0; d < DT; ++d) M.add[w][d][lane] = add[d];
                }
            } else {
                if (on) held();
                if (more) fetch_keys(next);
            }
            __syncthreads();                // (Q^T (c e dO) is written)
            if constexpr (!chain) {
                if (more) {
                    fetch_matrices(next);
                    fetch_values(next);
                }
            } else {
                if (!on) continue;
                InvOp a[2];
                Op<3> pa[CT];
                Op<P> go[CF];
                f32x4 fe[CT], fb[CT], fw[CT];
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    pa[t] = op_rows<3>(M.p + Tr::at(t / 2, row_of(0, t & 1, c)) + 32 * (CF - 1) + 8 * g, TPL);
                    fe[t] = factors(M.e, t);
                    fb[t] = factors(M.beta, t);
                    fw[t] = factors(M.w, t);
                }
                inverse(a[0], CT - 2, CF - 1);
#pragma unroll
                for (int t = 0; t < CT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[t][r] *= fw[t][r];
#pragma unroll
                for (int f = 0; f < CF; ++f) {
                    float y[8];
                    tokens8(y, f);
                    go[f] = op_of<P>(y);
                }
                __builtin_amdgcn_sched_barrier(0);
                // c P^T dO: the last 32 tokens reach all rows, the first 32 their own
#pragma unroll
                for (int i = 0; i < PAIRS<3, P>; ++i)
#pragma unroll
                    for (int t = 0; t < CT; ++t) mm<3, P>(i, z[t], pa[t], go[CF - 1]);
                auto written = [&](int f) {
                    record_rows(L.rec_du, f);
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int t = 2 * f + i / 4, r = i % 4;
                        y[i] = R[t][r] * (-fe[t][r] * fb[t][r]);
                    }
                    return op_of<3>(y);
                };
                auto plus = [&] {           // Q^T (c e dO)
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const f32x4 y = M.add[w][d][lane];
#pragma unroll
                        for (int r = 0; r < 4; ++r) S[d][r] += y[r];
                    }
                };
                KeyOp k[2];
                if constexpr (CF == 2) {
                    Op<3> pb[2];
#pragma unroll
                    for (int t = 0; t < 2; ++t) pb[t] = op_rows<3>(M.p + Tr::at(0, row_of(0, t, c)) + 8 * g, TPL);
                    const Op<3> z1 = op_of<3>(z[2], z[3]);
                    inverse(a[1], 0, 1);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < PAIRS<3, P>; ++i)
#pragma unroll
                        for (int t = 0; t < 2; ++t) mm<3, P>(i, z[t], pb[t], go[0]);
                    solve(a[0], 2, z1);
                    const Op<3> z0 = op_of<3>(z[0], z[1]);
                    inverse(a[0], 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    solve(a[1], 0, z1);
                    const Op<3> u1 = written(1);
                    plus();
                    key_cols(M.k, k[0], 1, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    solve(a[0], 0, z0);
                    update(k, 0, u1, false, 1);
                    const Op<3> u0 = written(0);
                    __builtin_amdgcn_sched_barrier(0);
                    update(k, DT / 4, u0, true, 0);
                } else {
                    const Op<3> z0 = op_of<3>(z[0], z[1]);
                    plus();
                    key_cols(M.k, k[0], 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    solve(a[0], 0, z0);
                    const Op<3> u0 = written(0);
                    __builtin_amdgcn_sched_barrier(0);
                    update(k, 0, u0, true, 0);
                }
            }
        }
    }

    if (chain && on) {
        if constexpr (MODE == STATES) {
            const long long at = seg * static_cast<long long>(L.heads) + head;
            record(unit ? L.seg_M + at * dk * dk : L.seg_N + at * cells);
        } else {
            float* dst = BACK ? L.dS0 : L.S_T;
            if (dst != nullptr && (MODE != FWD || seg == L.segments - 1)) record(dst + bh * cells);
            if constexpr (MODE == RECORD) record(L.rec_S + (head * (L.blocks + 1) + all) * cells);
        }
    }
    if constexpr (MODE == FWD) {            // the segment's tokens past the sequence's length
        E* const op = static_cast<E*>(L.o) + b * L.o_s[0] + h * L.o_s[1] + sl * SLICE;
        const long long lo = static_cast<long long>(seg) * L.seg_blocks * C, hi = seg == L.segments - 1 ? L.T : min(lo + static_cast<long long>(L.seg_blocks) * C, static_cast<long long>(L.T));
        if (lane < dv - sl * SLICE)
            for (long long t = (lo < len ? len : lo) + wave; t < hi; t += 2 * NW) Ops<E>::store1(op + t * L.o_s[2] + lane, 0.f);
    }
}

// the scan for a type, padded channels and direction: by two kinds of waves where the LDS holds what they pass on
template <typename E, int DKP, int MODE> struct Scan {
    static constexpr bool PAIR = sizeof(PairMem<E, DKP, MODE>) <= 160 * 1024;
    static constexpr int THREADS = PAIR ? PAIR_NT : NT;
    static constexpr size_t BYTES = PAIR ? sizeof(PairMem<E, DKP, MODE>) : sizeof(Mem<E, DKP, MODE>);
    static_assert(BYTES <= 160 * 1024, "one compute unit's LDS");
    static_assert(PAIR || MODE != STATES, "segments");
    static __device__ __forceinline__ void run(const DeltaLaunch& L, long head, int sl, int seg, unsigned char* smem)
    {
        if constexpr (PAIR) {
            const bool whole = MODE == STATES ? (L.dk | L.dv) % 4 == 0 : L.whole;
            const bool chain = __builtin_amdgcn_readfirstlane(threadIdx.x) < NT;
            if (chain && whole) pair_scan<E, DKP, MODE, true, true>(L, head, sl, seg, smem);
            else if (chain) pair_scan<E, DKP, MODE, true, false>(L, head, sl, seg, smem);
            else if (whole) pair_scan<E, DKP, MODE, false, true>(L, head, sl, seg, smem);
            else pair_scan<E, DKP, MODE, false, false>(L, head, sl, seg, smem);
        } else scan<E, DKP, MODE>(L, head, sl, smem);
    }
};

}  // namespace delta
}  // namespace sfda
