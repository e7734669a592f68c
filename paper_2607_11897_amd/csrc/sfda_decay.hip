// Linear attention with one decay for each head (gfx950): the chunked scan and the decode step.
//
// With lambda = exp(log_decay) of a head, S_i = lambda S_(i-1) + k_i v_i^T and o_i = S_i^T q_i.  For a
// block of C tokens with local indices i, j and the state S before it:
//   O   = (Q K^T . D) V + diag(lambda^(i+1)) Q S,      D_ij = lambda^(i-j) for j <= i, else 0
//   S'  = lambda^C S + sum_j lambda^(C-1-j) k_j v_j^T
// The backward is three scans of the same form (dL/dq forward on (dO, v, k) with the state
// transposed; dL/dk on (v, dO, q) and dL/dv on (k, q, dO) from the last token to the first), run as
// roles of one launch.
#include "sfda_device.h"
#include "sfda_layer.h"

#include <stddef.h>
#include <string.h>

namespace sfda {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 256;                  // threads of a scan workgroup
constexpr int NS = DECAY_SLICE;          // its value columns, 16 for each wave

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

// What the element type decides.  C: tokens of a block; VE: elements of a 16-byte vector; KB: the
// contraction length of one operand fragment; PAD: elements a row in LDS is longer than its channels (keeps
// the 16 rows of a fragment on different banks).
// Lane l of a fragment has index c = l % 16 of the free axis and, of the contraction, the
// places 4 g .. 4 g + 3 (g = l / 16) of each 16: what an accumulator tile holds of its
// rows, so that a tile becomes an operand without leaving its lane.
template <typename E> struct Ops;

template <> struct Ops<uint16_t> {
    static constexpr int C = 64, VE = 8, KB = 32, PAD = 8;
    typedef bf16x8 Frag;
    // row-major [free][contraction]: two 8-byte reads
    static __device__ __forceinline__ Frag rows(const uint16_t* p)
    {
        u32x4 w;
        w.lo = *reinterpret_cast<const u32x2*>(p);
        w.hi = *reinterpret_cast<const u32x2*>(p + 16);
        return __builtin_bit_cast(Frag, w);
    }
    // row-major [contraction][free]: the transposing LDS read takes, from each group of 16 lanes,
    // 4 rows of 16 (lane l: row l / 4, 4 elements from 4 (l % 4)) and gives lane l column l
    static __device__ __forceinline__ Frag cols(const uint16_t* base, int stride, int lane)
    {
        const uint16_t* p = base + (4 * (lane >> 4) + ((lane >> 2) & 3)) * stride + 4 * (lane & 3);
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * stride));
        u32x4 w;
        w.lo = __builtin_bit_cast(u32x2, a);
        w.hi = __builtin_bit_cast(u32x2, b);
        return __builtin_bit_cast(Frag, w);
    }
    // from the accumulator tiles t[0], t[1] whose rows are the contraction
    static __device__ __forceinline__ Frag acc(const f32x4* t)
    {
        u32x4 w = {pack2(t[0][0], t[0][1]), pack2(t[0][2], t[0][3]), pack2(t[1][0], t[1][1]), pack2(t[1][2], t[1][3])};
        return __builtin_bit_cast(Frag, w);
    }
    static __device__ __forceinline__ void mma(f32x4& d, const Frag& a, const Frag& b)
    {
        d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, d, 0, 0, 0);
    }
    static __device__ __forceinline__ void store4(uint16_t* p, const f32x4& x)
    {
        const u32x2 w = {pack2(x[0], x[1]), pack2(x[2], x[3])};
        memcpy(p, &w, 8);
    }
    static __device__ __forceinline__ void store1(uint16_t* p, float x) { *p = f32_to_bf16_bits(x); }
    // the weighted values as a sum of bfloat16 parts: the state has to keep 32 bits' worth of them, and one
    // rounding of the product to bfloat16 would leave 8 bits
    static constexpr int PARTS = 3;
    static __device__ __forceinline__ void weighted(Frag (&out)[PARTS], const Frag& v, const float (&w)[8])
    {
        const u32x4 x = __builtin_bit_cast(u32x4, v);
        u32x4 o[PARTS];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float a = lo_f32(x[e]) * w[2 * e], b = hi_f32(x[e]) * w[2 * e + 1];
#pragma unroll
            for (int s = 0; s < PARTS; ++s) {
                o[s][e] = pack2(a, b);
                if (s + 1 < PARTS) { a -= lo_f32(o[s][e]); b -= hi_f32(o[s][e]); }
            }
        }
#pragma unroll
        for (int s = 0; s < PARTS; ++s) out[s] = __builtin_bit_cast(Frag, o[s]);
    }
};

template <> struct Ops<float> {
    static constexpr int C = 32, VE = 4, KB = 16, PAD = 4;
    typedef f32x4 Frag;
    static __device__ __forceinline__ Frag rows(const float* p) { return *reinterpret_cast<const Frag*>(p); }
    static __device__ __forceinline__ Frag cols(const float* base, int stride, int lane)
    {
        const float* p = base + 4 * (lane >> 4) * stride + (lane & 15);
        return Frag{p[0], p[stride], p[2 * stride], p[3 * stride]};
    }
    static __device__ __forceinline__ Frag acc(const f32x4* t) { return t[0]; }
    static __device__ __forceinline__ void mma(f32x4& d, const Frag& a, const Frag& b)
    {
#pragma unroll
        for (int s = 0; s < 4; ++s) d = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s], b[s], d, 0, 0, 0);
    }
    static __device__ __forceinline__ void store4(float* p, const f32x4& x) { memcpy(p, &x, 16); }
    static __device__ __forceinline__ void store1(float* p, float x) { *p = x; }
    static constexpr int PARTS = 1;
    static __device__ __forceinline__ void weighted(Frag (&out)[PARTS], const Frag& v, const float (&w)[4])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) out[0][e] = v[e] * w[e];
    }
};

// lambda^n as hi + lo.  A state that lives for thousands of blocks is multiplied by the same rounded
// factor each time, and its relative error would add up; with the remainder it does not.
struct Pow { float hi, lo; };
__device__ __forceinline__ Pow decay_pow(int n, float g)
{
    if (n == 0) return {1.f, 0.f};
    const float x = static_cast<float>(n) * g;
    if (x > -0.5f && x < 0.5f) {
        const float e = expm1f(x), h = 1.f + e;
        return {h, e - (h - 1.f)};
    }
    return {expf(x), 0.f};
}

__device__ __forceinline__ int seq_length(const int* lengths, int b, int T)
{
    if (lengths == nullptr) return T;
    const int n = lengths[b];
    return n < 0 ? 0 : n > T ? T : n;
}

// A block's rows of one tensor on their way to LDS: ROWS tokens x COLS channels (COLS padded), 16-byte
// vectors held in registers between the load and the write.  Loads are unconditional and in bounds: rows
// past the block's n are clamped to its last, the vector that would cross a row's end is moved
// back to end with it (the write then goes by elements), and padding is never loaded.
template <typename E, int ROWS, int COLS> struct Tile {
    static constexpr int VE = Ops<E>::VE, VPR = COLS / VE, RPP = NT / VPR, N = ROWS / RPP, STRIDE = COLS + Ops<E>::PAD;
    static_assert(ROWS % RPP == 0 && NT % VPR == 0, "whole passes");
    u32x4 x[N];

    // row i at p + i * st (st may be negative); `cols` channels; n >= 1
    __device__ __forceinline__ void load(const E* p, long long st, int cols, int n, int tid)
    {
        const int col = (tid % VPR) * VE;
        if (cols >= VE) {
            const int at = col + VE <= cols ? col : cols - VE;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int r = tid / VPR + u * RPP;
                memcpy(&x[u], p + (r < n ? r : n - 1) * st + at, 16);
            }
        } else if (col == 0) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int r = tid / VPR + u * RPP;
                E e[VE] = {};
                for (int i = 0; i < VE - 1; ++i)
                    if (i < cols) e[i] = p[(r < n ? r : n - 1) * st + i];
                memcpy(&x[u], e, 16);
            }
        }
    }
    __device__ __forceinline__ void store(E* lds, int cols, int n, int tid) const
    {
        const int col = (tid % VPR) * VE;
        if (col >= cols) return;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int r = tid / VPR + u * RPP;
            const u32x4 z = {0, 0, 0, 0};
            const u32x4 w = r < n ? x[u] : z;
            if (col + VE <= cols || cols < VE) {
                *reinterpret_cast<u32x4*>(lds + r * STRIDE + col) = w;
            } else {
                E e[VE];
                memcpy(e, &w, 16);
#pragma unroll
                for (int i = 0; i < VE; ++i) lds[r * STRIDE + cols - VE + i] = e[i];
            }
        }
    }
};

// LDS of a scan: a block's q, k, v and scores, and the powers of lambda
template <typename E, int DAP> struct Smem {
    static constexpr int C = Ops<E>::C, P = Ops<E>::PAD;
    E q[C * (DAP + P)], k[C * (DAP + P)], v[C * (NS + P)], a[C * (C + P)];
    float pw[C + 1];
};

// One workgroup scans the tokens of one segment of one head for 64 value columns of one role.  Wave w
// owns 16 of the columns: its part of the state stays in accumulator tiles S[d-tile] (rows d, columns n).
// STATES: only the segment's state from zero, to the workspace.
template <typename E, int DAP, bool STATES>
__global__ __launch_bounds__(NT) void decay_scan_kernel(DecayLaunch L)
{
    typedef Ops<E> O;
    typedef typename O::Frag Frag;
    constexpr int C = O::C, KB = O::KB, CT = C / 16, DT = DAP / 16, TPF = KB / 16;   // tiles of 16 in a fragment
    constexpr int SQ = DAP + O::PAD, SV = NS + O::PAD, SA = C + O::PAD;
    constexpr int SCORES = CT * (CT + 1) / 2, SPW = (SCORES + 3) / 4;                // causal score tiles; a wave's
    typedef Smem<E, DAP> Mem;
    extern __shared__ __align__(16) unsigned char smem[];
    Mem& M = *reinterpret_cast<Mem*>(smem);

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    int total = 0;
    for (int r = 0; r < L.roles; ++r) total += L.role[r].slices;
    long bh;
    int sl, ri = 0;
    head_slice(blockIdx.x, total, static_cast<long>(L.B) * L.H, bh, sl);
    while (sl >= L.role[ri].slices) sl -= L.role[ri++].slices;
    const DecayRole& R = L.role[ri];
    const int b = static_cast<int>(bh / L.H), h = static_cast<int>(bh - static_cast<long>(b) * L.H);
    const int seg = blockIdx.y, len = seq_length(L.lengths, b, L.T);
    const long long first = static_cast<long long>(seg) * L.seg_tokens;              // in scan order
    const int begin = first < len ? static_cast<int>(first) : len;
    const int end = first + L.seg_tokens < len ? static_cast<int>(first) + L.seg_tokens : len;
    const int n0 = sl * NS, dbs = R.db - n0 < NS ? R.db - n0 : NS;
    const int da = R.da;
    const float gl = L.log_decay[h];

    // token of scan place i: i, or len - 1 - i
    const int dir = R.reverse ? -1 : 1;
    const long long tok0 = R.reverse ? len - 1 : 0;
    const E* qp = static_cast<const E*>(R.q) + b * R.q_s[0] + h * R.q_s[1];
    const E* kp = static_cast<const E*>(R.k) + b * R.k_s[0] + h * R.k_s[1];
    const E* vp = static_cast<const E*>(R.v) + b * R.v_s[0] + h * R.v_s[1] + n0;
    E* op = static_cast<E*>(R.o) + b * R.o_s[0] + h * R.o_s[1] + n0;
    const long long qst = dir * R.q_s[2], kst = dir * R.k_s[2], vst = dir * R.v_s[2], ost = dir * R.o_s[2];
    qp += tok0 * R.q_s[2];
    kp += tok0 * R.k_s[2];
    vp += tok0 * R.v_s[2];

    {   // padding of the tiles, and the score tiles above the diagonal that a fragment reads, stay zero
        u32x4* z = reinterpret_cast<u32x4*>(smem);
        const u32x4 zero = {0, 0, 0, 0};
        for (int i = tid; i < static_cast<int>(offsetof(Mem, pw)) / 16; i += NT) z[i] = zero;
        if (tid <= C) M.pw[tid] = tid == 0 ? 1.f : expf(static_cast<float>(tid) * gl);
    }

    Tile<E, C, DAP> tq, tk;
    Tile<E, C, NS> tv;
    int n = end - begin < C ? end - begin : C;
    if (n > 0) {
        if (!STATES) tq.load(qp + begin * qst, qst, da, n, tid);
        tk.load(kp + begin * kst, kst, da, n, tid);
        tv.load(vp + begin * vst, vst, dbs, n, tid);
    }

    // the state's tiles: lane (c, g) has rows 16 d + 4 g + r of column 16 w + c
    f32x4 S[DT];
    const int col = 16 * w + c;
    const bool scol = col < dbs;
    {
        const float* src = nullptr;
        long long rs = 0, cs = 0;
        if (!STATES) {
            if (R.ws != nullptr) {
                src = R.ws + (static_cast<long long>(seg) * L.B * L.H + bh) * da * R.db;
                rs = R.db;
                cs = 1;
            } else if (R.S0 != nullptr) {
                src = R.S0 + bh * da * static_cast<long long>(R.db);
                rs = R.s_row;
                cs = R.s_col;
            }
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * d + 4 * g + r;
                S[d][r] = src != nullptr && scol && row < da ? src[row * rs + (n0 + col) * cs] : 0.f;
            }
    }
    __syncthreads();

    // weights that are the same for every whole block: of the scores, of the start state's rows, of the values
    float wd[SPW][4], wi[CT], wv[C / KB][KB / 4];
#pragma unroll
    for (int s = 0; s < SPW; ++s) {
        const int id = w + 4 * s;
        int ti = 0;
        while ((ti + 1) * (ti + 2) / 2 <= id) ++ti;
        const int tj = id - ti * (ti + 1) / 2;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int far = 16 * (ti - tj) + c - (4 * g + r);
            wd[s][r] = far >= 0 && far <= C ? R.intra * M.pw[far] : 0.f;
        }
    }
#pragma unroll
    for (int t = 0; t < CT; ++t) wi[t] = R.inter * M.pw[16 * t + c + (R.reverse ? 0 : 1)];
    auto value_weights = [&](int m) {
#pragma unroll
        for (int f = 0; f < C / KB; ++f)
#pragma unroll
            for (int e = 0; e < KB / 4; ++e) {
                const int j = KB * f + 16 * (e / 4) + 4 * g + (e & 3), far = m - 1 - j + (R.reverse ? 1 : 0);
                wv[f][e] = R.upd * M.pw[far < 0 ? 0 : far];
            }
    };
    value_weights(C);
    Pow lam = decay_pow(C, gl);

    for (int at = begin; at < end; at += C) {
        n = end - at < C ? end - at : C;
        if (!STATES) tq.store(M.q, da, n, tid);
        tk.store(M.k, da, n, tid);
        tv.store(M.v, dbs, n, tid);
        const int next = at + C;
        if (next < end) {
            const int m = end - next < C ? end - next : C;
            if (!STATES) tq.load(qp + next * qst, qst, da, m, tid);
            tk.load(kp + next * kst, kst, da, m, tid);
            tv.load(vp + next * vst, vst, dbs, m, tid);
        }
        if (n < C) {
            value_weights(n);
            lam = decay_pow(n, gl);
        }
        __syncthreads();

        Frag vf[C / KB];
#pragma unroll
        for (int f = 0; f < C / KB; ++f) vf[f] = O::cols(M.v + KB * f * SV + 16 * w, SV, lane);
        if (!STATES) {
            // scores, transposed: rows j, columns i, so that a lane writes four of a row
#pragma unroll
            for (int s = 0; s < SPW; ++s) {
                const int id = w + 4 * s;
                if (id < SCORES) {
                    int ti = 0;
                    while ((ti + 1) * (ti + 2) / 2 <= id) ++ti;
                    const int tj = id - ti * (ti + 1) / 2;
                    f32x4 x = zero4();
#pragma unroll
                    for (int f = 0; f < DAP / KB; ++f)
                        O::mma(x, O::rows(M.k + (16 * tj + c) * SQ + KB * f + 4 * g), O::rows(M.q + (16 * ti + c) * SQ + KB * f + 4 * g));
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = ti > tj || c >= 4 * g + r ? x[r] * wd[s][r] : 0.f;
                    // one rounding to the element type: the scores are an operand of the product with v
                    O::store4(M.a + (16 * ti + c) * SA + 16 * tj + 4 * g, x);
                }
            }
            __syncthreads();

            Frag sf[DAP / KB];      // the state as an operand, rounded to the element type
#pragma unroll
            for (int f = 0; f < DAP / KB; ++f) sf[f] = O::acc(&S[TPF * f]);
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                // O^T: rows n, columns i
                f32x4 x = zero4();
#pragma unroll
                for (int f = 0; f < DAP / KB; ++f)
                    O::mma(x, sf[f], O::rows(M.q + (16 * t + c) * SQ + KB * f + 4 * g));
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] *= wi[t];
#pragma unroll
                for (int f = 0; f < C / KB; ++f)
                    if (KB * f < 16 * (t + 1)) O::mma(x, vf[f], O::rows(M.a + (16 * t + c) * SA + KB * f + 4 * g));
                const int i = 16 * t + c, at_n = 16 * w + 4 * g;
                if (i < n) {
                    E* p = op + (tok0 * R.o_s[2] + (at + i) * ost) + at_n;
                    if (at_n + 4 <= dbs) {
                        O::store4(p, x);
                    } else {
                        for (int r = 0; r < 4; ++r)
                            if (at_n + r < dbs) O::store1(p + r, x[r]);
                    }
                }
            }
        }
        Frag vw[C / KB][O::PARTS];
#pragma unroll
        for (int f = 0; f < C / KB; ++f) O::weighted(vw[f], vf[f], wv[f]);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
#pragma unroll
            for (int r = 0; r < 4; ++r) S[d][r] = __builtin_fmaf(S[d][r], lam.hi, S[d][r] * lam.lo);
#pragma unroll
            for (int f = 0; f < C / KB; ++f) {
                const Frag kf = O::cols(M.k + KB * f * SQ + 16 * d, SQ, lane);
#pragma unroll
                for (int s = O::PARTS - 1; s >= 0; --s) O::mma(S[d], kf, vw[f][s]);
            }
        }
        __syncthreads();
    }

    float* dst = nullptr;
    long long rs = 0, cs = 0;
    if (STATES) {
        dst = R.ws + (static_cast<long long>(seg) * L.B * L.H + bh) * da * R.db;
        rs = R.db;
        cs = 1;
    } else if (seg == L.segments - 1 && R.S_T != nullptr) {
        dst = R.S_T + bh * da * static_cast<long long>(R.db);
        rs = R.s_row;
        cs = R.s_col;
    }
    if (dst != nullptr && scol) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * d + 4 * g + r;
                if (row < da) dst[row * rs + (n0 + col) * cs] = S[d][r];
            }
    }
    if (!STATES && len < L.T) {     // tokens past the sequence's length
        const long long hi = first + L.seg_tokens < L.T ? first + L.seg_tokens : L.T;
        for (long long t = (first < len ? len : first) + w; t < hi; t += NT / 64)
            if (lane < dbs) O::store1(op + t * R.o_s[2] + lane, 0.f);
    }
}

// The segments' states from zero become the states that enter them: one thread for an element of a
// head's state, in place.
__global__ __launch_bounds__(NT) void decay_join_kernel(DecayLaunch L)
{
    const DecayRole& R = L.role[blockIdx.z];
    const long long size = static_cast<long long>(R.da) * R.db, heads = static_cast<long long>(L.B) * L.H;
    const long long at = static_cast<long long>(blockIdx.x) * NT + threadIdx.x, bh = at / size, e = at - bh * size;
    if (bh >= heads) return;
    const int b = static_cast<int>(bh / L.H), h = static_cast<int>(bh - static_cast<long long>(b) * L.H);
    const int len = seq_length(L.lengths, b, L.T);
    const float gl = L.log_decay[h];
    const long long row = e / R.db, col = e - row * R.db;
    float s = R.S0 == nullptr ? 0.f : R.S0[bh * size + row * R.s_row + col * R.s_col];
    const Pow whole = decay_pow(L.seg_tokens, gl);
    float* p = R.ws + bh * size + e;
    for (int i = 0; i < L.segments; ++i, p += heads * size) {
        const long long left = len - static_cast<long long>(i) * L.seg_tokens;
        const Pow lam = left >= L.seg_tokens ? whole : decay_pow(left < 0 ? 0 : static_cast<int>(left), gl);
        const float add = i + 1 < L.segments ? *p : 0.f;
        *p = s;
        s = __builtin_fmaf(s, lam.hi, __builtin_fmaf(s, lam.lo, add));
    }
}

template <typename E, int DAP> hipError_t scan(const DecayLaunch& L, unsigned groups, bool states, hipStream_t st)
{
    constexpr size_t bytes = sizeof(Smem<E, DAP>);
    static_assert(bytes <= 160 * 1024, "one compute unit's LDS");
    if (states)
        hipLaunchKernelGGL((decay_scan_kernel<E, DAP, true>), dim3(groups, L.segments - 1), dim3(NT), bytes, st, L);
    else
        hipLaunchKernelGGL((decay_scan_kernel<E, DAP, false>), dim3(groups, L.segments), dim3(NT), bytes, st, L);
    return hipGetLastError();
}

template <typename E> hipError_t scan_da(const DecayLaunch& L, int da, unsigned groups, bool states, hipStream_t st)
{
    return da <= 64 ? scan<E, 64>(L, groups, states, st) : da <= 128 ? scan<E, 128>(L, groups, states, st)
                                                                      : scan<E, 256>(L, groups, states, st);
}

// ------------------------------------------------------------------ decode step
// S <- lambda S + k v^T, o = scale S^T q.  One workgroup for a head and 16 float4 columns; the 16 row
// groups of a workgroup each take every 16th row, and their parts of o are added through LDS.
constexpr int SW = 64;      // value columns of a workgroup
template <typename E>
__global__ __launch_bounds__(NT) void decay_step_kernel(DecayStepLaunch L, int slices)
{
    __shared__ float part[NT / 16][SW];
    const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4;
    const long long bh = blockIdx.x / slices;
    const int sl = static_cast<int>(blockIdx.x - bh * slices), n = sl * SW + 4 * cg;
    const int b = static_cast<int>(bh / L.H), h = static_cast<int>(bh - static_cast<long long>(b) * L.H);
    const E* q = static_cast<const E*>(L.q) + b * L.q_s[0] + h * L.q_s[1];
    const E* k = static_cast<const E*>(L.k) + b * L.k_s[0] + h * L.k_s[1];
    const E* v = static_cast<const E*>(L.v) + b * L.v_s[0] + h * L.v_s[1];
    float* S = L.S + bh * L.dk * static_cast<long long>(L.dv);
    const Pow lam = decay_pow(1, L.log_decay[h]);
    float vv[4], o[4] = {0.f, 0.f, 0.f, 0.f};
    int m = L.dv - n < 4 ? L.dv - n : 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) vv[e] = e < m ? Elem<E>::load(v, n + e) : 0.f;
    if (m > 0)
        for (int d = rg; d < L.dk; d += NT / 16) {
            float* row = S + static_cast<long long>(d) * L.dv + n;
            const float kd = Elem<E>::load(k, d), qd = Elem<E>::load(q, d);
            f32x4 s = zero4();
            if (m == 4) {
                memcpy(&s, row, 16);
            } else {
                for (int e = 0; e < m; ++e) s[e] = row[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[e] = __builtin_fmaf(s[e], lam.hi, __builtin_fmaf(s[e], lam.lo, kd * vv[e]));
                o[e] = __builtin_fmaf(qd, s[e], o[e]);
            }
            if (m == 4) {
                memcpy(row, &s, 16);
            } else {
                for (int e = 0; e < m; ++e) row[e] = s[e];
            }
        }
#pragma unroll
    for (int e = 0; e < 4; ++e) part[rg][4 * cg + e] = o[e];
    __syncthreads();
    if (tid < SW && sl * SW + tid < L.dv) {
        float x = 0.f;
        for (int i = 0; i < NT / 16; ++i) x += part[i][tid];
        Ops<E>::store1(static_cast<E*>(L.o) + b * L.o_s[0] + h * L.o_s[1] + sl * SW + tid, L.scale * x);
    }
}

}  // namespace

hipError_t launch_decay(const DecayLaunch& L, hipStream_t st)
{
    const long heads = static_cast<long>(L.B) * L.H;
    // roles with the same padded key channels share a launch
    for (int pass = L.segments > 1 ? 0 : 2; pass < 3; ++pass) {
        if (pass == 1) {
            long long most = 0;
            for (int r = 0; r < L.roles; ++r) {
                const long long size = static_cast<long long>(L.role[r].da) * L.role[r].db;
                most = size > most ? size : most;
            }
            hipLaunchKernelGGL(decay_join_kernel, dim3(static_cast<unsigned>((most * heads + NT - 1) / NT), 1, L.roles),
                               dim3(NT), 0, st, L);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            continue;
        }
        for (int lim = 64, low = 0; lim <= 256; low = lim, lim *= 2) {
            DecayLaunch P = L;
            P.roles = 0;
            long slices = 0;
            for (int r = 0; r < L.roles; ++r)
                if (L.role[r].da > low && L.role[r].da <= lim) {
                    P.role[P.roles++] = L.role[r];
                    slices += L.role[r].slices;
                }
            if (P.roles == 0) continue;
            const unsigned groups = static_cast<unsigned>(heads * slices);
            const hipError_t e = L.bf16 ? scan_da<uint16_t>(P, lim, groups, pass == 0, st) : scan_da<float>(P, lim, groups, pass == 0, st);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

hipError_t launch_decay_step(const DecayStepLaunch& L, hipStream_t st)
{
    const int slices = (L.dv + SW - 1) / SW;
    const unsigned groups = static_cast<unsigned>(static_cast<long long>(L.B) * L.H * slices);
    if (L.bf16)
        hipLaunchKernelGGL(decay_step_kernel<uint16_t>, dim3(groups), dim3(NT), 0, st, L, slices);
    else
        hipLaunchKernelGGL(decay_step_kernel<float>, dim3(groups), dim3(NT), 0, st, L, slices);
    return hipGetLastError();
}

}  // namespace sfda
