// Linear attention with one decay for each head (gfx950): the chunked scan and the decode step.
//
// With lambda = exp(log_decay) of a head, S_i = lambda S_(i-1) + k_i v_i^T and o_i = S_i^T q_i.  For a
// block of C tokens with local indices i, j and the state S before it:
//   O   = (Q K^T . D) V + diag(lambda^(i+1)) Q S,      D_ij = lambda^(i-j) for j <= i, else 0
//   S'  = lambda^C S + sum_j lambda^(C-1-j) k_j v_j^T
// The backward is three scans of the same form (dL/dq forward on (dO, v, k) with the state
// transposed; dL/dk on (v, dO, q) and dL/dv on (k, q, dO) from the last token to the first), run as
// roles of one launch.
//
// Times, as calls among others (a call alone, with a wait behind it, takes 12 to 25 us more): B8 H16 d 128, bfloat16 T4096 forward
// 151 to 162 us (by the card) and backward 403 to 409, float32 T2048 forward 234 and backward 626.  A chain of blocks bounds them, 2.4 us for 64 tokens in
// bfloat16: products, LDS reads and vector arithmetic of a block wait for each other with one or two waves on a SIMD.  Below,
// choices are given as ratios of both sides' times, measured in turn on one card.
#include "sfda_device.h"
#include "sfda_layer.h"
#include "sfda_mma.h"

#include <stddef.h>
#include <string.h>

namespace sfda {
namespace {

using namespace mx;

constexpr int NJ = 256;                  // threads of the small kernels

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

// Where a block's rows are: an address that is the same for all lanes and 32-bit offsets of their 16-byte vectors, which
// are the same for every whole block.  The first block of a segment may be short: its tokens then take its last rows,
// and the `pad` rows before them are clamped to its first token, so that loads are unconditional and in bounds.
struct Rows {
    const char* p;          // the sequence's first place in scan order
    long long st;           // bytes from a place to the next (negative: reversed)
    __device__ __forceinline__ const char* base(int at, int n) const { return p + (at + (st < 0 ? n - 1 : 0)) * st; }
    __device__ __forceinline__ uint32_t offset(int row, int pad, int n) const
    {
        const int r = row > pad ? row - pad : 0;
        return static_cast<uint32_t>(st < 0 ? (n - 1 - r) * -st : r * st);
    }
};

// A block's rows of one tensor on their way to LDS: ROWS tokens x COLS channels (COLS padded), 16-byte
// vectors held in registers between the load and the write.  Padding channels are clamped to channel 0, and never written.
// EXACT: the channels are whole vectors.  Otherwise the vector that would cross a row's end is moved back to end with it (into
// the `before` channels that the row has before these, where they are few) and moved into place when it is written, and rows
// shorter than a vector are read by elements.
template <typename E, int NT, int ROWS, int COLS, int STRIDE, bool EXACT> struct Tile {
    static constexpr int VE = Ops<E>::VE, VPR = COLS / VE, RPP = NT / VPR, N = ROWS / RPP, PLANE = ROWS * STRIDE;
    static_assert(ROWS % RPP == 0 && NT % VPR == 0, "whole passes");
    u32x4 x[N];
    uint32_t off, step;     // a whole block's first vector in memory order, and from a pass to the next

    bool few;               // by elements
    int back;               // elements that the lane's vector was moved back

    __device__ __forceinline__ uint32_t at(int cols, int before, int tid) const
    {
        const int col = (tid % VPR) * VE;
        return (before + (col + VE <= cols ? col : EXACT || few ? 0 : cols - VE)) * static_cast<int>(sizeof(E));
    }
    __device__ __forceinline__ void place(const Rows& R, int cols, int before, int tid)
    {
        few = !EXACT && cols + before < VE;
        off = R.offset(tid / VPR + (R.st < 0 ? (N - 1) * RPP : 0), 0, ROWS);
        step = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(RPP * (R.st < 0 ? -R.st : R.st)));
        off += at(cols, before, tid);
        const int past = (tid % VPR) * VE + VE - cols;
        back = EXACT || few || past <= 0 || past >= VE ? 0 : past;
    }
    __device__ __forceinline__ u32x4 one(const From<EXACT>& from, uint32_t o, uint32_t more, int cols, int tid) const
    {
        if constexpr (!EXACT) {
            if (few) return tid % VPR == 0 ? short_row<E>(from.p + more + o, cols) : u32x4{0, 0, 0, 0};
        }
        return from.load(o, more);
    }
    __device__ __forceinline__ void load(const char* base, bool reverse, int cols, int tid)
    {
        const From<EXACT> from(base);
#pragma unroll
        for (int u = 0; u < N; ++u) x[u] = one(from, off, __builtin_amdgcn_readfirstlane((reverse ? N - 1 - u : u) * step), cols, tid);
    }
    // a segment's first block, from its first token on
    __device__ __forceinline__ void load_first(const Rows& R, int begin, int pad, int cols, int before, int tid)
    {
        const From<EXACT> from(R.base(begin, ROWS - pad));
#pragma unroll
        for (int u = 0; u < N; ++u) x[u] = one(from, R.offset(tid / VPR + u * RPP, pad, ROWS - pad) + at(cols, before, tid), 0, cols, tid);
    }
    // rows before `pad` are zero
    template <bool WHOLE> __device__ __forceinline__ void store(uint16_t* lds, int cols, int pad, int tid) const
    {
        int col = (tid % VPR) * VE;
        if (EXACT) col = col < cols ? col : 0;      // (padding lanes hold channel 0's vector, and write it once more)
        else if (col >= cols) return;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int r = tid / VPR + u * RPP;
            const u32x4 z = {0, 0, 0, 0};
            const u32x4 w = WHOLE || r >= pad ? x[u] : z;
            Ops<E>::put(lds + r * STRIDE + col, PLANE, EXACT ? w : move_down<E>(w, back));
        }
    }
};

// A fragment's 16 bytes of a row of `cols` channels, from channel `col` on, on their way from global memory:
// loaded in bounds (as a tile's vectors) and put in place when it is used.  Past the row: zero, but with EXACT what the
// clamped vector holds, the row's own first channels, whose partners in LDS are zero.
template <typename E, bool EXACT> __device__ __forceinline__ uint32_t row_at(int col, int cols)
{
    constexpr int VE = Ops<E>::VE;
    return (col + VE <= cols ? col : EXACT || cols < VE ? 0 : cols - VE) * static_cast<uint32_t>(sizeof(E));
}
template <typename E, bool EXACT> __device__ __forceinline__ u32x4 row_load(const From<EXACT>& from, uint32_t off, int col, int cols)
{
    if constexpr (!EXACT) {
        if (cols < Ops<E>::VE) return col == 0 ? short_row<E>(from.p + off, cols) : u32x4{0, 0, 0, 0};
    }
    return from.load(off, 0);
}
template <typename E, bool EXACT> __device__ __forceinline__ u32x4 row_place(u32x4 x, int col, int cols)
{
    constexpr int VE = Ops<E>::VE;
    if (EXACT) return x;
    const int past = col + VE - cols;
    if (past >= VE) return u32x4{0, 0, 0, 0};
    return move_down<E>(x, past <= 0 || cols < VE ? 0 : past);
}

// A scan workgroup, for the type and the (padded) channels of the state: C tokens of a block, NS value columns, NW waves, KVB
// buffers of keys and values, VP elements that a row of values in LDS is longer (4 rows of 64 bytes, every other 8 of
// them, or of 32 bytes, on different banks).
//  * bfloat16: four waves (one on a SIMD) form no scores and no weighted values twice, eight hide more latency and have
//    half the registers' worth of work each.  B8 H16 T4096 d 128: eight take 1.08 times as long forward, 1.21 times backward (slices
//    of 32 columns: 1.2 times); with 256 channels four do not have the registers.
//  * float32: three planes fill LDS, so that there is one buffer of them and one workgroup on a compute unit; with 256 channels
//    half the block and half the columns.  Four waves with the registers of all (B8 H16 T2048 d 128: eight take 1.09 times as long
//    forward, 1.08 times backward), but eight where rows are not whole vectors, whose address arithmetic they hide (B3 H5
//    T1003 keys of 88, values of 74: four take 1.16 times as long).
template <typename E, int DAP, bool EXACT> struct Shape {
    static constexpr bool HALF = sizeof(E) == 4 && DAP > 128;
    static constexpr int C = HALF ? 32 : 64, NS = decay_slice(sizeof(E) == 2, DAP), NW = (sizeof(E) == 2 ? DAP > 128 : DAP <= 128 && !EXACT) ? 8 : 4;
    static constexpr int KVB = sizeof(E) == 2 ? 2 : 1, VP = NS == 64 ? 32 : 16;
    static constexpr int PER = sizeof(E) == 2 ? 2 : 1;      // workgroups that registers have to allow on a compute unit
};

// LDS of a scan: the keys and values of a block (and of the next), the state as an operand ([column][channel]; twice with SB 2, so
// that a block needs one barrier), and the powers of lambda
template <typename E, int DAP, int SB> struct Smem {
    typedef Shape<E, DAP, true> Sh;
    static constexpr int PL = Ops<E>::PL, SK = DAP + KP, SV = Sh::NS + Sh::VP, SS = DAP + SP;
    static constexpr int KPL = Sh::C * SK, VPL = Sh::C * SV, SPL = Sh::NS * SS;         // planes
    uint16_t k[Sh::KVB][PL * KPL], v[Sh::KVB][PL * VPL], s[SB][PL * SPL];
    float pw[Sh::C + 1];
};

// One workgroup scans the tokens of one segment of one head for NS value columns of one role.  For a block, a wave
// forms the outputs of one row tile (16 of the block's tokens) for 16 NP columns: scores against the keys of earlier
// tiles and its own, kept in registers as the operand of the product with the values, and the queries (which no
// other row tile needs: from global memory straight into fragments) times the state.  Then it updates its share of
// the state, DTW of the channel tiles for 16 columns, and puts it into LDS as the next block's operand.
// STATES: only the segment's state from zero, to the workspace.
// RT: the wave's row tile.  Every wave runs the copy of its own, straight-line code in the loop; all of them have the same barriers, one
// a block (two with one state buffer).
template <typename E, int DAP, int SB, bool STATES, bool EXACT, int RT>
__device__ __forceinline__ void decay_scan(const DecayLaunch& L, const DecayRole R, long bh, int sl, unsigned char* smem, int w)
{
    typedef Ops<E> O;
    typedef typename O::Frag Frag;
    typedef Smem<E, DAP, SB> Mem;
    typedef Shape<E, DAP, EXACT> Sh;
    constexpr int NW = Sh::NW, NS = Sh::NS, NT = 64 * NW, C = Sh::C, VE = O::VE, CT = C / 16, CG = NW / CT, NP = NS / 16 / CG;
    constexpr int DT = DAP / 16, DTW = DT * NP / CT, DF = DAP / KB, CF = C / KB, TPF = KB / 16, ES = sizeof(E), QV = O::QV;
    constexpr int SK = Mem::SK, SV = Mem::SV, SS = Mem::SS, KPL = Mem::KPL, VPL = Mem::VPL, SPL = Mem::SPL;
    constexpr bool WIDE = O::PL > 1, ONE = Sh::KVB == 1;
    static_assert(NP * CG * 16 == NS && CT % NP == 0, "tiles");
    Mem& M = *reinterpret_cast<Mem*>(smem);

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4, cg = w / CT;
    const int b = __builtin_amdgcn_readfirstlane(static_cast<int>(bh / L.H)), h = static_cast<int>(bh - static_cast<long>(b) * L.H);
    const int seg = blockIdx.y, len = __builtin_amdgcn_readfirstlane(seq_length(L.lengths, b, L.T));
    const long long first = static_cast<long long>(seg) * L.seg_tokens;              // in scan order
    const int begin = first < len ? static_cast<int>(first) : len;
    const int end = first + L.seg_tokens < len ? static_cast<int>(first) + L.seg_tokens : len;
    const int n0 = sl * NS, dbs = R.db - n0 < NS ? R.db - n0 : NS;
    const int da = R.da, reverse = R.reverse;
    const float gl = L.log_decay[h];

    // token of scan place i: i, or len - 1 - i
    const long long tok0 = reverse ? len - 1 : 0, dir = reverse ? -ES : ES;
    const Rows qr = {static_cast<const char*>(R.q) + (b * R.q_s[0] + h * R.q_s[1] + tok0 * R.q_s[2]) * ES, dir * R.q_s[2]};
    const Rows kr = {static_cast<const char*>(R.k) + (b * R.k_s[0] + h * R.k_s[1] + tok0 * R.k_s[2]) * ES, dir * R.k_s[2]};
    const Rows vr = {static_cast<const char*>(R.v) + (b * R.v_s[0] + h * R.v_s[1] + tok0 * R.v_s[2]) * ES, dir * R.v_s[2]};
    E* const op = static_cast<E*>(R.o) + b * R.o_s[0] + h * R.o_s[1] + n0;
    const Rows orow = {reinterpret_cast<const char*>(op) + tok0 * R.o_s[2] * ES, dir * R.o_s[2]};

    Tile<E, NT, C, DAP, SK, EXACT> tk;
    Tile<E, NT, C, NS, SV, EXACT> tv;
    u32x4 qn[DF * QV];
    // blocks end where the segment ends; the first one has `pad` rows too many
    const int pad = begin < end ? (C - (end - begin) % C) % C : 0;
    tk.place(kr, da, 0, tid);
    tv.place(vr, dbs, n0, tid);
    auto load_queries = [&](const char* base, uint32_t row) {
        const From<EXACT> from(base);
#pragma unroll
        for (int i = 0; i < DF * QV; ++i) {
            const int col = KB * (i / QV) + 8 * g + VE * (i % QV);
            qn[i] = row_load<E, EXACT>(from, row + row_at<E, EXACT>(col, da), col, da);
        }
    };
    if (begin < end) {
        tk.load_first(kr, begin, pad, da, 0, tid);
        tv.load_first(vr, begin, pad, dbs, n0, tid);
        if (!STATES) load_queries(qr.base(begin, C - pad), qr.offset(16 * RT + c, pad, C - pad));
    }
    const uint32_t qoff = STATES ? 0 : qr.offset(16 * RT + c, 0, C);

#ifdef SFDA_LDS_POISON
    lds_poison(&M, sizeof(Mem), tid, NT);
    __syncthreads();
#endif
    {   // padding stays zero (and with whole rows none is read)
        u32x4* z = reinterpret_cast<u32x4*>(smem);
        const u32x4 zero = {0, 0, 0, 0};
        if (da < DAP || dbs < NS)
            for (int i = tid; i < static_cast<int>(offsetof(Mem, pw)) / 16; i += NT) z[i] = zero;
        if (tid <= C) M.pw[tid] = tid == 0 ? 1.f : expf(static_cast<float>(tid) * gl);
    }

    // the wave's columns: lane c of tile p has column col0 + col_of(p), so that a lane's outputs of two tiles are 8 neighbours
    const int col0 = 16 * NP * cg + (NP == 1 ? c : 8 * (c >> 2) + (c & 3));
    auto col_of = [](int p) { return 32 * (p >> 1) + 4 * (p & 1); };
    // its share of the state: column (c, sp), lane (c, g) has rows srow + 16 d + r
    const int scol = col0 + col_of(RT % NP), srow = 16 * DTW * (RT / NP) + 4 * g;
    f32x4 S[DTW];
    // where the state comes from and goes to: elements of 4 bytes at row * rs + column * cs of da * db; a lane's first one, and
    // what is past the rows or columns nowhere
    constexpr uint32_t NOWHERE = 0x80000000u;
    auto state_at = [&](int rs, int cs) { return scol < dbs ? static_cast<uint32_t>(srow * rs + (n0 + scol) * cs) * 4u : NOWHERE; };
    const long long cells = static_cast<long long>(da) * R.db;
    const long long ws_at = (static_cast<long long>(seg) * L.B * L.H + bh) * cells;
    {
        const float* src = nullptr;
        int rs = 0, cs = 0;
        if (!STATES) {
            src = R.ws != nullptr ? R.ws + ws_at : R.S0 != nullptr ? R.S0 + bh * cells : nullptr;
            rs = R.ws != nullptr ? R.db : static_cast<int>(R.s_row);
            cs = R.ws != nullptr ? 1 : static_cast<int>(R.s_col);
        }
#pragma unroll
        for (int d = 0; d < DTW; ++d) S[d] = zero4();
        if (src != nullptr) {
            const From<true> from(reinterpret_cast<const char*>(src));
            const uint32_t at = state_at(rs, cs);
#pragma unroll
            for (int d = 0; d < DTW; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    S[d][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
                        from.r, srow + 16 * d + r < da ? at : NOWHERE, __builtin_amdgcn_readfirstlane((16 * d + r) * rs * 4), 0));
        }
    }
    __syncthreads();

    // weights that are the same for every whole block: of the scores, of the start state's rows, of the values
    float wd[CT][4], wv[CF][8];
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int far = 16 * (RT - t) + c - (4 * g + r);
            wd[t][r] = far >= 0 ? R.intra * M.pw[far] : 0.f;
        }
    const float upd = R.upd;
#pragma unroll
    for (int f = 0; f < CF; ++f)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            wv[f][e] = upd * M.pw[C - 1 - (KB * f + 16 * (e / 4) + 4 * g + (e & 3)) + (reverse ? 1 : 0)];
    // the first block's decays of the state that enters it are those of its tokens
    const int after = 16 * RT + c + (reverse ? 0 : 1);
    const float wi_whole = R.inter * M.pw[after];
    float wi = R.inter * M.pw[after > pad ? after - pad : 0];
    // hi is what a block multiplies the state by; lo is carried until it moves the rounded factor
    const Pow lam = decay_pow(C, gl), lam_first = pad > 0 ? decay_pow(C - pad, gl) : lam;
    float factor = lam_first.hi, carry = lam_first.lo;
    int low = pad;                  // first row with a token
    const uint32_t ooff = orow.offset(16 * RT + c, 0, C);

    // The state, rounded to the element type (bfloat16), as the operand of its product with the queries; so are the scores below as
    // the operand of theirs with the values.  Both in two parts would leave only the result's own rounding, an error of 0.0017 of the
    // results instead of 0.0023, and take 1.18 times as long forward at B8 H16 T4096 d 128, 1.21 at H16 T65536, 1.33 at B3 H5 T1003, 1.27
    // backward.  The state that is carried on keeps float32 (see `weighted`); float32 tensors have none of these roundings.
    auto state_out = [&](uint16_t* to) {
#pragma unroll
        for (int d = 0; d < DTW; ++d) O::put4(to + scol * SS + srow + 16 * d, SPL, S[d]);
    };
    if (begin < end) {
        tk.template store<false>(M.k[0], da, pad, tid);
        tv.template store<false>(M.v[0], dbs, pad, tid);
        if (!STATES) state_out(M.s[0]);
    }
    __syncthreads();

    constexpr int sp = RT % NP;
    {
        const char *kbase = kr.base(begin - pad, C), *vbase = vr.base(begin - pad, C), *qbase = qr.base(begin - pad, C);
        const char* obase = orow.base(begin - pad, C);
        int buf = 0;
#pragma clang loop unroll(disable)
        for (int at = begin - pad; at < end; at += C, buf ^= 1) {
            const int next = at + C;
            const uint16_t *K = M.k[ONE ? 0 : buf], *V = M.v[ONE ? 0 : buf], *SL = M.s[SB == 2 ? buf : 0];
            // the block's queries as fragments (float32: where they are used, so that the next block's are not requested before)
            auto query = [&](int f) {
                u32x4 v[QV];
#pragma unroll
                for (int i = 0; i < QV; ++i) v[i] = row_place<E, EXACT>(qn[QV * f + i], KB * f + 8 * g + VE * i, da);
                return O::frag(v);
            };
            Frag qf[WIDE ? 1 : DF];
            if (!STATES && !WIDE) {
#pragma unroll
                for (int f = 0; f < DF; ++f) qf[f] = query(f);
            }
            if (next < end) {
                kbase += kr.st * C;
                vbase += vr.st * C;
                qbase += qr.st * C;
                tk.load(kbase, reverse, da, tid);
                tv.load(vbase, reverse, dbs, tid);
                if (!STATES && !WIDE) load_queries(qbase, qoff);
            }
            auto values = [&](int f, int p) {
                return O::cols(V + KB * f * SV + 16 * NP * cg + col_of(p) + cols_at(SV, NP == 1 ? 4 : 8, c, g), SV, VPL);
            };
            Frag vf[CF][NP];
            if (!WIDE) {
#pragma unroll
                for (int f = 0; f < CF; ++f)
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        if ((!STATES && TPF * f <= RT) || p == sp) vf[f][p] = values(f, p);
            }
            if (!STATES) {
                // outputs, transposed: rows are columns of v, columns are tokens
                f32x4 x[NP];
#pragma unroll
                for (int p = 0; p < NP; ++p) x[p] = zero4();
                // scores, transposed: rows are keys; rounded once to the element type (bfloat16), as the operand of the product
                // with v
                constexpr int ST = TPF * ((RT + TPF) / TPF);
                f32x4 sc[ST];
#pragma unroll
                for (int t = 0; t < ST; ++t) sc[t] = zero4();
                auto states = [&](int f, int p) { return O::rows(SL + (col0 + col_of(p)) * SS + KB * f + 8 * g, SPL); };
                auto key_rows = [&](int f, int t) { return O::rows(K + (16 * t + c) * SK + KB * f + 8 * g, KPL); };
                if constexpr (WIDE) {
#pragma unroll
                    for (int f = 0; f < DF; ++f) {
                        Frag sf[NP], kf[RT + 1];
#pragma unroll
                        for (int p = 0; p < NP; ++p) sf[p] = states(f, p);
#pragma unroll
                        for (int t = 0; t <= RT; ++t) kf[t] = key_rows(f, t);
                        const Frag q = query(f);
#pragma unroll
                        for (int i = 0; i < O::PAIRS; ++i) {
#pragma unroll
                            for (int p = 0; p < NP; ++p) O::mma(i, x[p], sf[p], q);
#pragma unroll
                            for (int t = 0; t <= RT; ++t) O::mma(i, sc[t], kf[t], q);
                        }
                    }
                    if (next < end) load_queries(qbase, qoff);
                } else {
#pragma unroll
                    for (int f = 0; f < DF; ++f)
#pragma unroll
                        for (int p = 0; p < NP; ++p) O::mma(0, x[p], states(f, p), qf[f]);
                    __builtin_amdgcn_sched_barrier(0);     // (phases kept apart: mixed, they measure 2 to 5% more)
#pragma unroll
                    for (int f = 0; f < DF; ++f)
#pragma unroll
                        for (int t = 0; t <= RT; ++t) O::mma(0, sc[t], key_rows(f, t), qf[f]);
                }
#pragma unroll
                for (int t = 0; t <= RT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[t][r] = t < RT || c >= 4 * g + r ? sc[t][r] * wd[t][r] : 0.f;
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[p][r] *= wi;
#pragma unroll
                for (int f = 0; TPF * f <= RT; ++f) {
                    const Frag a = O::acc(&sc[TPF * f]);
                    if constexpr (WIDE) {
#pragma unroll
                        for (int p = 0; p < NP; ++p) vf[f][p] = values(f, p);
                    }
#pragma unroll
                    for (int i = 0; i < O::PAIRS; ++i)
#pragma unroll
                        for (int p = 0; p < NP; ++p) O::mma(i, x[p], vf[f][p], a);
                }
                __builtin_amdgcn_sched_barrier(0);
                const From<EXACT> out(obase);
                const bool row = 16 * RT + c >= low;
                constexpr int PN = NP == 1 ? 4 : 8;         // neighbours
#pragma unroll
                for (int u = 0; u < (NP + 1) / 2; ++u) {
                    const int at_n = 16 * NP * cg + 32 * u + PN * g;
                    const uint32_t off = ooff + at_n * ES;
                    if constexpr (EXACT) {      // (stores past the resource's range are dropped)
                        if constexpr (ES == 2) {
                            out.store(row && at_n < dbs ? off : NOWHERE, 0, O::pack8(x[2 * u], x[2 * u + 1]));
                        } else {
                            out.store(row && at_n < dbs ? off : NOWHERE, 0, __builtin_bit_cast(u32x4, x[2 * u]));
                            if constexpr (NP > 1)
                                out.store(row && at_n + 4 < dbs ? off + 16 : NOWHERE, 0, __builtin_bit_cast(u32x4, x[2 * u + 1]));
                        }
                    } else if (row && at_n + PN <= dbs) {
                        if constexpr (ES == 2) {
                            out.store(off, 0, O::pack8(x[2 * u], x[2 * u + 1]));
                        } else {
                            out.store(off, 0, __builtin_bit_cast(u32x4, x[2 * u]));
                            if constexpr (NP > 1) out.store(off, 16, __builtin_bit_cast(u32x4, x[2 * u + 1]));
                        }
                    } else if (row) {
                        E* to = reinterpret_cast<E*>(const_cast<char*>(obase) + off);
                        int left = dbs - at_n;
                        asm("" : "+v"(left));       // (or the masks of the stores are kept over the blocks, and spilled)
#pragma unroll
                        for (int i = 0; i < PN; ++i)
                            if (i < left) O::store1(to + i, x[2 * u + i / 4][i % 4]);
                    }
                }
                obase += orow.st * C;
                if (SB == 1 && !ONE) __syncthreads();
                wi = wi_whole;
                low = 0;
            }
#pragma unroll
            for (int d = 0; d < DTW; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[d][r] *= factor;
#pragma unroll
            for (int f = 0; f < CF; ++f) {
                Frag vw[O::PARTS];
                auto keys = [&](int d) { return O::cols(K + KB * f * SK + srow - 4 * g + 16 * d + cols_at(SK, 4, c, g), SK, KPL); };
                Frag kf[DTW];
#pragma unroll
                for (int d = 0; d < DTW; ++d) kf[d] = keys(d);
                if constexpr (WIDE) vf[f][sp] = values(f, sp);
                O::weighted(vw, vf[f][sp], wv[f]);
#pragma unroll
                for (int s = O::PARTS - 1; s >= 0; --s)
#pragma unroll
                    for (int i = 0; i < O::PAIRS; ++i)
#pragma unroll
                        for (int d = 0; d < DTW; ++d) O::mma(i, S[d], kf[d], vw[s]);
            }
            carry += lam.lo;
            factor = lam.hi + carry;
            carry -= factor - lam.hi;
            // (after the last block what is written is not read: no branch splits the block's instructions)
            if (ONE) __syncthreads();
            if (EXACT || next < end) {
                if (!STATES) state_out(M.s[SB == 2 ? buf ^ 1 : 0]);
                tk.template store<true>(M.k[ONE ? 0 : buf ^ 1], da, 0, tid);
                tv.template store<true>(M.v[ONE ? 0 : buf ^ 1], dbs, 0, tid);
            }
            __syncthreads();
        }
    }

    float* dst = nullptr;
    int rs = R.db, cs = 1;
    if (STATES) {
        dst = R.ws + ws_at;
    } else if (seg == L.segments - 1 && R.S_T != nullptr) {
        dst = R.S_T + bh * cells;
        rs = static_cast<int>(R.s_row);
        cs = static_cast<int>(R.s_col);
    }
    if (dst != nullptr) {
        const From<true> to(reinterpret_cast<const char*>(dst));
        const uint32_t at = state_at(rs, cs);
#pragma unroll
        for (int d = 0; d < DTW; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[d][r]), to.r, srow + 16 * d + r < da ? at : NOWHERE,
                                                      __builtin_amdgcn_readfirstlane((16 * d + r) * rs * 4), 0);
    }
    if (!STATES && len < L.T) {     // tokens past the sequence's length
        const long long hi = first + L.seg_tokens < L.T ? first + L.seg_tokens : L.T;
        for (long long t = (first < len ? len : first) + w; t < hi; t += NW)
            if (lane < dbs) O::store1(op + t * R.o_s[2] + lane, 0.f);
    }
}

template <typename E, int DAP, int SB, bool STATES, bool EXACT>
__global__ __launch_bounds__((64 * Shape<E, DAP, EXACT>::NW), (Shape<E, DAP, EXACT>::PER)) void decay_scan_kernel(DecayLaunch L)
{
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int CT = Shape<E, DAP, EXACT>::C / 16;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (waves w and w + 4 share a SIMD: their row tiles add up to the same number of score tiles)
    const int rt = CT == 2 ? w & 1 : w < 4 ? w : 7 - w;
    // (the roles are told apart by constants: an argument indexed at run time would be copied to memory, and its fields would no
    // longer be known to be the same for all lanes; divisions run on the vector unit, with the same result)
    int total = 0;
#pragma unroll
    for (int r = 0; r < DECAY_ROLES; ++r) total += r < L.roles ? L.role[r].slices : 0;
    long bh;
    int sl;
    head_slice(blockIdx.x, total, static_cast<long>(L.B) * L.H, bh, sl);
    bh = static_cast<long>(same_for_all(static_cast<uint64_t>(bh)));
    sl = __builtin_amdgcn_readfirstlane(sl);
    DecayRole R = L.role[0];
    if (sl >= R.slices && L.roles > 1) {
        sl -= R.slices;
        R = L.role[1];
        if (sl >= R.slices && L.roles > 2) {
            sl -= R.slices;
            R = L.role[2];
        }
    }
    if (rt == 0) decay_scan<E, DAP, SB, STATES, EXACT, 0>(L, R, bh, sl, smem, w);
    else if (CT == 2 || rt == 1) decay_scan<E, DAP, SB, STATES, EXACT, 1>(L, R, bh, sl, smem, w);
    else if (rt == 2) decay_scan<E, DAP, SB, STATES, EXACT, CT == 4 ? 2 : 0>(L, R, bh, sl, smem, w);
    else decay_scan<E, DAP, SB, STATES, EXACT, CT == 4 ? 3 : 0>(L, R, bh, sl, smem, w);
}

// The segments' states from zero become the states that enter them: one thread for an element of a
// head's state, in place; eight segments' values are requested at a time.  6 us for 32 states of 128 x 128 in 4 segments.
__global__ __launch_bounds__(NJ) void decay_join_kernel(DecayLaunch L)
{
    const DecayRole R = blockIdx.z == 0 ? L.role[0] : blockIdx.z == 1 ? L.role[1] : L.role[2];
    const unsigned size = static_cast<unsigned>(R.da) * R.db, heads = static_cast<unsigned>(L.B) * L.H;
    const unsigned at = blockIdx.x * NJ + threadIdx.x, bh = at / size, e = at - bh * size;
    if (bh >= heads) return;
    const int b = static_cast<int>(bh / static_cast<unsigned>(L.H)), h = static_cast<int>(bh - static_cast<unsigned>(b) * L.H);
    const int len = seq_length(L.lengths, b, L.T);
    const float gl = L.log_decay[h];
    const unsigned row = e / R.db, col = e - row * R.db;
    float s = R.S0 == nullptr ? 0.f : R.S0[bh * static_cast<long long>(size) + row * R.s_row + col * R.s_col];
    const Pow whole = decay_pow(L.seg_tokens, gl);
    const long long step = static_cast<long long>(heads) * size;
    float* p = R.ws + bh * static_cast<long long>(size) + e;
    constexpr int K = 8;
    for (int i = 0; i < L.segments; i += K, p += K * step) {
        float add[K];
#pragma unroll
        for (int k = 0; k < K; ++k) add[k] = i + k + 1 < L.segments ? p[k * step] : 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (i + k >= L.segments) break;
            const long long left = len - static_cast<long long>(i + k) * L.seg_tokens;
            const Pow lam = left >= L.seg_tokens ? whole : decay_pow(left < 0 ? 0 : static_cast<int>(left), gl);
            p[k * step] = s;
            s = __builtin_fmaf(s, lam.hi, __builtin_fmaf(s, lam.lo, add[k]));
        }
    }
}

template <typename E, int DAP, int SB, bool STATES, bool EXACT> hipError_t scan_sb(const DecayLaunch& L, unsigned groups, hipStream_t st)
{
    constexpr size_t bytes = sizeof(Smem<E, DAP, SB>);
    static_assert(bytes <= 160 * 1024, "one compute unit's LDS");
    hipLaunchKernelGGL((decay_scan_kernel<E, DAP, SB, STATES, EXACT>), dim3(groups, STATES ? L.segments - 1 : L.segments),
                       dim3(64 * Shape<E, DAP, EXACT>::NW), bytes, st, L);
    return hipGetLastError();
}

// One state buffer or two.  Two where a second workgroup fits beside it all the same, or where there is none: with
// bfloat16 and 128 channels one buffer lets two workgroups share a compute unit (B8 H16 T4096 forward, 256 workgroups:
// one buffer takes 1.06 times as long; backward, 768 workgroups: two take 1.05 times as long).  The segments' states need no buffer.
template <typename E, int DAP, bool STATES, bool EXACT> hipError_t scan(const DecayLaunch& L, unsigned groups, hipStream_t st)
{
    constexpr size_t HALF = 80 * 1024;
    if constexpr (Shape<E, DAP, EXACT>::KVB == 1)
        return scan_sb<E, DAP, 1, STATES, EXACT>(L, groups, st);
    else if constexpr (!STATES && sizeof(Smem<E, DAP, 2>) <= HALF)
        return scan_sb<E, DAP, 2, STATES, EXACT>(L, groups, st);
    else if constexpr (!STATES && sizeof(Smem<E, DAP, 1>) <= HALF)
        return static_cast<long long>(groups) * L.segments <= L.cus ? scan_sb<E, DAP, 2, STATES, EXACT>(L, groups, st)
                                                                    : scan_sb<E, DAP, 1, STATES, EXACT>(L, groups, st);
    else
        return scan_sb<E, DAP, 1, STATES, EXACT>(L, groups, st);
}

template <typename E, bool STATES, bool EXACT> hipError_t scan_da(const DecayLaunch& L, int da, unsigned groups, hipStream_t st)
{
    return da <= 64 ? scan<E, 64, STATES, EXACT>(L, groups, st) : da <= 128 ? scan<E, 128, STATES, EXACT>(L, groups, st)
                                                                             : scan<E, 256, STATES, EXACT>(L, groups, st);
}

// EXACT where every role's channels are whole 16-byte vectors at 4-byte addresses: the general kernels' loads and stores by
// parts, and their 64-bit addresses, cost them registers and instructions
template <typename E> bool exact(const void* p, const long long (&st)[3], int n)
{
    constexpr long long ES = sizeof(E);
    if (n % Ops<E>::VE != 0 || reinterpret_cast<uintptr_t>(p) % 4 != 0) return false;
    for (long long s : st)
        if (s * ES % 4 != 0) return false;
    return true;
}
template <typename E> hipError_t scan_any(const DecayLaunch& L, int da, unsigned groups, bool states, hipStream_t st)
{
    bool all = true;
    for (int r = 0; r < L.roles; ++r) {
        const DecayRole& R = L.role[r];
        all = all && exact<E>(R.q, R.q_s, R.da) && exact<E>(R.k, R.k_s, R.da) && exact<E>(R.v, R.v_s, R.db) && exact<E>(R.o, R.o_s, R.db);
    }
    if (all) return states ? scan_da<E, true, true>(L, da, groups, st) : scan_da<E, false, true>(L, da, groups, st);
    return states ? scan_da<E, true, false>(L, da, groups, st) : scan_da<E, false, false>(L, da, groups, st);
}

// ------------------------------------------------------------------ decode step
// S <- lambda S + k v^T, o = scale S^T q.  One workgroup for a head and 16 float4 columns; the 16 row
// groups of a workgroup each take every 16th row, and their parts of o are added through LDS.  Memory-bound:
// float32, 16384 states of 128 x 128: 412 us for 2.18 GB read and written, 5.3 TB/s (a large copy: 4.8).
constexpr int SW = 64;      // value columns of a workgroup
template <typename E>
__global__ __launch_bounds__(NJ) void decay_step_kernel(DecayStepLaunch L, int slices)
{
    __shared__ float part[NJ / 16][SW];
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
        for (int d = rg; d < L.dk; d += NJ / 16) {
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
        for (int i = 0; i < NJ / 16; ++i) x += part[i][tid];
        Ops<E>::store1(static_cast<E*>(L.o) + b * L.o_s[0] + h * L.o_s[1] + sl * SW + tid, L.scale * x);
    }
}

}  // namespace

hipError_t launch_decay(const DecayLaunch& L, hipStream_t st)
{
    const long heads = static_cast<long>(L.B) * L.H;
    // Roles with the same padded channels of the state share a launch.  All of them do, with the padding of the largest, where
    // that leaves each workgroup a compute unit: launches one after the other add up their latencies (backward float32
    // B2 H6 T509, keys of 72 and values of 58 channels: two take 1.5 times as long).
    int widest = 64;
    for (int r = 0; r < L.roles; ++r)
        while (L.role[r].da > widest) widest *= 2;
    long all = 0;
    for (int r = 0; r < L.roles; ++r) all += heads * decay_slices(L.bf16, widest, L.role[r].db) * L.segments;
    const int narrowest = all <= L.cus ? widest : 64;
    for (int pass = L.segments > 1 ? 0 : 2; pass < 3; ++pass) {
        if (pass == 1) {
            long long most = 0;
            for (int r = 0; r < L.roles; ++r) {
                const long long size = static_cast<long long>(L.role[r].da) * L.role[r].db;
                most = size > most ? size : most;
            }
            hipLaunchKernelGGL(decay_join_kernel, dim3(static_cast<unsigned>((most * heads + NJ - 1) / NJ), 1, L.roles),
                               dim3(NJ), 0, st, L);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            continue;
        }
        for (int lim = narrowest, low = 0; lim <= widest; low = lim, lim *= 2) {
            DecayLaunch P = L;
            P.roles = 0;
            long slices = 0;
            for (int r = 0; r < L.roles; ++r)
                if (L.role[r].da > low && L.role[r].da <= lim) {
                    P.role[P.roles++] = L.role[r];
                    slices += P.role[P.roles - 1].slices = decay_slices(L.bf16, lim, L.role[r].db);
                }
            if (P.roles == 0) continue;
            const unsigned groups = static_cast<unsigned>(heads * slices);
            const hipError_t e = L.bf16 ? scan_any<uint16_t>(P, lim, groups, pass == 0, st) : scan_any<float>(P, lim, groups, pass == 0, st);
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
        hipLaunchKernelGGL(decay_step_kernel<uint16_t>, dim3(groups), dim3(NJ), 0, st, L, slices);
    else
        hipLaunchKernelGGL(decay_step_kernel<float>, dim3(groups), dim3(NJ), 0, st, L, slices);
    return hipGetLastError();
}

}  // namespace sfda
