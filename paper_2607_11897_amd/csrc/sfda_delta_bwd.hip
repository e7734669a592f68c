// The gated delta rule's backward (gfx950).  With the notation of the scan, u = beta R the writes and dv = beta du:
//   dbeta_i = du_i . R_i,   dq = c e dO S^T + (c D . dO u^T) K,
//   dk = w u U^T - e dv S^T + (c D . dO u^T)^T Q - (M + M^T) K,   M_ij = D_ij dv_i . u_j  (j < i).
// A log decay at token t scales what the outputs from t on read and what their writes cancel: with G the sum of the log decays,
// dL/dG_t = dO_t . o_t - v_t . dv_t, and what the state after the block carries on is S' . U, so that
//   dlog_decay_t = S' . U + sum_(s >= t, in the block) (dO_s . o_s - v_s . dv_s).
// Three launches after the inverses: the forward scan again, which records the states and the rows R, and the adjoint scan,
// which records U and du, side by side as roles of one; then all blocks at once form the products above.
// bfloat16 B8 H16 T4096 of 128 channels: inverses and scores 250 us, scans 900 (256 compute units, each a head's 64 columns of one
// direction after the other's), gradients 1130.
#include "sfda_delta.h"

#include <type_traits>

namespace sfda {
namespace delta {

hipError_t prep(const DeltaLaunch& L, int inverses, hipStream_t st);

namespace {

template <typename E, int DKP> struct Scans {
    typedef Scan<E, DKP, RECORD> Rec;
    typedef Scan<E, DKP, ADJOINT> Adj;
    static_assert(Rec::THREADS == Adj::THREADS, "roles of one launch");
    static constexpr int THREADS = Rec::THREADS;
    static constexpr size_t BYTES = Rec::BYTES > Adj::BYTES ? Rec::BYTES : Adj::BYTES;
};

template <typename E, int DKP> __global__ __launch_bounds__((Scans<E, DKP>::THREADS)) void sfda_delta_scans(DeltaLaunch L, int slices)
{
    extern __shared__ __align__(16) unsigned char smem[];
    long head;
    int sl;
    head_slice(blockIdx.x, slices, L.heads, head, sl);
    head = static_cast<long>(same_for_all(static_cast<uint64_t>(head)));
    sl = __builtin_amdgcn_readfirstlane(sl);
    if (blockIdx.y == 0) Scans<E, DKP>::Rec::run(L, head, sl, 0, smem);
    else Scans<E, DKP>::Adj::run(L, head, sl, 0, smem);
}

// ------------------------------------------------------------------ the blocks' gradients

constexpr int SLAB = 64;        // value columns at a time

template <typename E, int DKP> struct GradMem {
    typedef Block<E> B;
    static constexpr int NW = DKP == 64 ? 4 : 8, NT = 64 * NW;
    // SP: parts of the states, of the rows of dv and u, and of the scores.  bfloat16: two of each leave dq and dk their own rounding, 0.0017 of
    // themselves; the rows and scores in one part 0.0022, and up to 0.011 where keys are alike and terms cancel
    static constexpr int C = B::C, P = B::P, SP = P == 1 ? 2 : 3, SK = DKP + 16, SV = SLAB + 8, ST = C + 8;
    static constexpr int KPL = C * SK, VPL = C * SV, TPL = C * ST;
    union {
        // dO, dv, u, and dv times -e, u times w: [token][value column]
        struct { uint16_t o[P * VPL], v[SP * VPL], u[SP * VPL], ev[SP * VPL], wu[SP * VPL]; } row;
        struct { uint16_t k[P * KPL], q[P * KPL]; } key;
    };
    uint16_t w[SP * TPL], m[SP * TPL];                                  // c D . dO u^T, and -(M + M^T): [i][j]
    float e[C], wt[C], beta[C], gh[C], gl[C], db[C], vd[C], dot[NW], od[NT];
};

// 4 neighbours of a row of n elements from column `col` on, zeros past them and where the row is not there (its address has to be one);
// WHOLE: n is a multiple of 4.  Without branches, so that loads go out together.
template <bool WHOLE, typename T> __device__ __forceinline__ f32x4 four(const T* row, int col, int n, bool there)
{
    f32x4 x;
    if constexpr (WHOLE) {
        const T* p = row + (col < n ? col : 0);
        there = there && col < n;
        if constexpr (sizeof(T) == 4) {
            memcpy(&x, p, 16);
        } else {
            u32x2 y;
            memcpy(&y, p, 8);
            x = f32x4{lo_f32(y[0]), hi_f32(y[0]), lo_f32(y[1]), hi_f32(y[1])};
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = there ? x[i] : 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = col + i < n ? col + i : n - 1;
            const float y = value<T>(reinterpret_cast<const char*>(row + at));
            x[i] = there && col + i < n ? y : 0.f;
        }
    }
    return x;
}
template <typename E> __device__ __forceinline__ void put_four(E* row, int col, int n, const f32x4& x)
{
    if (col + 4 <= n) {
        if constexpr (sizeof(E) == 4) {
            memcpy(row + col, &x, 16);
        } else {
            const u32x2 y = {pack2(x[0], x[1]), pack2(x[2], x[3])};
            memcpy(row + col, &y, 8);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (col + i < n) Ops<E>::store1(row + col + i, x[i]);
    }
}

// (what is computed from it is not kept over the loops: spilled, it took 1.9 of the 2.3 GB that the kernel wrote)
__device__ __forceinline__ int thread() { return anew(threadIdx.x); }

// One workgroup for a block of a key head, its value heads one after the other.  A wave owns one or two tiles of 16 channels of dq and dk
// (rows; tokens are the columns), whose rows of the states it alone reads.  Reads three states, R and du, 3.0 GB at the size above, and
// writes 0.4: 3.0 TB/s, since the registers leave a compute unit one workgroup (at half of them 127 to 263 spill; four waves with two tiles
// each spill 147), whose loads and products overlap little (waves wait 69% of their time, matrix units are busy 8%).  Neighbouring blocks on one XCD, for the state that both read: no gain (1012 us).
template <typename E, int DKP> __global__ __launch_bounds__((GradMem<E, DKP>::NT)) void sfda_delta_grad(DeltaLaunch L)
{
    typedef Block<E> B;
    typedef GradMem<E, DKP> M_;
    constexpr int NW = M_::NW, NT = M_::NT, C = B::C, CT = B::CT, CF = B::CF, P = B::P, ES = sizeof(E), DW = DKP / 16 / NW;
    constexpr int SP = M_::SP, SK = M_::SK, SV = M_::SV, ST = M_::ST, KPL = M_::KPL, VPL = M_::VPL, TPL = M_::TPL;
    constexpr int RPP = NT / (SLAB / 4), N = C / RPP, TW = (CT * CT + NW - 1) / NW;    // rows of a pass, passes, tiles of scores of a wave
    extern __shared__ __align__(16) unsigned char smem[];
    M_& M = *reinterpret_cast<M_*>(smem);

    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned group = blockIdx.x / static_cast<unsigned>(L.blocks);
    const int blk = static_cast<int>(blockIdx.x - group * static_cast<unsigned>(L.blocks)), per = L.H / L.Hk;
    const long long key = L.first / per + group;
    const int b = __builtin_amdgcn_readfirstlane(static_cast<int>(key / L.Hk)), hk = __builtin_amdgcn_readfirstlane(static_cast<int>(key - static_cast<long long>(b) * L.Hk));
    const int len = __builtin_amdgcn_readfirstlane(seq_length(L.lengths, b, L.T));
    const int t0 = blk * C, rows = L.T - t0 < C ? L.T - t0 : C, cnt = len - t0 < 0 ? 0 : len - t0 < C ? len - t0 : C;
    const int dk = L.dk, dv = L.dv;
    const long long cells = static_cast<long long>(dk) * dv;
    const bool whole = dv % 4 == 0;

    E* const dqp = static_cast<E*>(L.dq) + b * L.dq_s[0] + hk * L.dq_s[1] + t0 * L.dq_s[2];
    E* const dkp = static_cast<E*>(L.dk_out) + b * L.dk_s[0] + hk * L.dk_s[1] + t0 * L.dk_s[2];
    f32x4 dq[DW][CT], dkk[DW][CT];
#pragma unroll
    for (int i = 0; i < DW; ++i)
#pragma unroll
        for (int t = 0; t < CT; ++t) dq[i][t] = dkk[i][t] = zero4();

#ifdef SFDA_LDS_POISON
    lds_poison(&M, sizeof(M_), threadIdx.x, NT);
    __syncthreads();
#endif
    {   // the upper tiles of c D . dO u^T stay zero
        const int tid = thread();
        u32x4* z = reinterpret_cast<u32x4*>(M.w);
        const u32x4 zero = {0, 0, 0, 0};
        for (int i = tid; i < SP * TPL / 8; i += NT) z[i] = zero;
    }

    for (int j = 0; j < per; ++j) {
        const long head = static_cast<long>(group) * per + j;
        const int h = hk * per + j;
        const float* const S = L.rec_S + (head * (L.blocks + 1) + blk) * cells;
        const float* const U = L.rec_U + (head * L.blocks + blk) * cells;
        const long long row0 = head * (static_cast<long long>(L.blocks) * C) + t0;
        const E* const vp = static_cast<const E*>(L.v) + b * L.v_s[0] + h * L.v_s[1] + t0 * L.v_s[2];
        const E* const gp = static_cast<const E*>(L.dO) + b * L.g_s[0] + h * L.g_s[1] + t0 * L.g_s[2];
        E* const dvp = static_cast<E*>(L.dv_out) + b * L.dv_s[0] + h * L.dv_s[1] + t0 * L.dv_s[2];
        float* const dlp = L.dlog_decay + b * L.dl_s[0] + h * L.dl_s[1] + t0 * L.dl_s[2];
        float* const dbp = L.dbeta + b * L.db_s[0] + h * L.db_s[1] + t0 * L.db_s[2];

        const int tid = thread();
        if (cnt == 0) {                 // nothing there: zeros
            for (int i = tid; i < rows * SLAB / 4; i += NT)
                for (int col = 4 * (i % (SLAB / 4)); col < dv; col += SLAB) put_four(dvp + (i / (SLAB / 4)) * L.dv_s[2], col, dv, zero4());
            if (tid < rows) dlp[tid * L.dl_s[2]] = dbp[tid * L.db_s[2]] = 0.f;
            continue;
        }
        RowTile<E, DKP, C, SK, NT> tk, tq;
        auto keys = [&] {
            tk.load(reinterpret_cast<const char*>(static_cast<const E*>(L.k) + b * L.k_s[0] + hk * L.k_s[1] + t0 * L.k_s[2]), static_cast<uint32_t>(L.k_s[2] * ES), cnt, dk, tid);
            tq.load(reinterpret_cast<const char*>(static_cast<const E*>(L.q) + b * L.q_s[0] + hk * L.q_s[1] + t0 * L.q_s[2]), static_cast<uint32_t>(L.q_s[2] * ES), cnt, dk, tid);
        };
        if (DW == 1) keys();            // (ahead where there are the registers, here and below)

        float4 sc[2];
        float decay = 0.f, od = 0.f;
        if (tid < C) {
            sc[0] = L.scalars[2 * (row0 + tid)];
            sc[1] = L.scalars[2 * (row0 + tid) + 1];
            decay = L.log_decay[b * L.l_s[0] + h * L.l_s[1] + (t0 + (tid < cnt ? tid : 0)) * L.l_s[2]];
        }
        for (int p = tid / C; p < L.parts; p += NT / C)         // (a part of 16 columns for a thread, or two)
            od += tid % C < cnt ? L.odo[(head * L.parts + p) * (static_cast<long long>(L.blocks) * C) + t0 + tid % C] : 0.f;
        __syncthreads();                // (the last head's tokens and keys are read)
        M.od[tid] = od;
        if (tid < C) {
            M.gh[tid] = sc[0].x;
            M.gl[tid] = sc[0].y;
            M.beta[tid] = sc[0].z;
            M.e[tid] = sc[0].w;
            M.wt[tid] = sc[1].x;
        }
        float dot = 0.f;
        f32x4 held[DW][CT], ws[TW], ms[TW], md[TW];      // S dO, and the scores
#pragma unroll
        for (int i = 0; i < DW; ++i)
#pragma unroll
            for (int t = 0; t < CT; ++t) held[i][t] = zero4();
#pragma unroll
        for (int i = 0; i < TW; ++i) ws[i] = ms[i] = md[i] = zero4();
        float sdb[N] = {}, svd[N] = {};

        for (int n0 = 0; n0 < dv; n0 += SLAB) {
            const int tid = thread(), c = tid & 15, g = (tid & 63) >> 4;
            // all of the slab's loads are on their way before the first is waited for
            f32x4 lu[N], lr[N], lv[N], lo[N], st[SLAB / 32][DW][4];
            auto states = [&](int f, auto whole) {
                constexpr bool W = decltype(whole)::value;
#pragma unroll
                for (int i = 0; i < DW; ++i) {
                    const int ch = 16 * (w * DW + i) + c, col = n0 + 32 * f + 8 * g;
                    const bool there = ch < dk;
                    const uint32_t off = there ? static_cast<uint32_t>(ch) * dv : 0;
                    st[f][i][0] = four<W>(S + off, col, dv, there);
                    st[f][i][1] = four<W>(S + off, col + 4, dv, there);
                    st[f][i][2] = four<W>(U + off, col, dv, there);
                    st[f][i][3] = four<W>(U + off, col + 4, dv, there);
                }
            };
            auto fetch = [&](auto whole) {
                constexpr bool W = decltype(whole)::value;
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    const int r = tid / (SLAB / 4) + u * RPP, rr = r < cnt ? r : cnt - 1, col = n0 + 4 * (tid % (SLAB / 4));
                    const bool there = r < cnt;
                    lu[u] = four<W>(L.rec_du + row0 * dv + static_cast<uint32_t>(rr) * dv, col, dv, there);
                    lr[u] = four<W>(L.rec_R + row0 * dv + static_cast<uint32_t>(rr) * dv, col, dv, there);
                    lv[u] = four<W>(vp + rr * L.v_s[2], col, dv, there);
                    lo[u] = four<W>(gp + rr * L.g_s[2], col, dv, there);
                }
                if (DW == 1) {
#pragma unroll
                    for (int f = 0; f < SLAB / 32; ++f) states(f, whole);
                }
            };
            if (whole) fetch(std::true_type());
            else fetch(std::false_type());
            if (n0 == 0) {              // S' . U
                const int size = static_cast<int>(cells);
                if (whole) {
#pragma unroll 4
                    for (int i = 4 * tid; i < size; i += 4 * NT) {
                        const f32x4 x = *reinterpret_cast<const f32x4*>(S + cells + i), y = *reinterpret_cast<const f32x4*>(U + i);
#pragma unroll
                        for (int r = 0; r < 4; ++r) dot = __builtin_fmaf(x[r], y[r], dot);
                    }
                } else {
#pragma unroll 4
                    for (int i = tid; i < size; i += NT) dot = __builtin_fmaf(S[cells + i], U[i], dot);
                }
            }
            __syncthreads();            // (the last columns' rows are read, the tokens' factors written)
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int r = tid / (SLAB / 4) + u * RPP, col = n0 + 4 * (tid % (SLAB / 4));
                const float be = M.beta[r], fe = M.e[r], fw = M.wt[r];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sdb[u] = __builtin_fmaf(lu[u][i], lr[u][i], sdb[u]);
                    lu[u][i] *= be;
                    lr[u][i] *= be;
                    svd[u] = __builtin_fmaf(lv[u][i], lu[u][i], svd[u]);
                }
                if (r < rows && col < dv) put_four(dvp + r * L.dv_s[2], col, dv, lu[u]);
                const int at = r * SV + 4 * (tid % (SLAB / 4));
                Ops<E>::put4(M.row.o + at, VPL, lo[u]);
                put_parts<SP>(M.row.v + at, VPL, lu[u]);
                put_parts<SP>(M.row.u + at, VPL, lr[u]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lu[u][i] *= -fe;
                    lr[u][i] *= fw;
                }
                put_parts<SP>(M.row.ev + at, VPL, lu[u]);
                put_parts<SP>(M.row.wu + at, VPL, lr[u]);
            }
            __syncthreads();
#pragma unroll
            for (int f = 0; f < SLAB / 32; ++f) {
                if (n0 + 32 * f >= dv) break;
                const int at = 32 * f + 8 * g;
                // dq, dk from the states: a wave's channels
                if (DW > 1) {
                    if (whole) states(f, std::true_type());
                    else states(f, std::false_type());
                }
                Op<SP> so[DW], uo[DW];
#pragma unroll
                for (int i = 0; i < DW; ++i) {
                    so[i] = op_of<SP>(st[f][i][0], st[f][i][1]);
                    uo[i] = op_of<SP>(st[f][i][2], st[f][i][3]);
                }
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const int p = (16 * t + c) * SV + at;
                    const Op<P> bo = op_rows<P>(M.row.o + p, VPL);
                    const Op<SP> bv = op_rows<SP>(M.row.ev + p, VPL), bu = op_rows<SP>(M.row.wu + p, VPL);
#pragma unroll
                    for (int y = 0; y < PAIRS<SP, P>; ++y)
#pragma unroll
                        for (int i = 0; i < DW; ++i) mm<SP, P>(y, held[i][t], so[i], bo);
#pragma unroll
                    for (int y = 0; y < PAIRS<SP, SP>; ++y)
#pragma unroll
                        for (int i = 0; i < DW; ++i) {
                            mm<SP, SP>(y, dkk[i][t], so[i], bv);
                            mm<SP, SP>(y, dkk[i][t], uo[i], bu);
                        }
                    __builtin_amdgcn_sched_barrier(0);      // (mixed, the tiles' operands take more registers than there are)
                }
                // scores (rows j, columns i): dO_i . u_j below the diagonal, dv_i . u_j on both sides of it
#pragma unroll
                for (int x = 0; x < TW; ++x) {
                    const int ti = (w + NW * x) / CT, tj = (w + NW * x) % CT;
                    if (ti >= CT) break;
                    const Op<SP> uj = op_rows<SP>(M.row.u + (16 * tj + c) * SV + at, VPL), vj = op_rows<SP>(M.row.v + (16 * tj + c) * SV + at, VPL);
                    const Op<P> oi = op_rows<P>(M.row.o + (16 * ti + c) * SV + at, VPL);
                    const Op<SP> vi = op_rows<SP>(M.row.v + (16 * ti + c) * SV + at, VPL), ui = op_rows<SP>(M.row.u + (16 * ti + c) * SV + at, VPL);
#pragma unroll
                    for (int y = 0; y < PAIRS<SP, SP>; ++y) {
                        if (ti >= tj && y < PAIRS<SP, P>) mm<SP, P>(y, ws[x], uj, oi);
                        if (ti >= tj) mm<SP, SP>(y, ms[x], uj, vi);
                        if (ti <= tj) mm<SP, SP>(y, md[x], vj, ui);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if (DW > 1) keys();
        __syncthreads();                // (the rows are read: keys and queries take their place)
        tk.store(M.key.k, cnt, dk, tid);
        tq.store(M.key.q, cnt, dk, tid);
        const int lane = thread() & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
        for (int x = 0; x < TW; ++x) {
            const int ti = (w + NW * x) / CT, tj = (w + NW * x) % CT, i = 16 * ti + c;
            if (ti >= CT) break;
            f32x4 a, m;
            float down[4], up[4];
            decays(down, M.gh, M.gl, i, 16 * tj + 4 * g, false);
            decays(up, M.gh, M.gl, i, 16 * tj + 4 * g, true);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int jj = 16 * tj + 4 * g + r;
                a[r] = masked(jj <= i, ws[x][r] * (L.scale * down[r]));
                m[r] = masked(jj != i, -(jj < i ? ms[x][r] * down[r] : md[x][r] * up[r]));
            }
            if (ti >= tj) put_parts<SP>(M.w + i * ST + 16 * tj + 4 * g, TPL, a);
            put_parts<SP>(M.m + i * ST + 16 * tj + 4 * g, TPL, m);
        }
        // sums of the tokens' rows over their 16 threads, and of S' . U over all
#pragma unroll
        for (int u = 0; u < N; ++u) {
#pragma unroll
            for (int d = 1; d < 16; d *= 2) {
                sdb[u] += __shfl_xor(sdb[u], d);
                svd[u] += __shfl_xor(svd[u], d);
            }
            if (tid % 16 == 0) {
                M.db[tid / 16 + u * RPP] = sdb[u];
                M.vd[tid / 16 + u * RPP] = svd[u];
            }
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) dot += __shfl_xor(dot, d);
        if (lane == 0) M.dot[w] = dot;
        __syncthreads();
        if (tid < C) {
            float x = 0.f;
            if (tid < cnt) {
#pragma unroll
                for (int p = 0; p < NT / C; ++p) x += M.od[p * C + tid];
                x -= M.vd[tid];
            }
#pragma unroll
            for (int d = 1; d < C; d *= 2) {
                const float y = __shfl_down(x, d);
                if (tid + d < C) x += y;
            }
#pragma unroll
            for (int i = 0; i < NW; ++i) x += M.dot[i];
            if (tid < rows) {
                const bool there = tid < cnt;
                dlp[tid * L.dl_s[2]] = !there || decay < -128.f ? 0.f : x;      // (such a decay is 0, and so is its gradient)
                dbp[tid * L.db_s[2]] = there ? M.db[tid] : 0.f;
            }
        }
        // dq has c e S dO; then the products over tokens
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const float fe = L.scale * M.e[16 * t + c];
#pragma unroll
            for (int i = 0; i < DW; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) dq[i][t][r] = __builtin_fmaf(fe, held[i][t][r], dq[i][t][r]);
        }
#pragma unroll
        for (int f = 0; f < CF; ++f) {
            const int row = (32 * f + 8 * g + (c >> 2)) * SK + 4 * (c & 3);
            Op<P> kc[DW], qc[DW];
#pragma unroll
            for (int i = 0; i < DW; ++i) {
                kc[i] = op_cols<P>(M.key.k + row + 16 * (w * DW + i), SK, KPL);
                qc[i] = op_cols<P>(M.key.q + row + 16 * (w * DW + i), SK, KPL);
            }
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const Op<SP> mt = op_rows<SP>(M.m + (16 * t + c) * ST + 32 * f + 8 * g, TPL);
#pragma unroll
                for (int x = 0; x < PAIRS<P, SP>; ++x)
#pragma unroll
                    for (int i = 0; i < DW; ++i) mm<P, SP>(x, dkk[i][t], kc[i], mt);
                if (f <= t / 2) {
                    const Op<SP> wt = op_rows<SP>(M.w + (16 * t + c) * ST + 32 * f + 8 * g, TPL);
#pragma unroll
                    for (int x = 0; x < PAIRS<P, SP>; ++x)
#pragma unroll
                        for (int i = 0; i < DW; ++i) mm<P, SP>(x, dq[i][t], kc[i], wt);
                }
                if (f >= t / 2) {
                    const Op<SP> wt = op_cols<SP>(M.w + (32 * f + 8 * g + (c >> 2)) * ST + 16 * t + 4 * (c & 3), ST, TPL);
#pragma unroll
                    for (int x = 0; x < PAIRS<P, SP>; ++x)
#pragma unroll
                        for (int i = 0; i < DW; ++i) mm<P, SP>(x, dkk[i][t], qc[i], wt);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    const int c = thread() & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        if (16 * t + c >= rows) continue;
#pragma unroll
        for (int i = 0; i < DW; ++i) {
            const int ch = 16 * (w * DW + i) + 4 * g;
            if (ch >= dk) continue;
            put_four(dqp + (16 * t + c) * L.dq_s[2], ch, dk, dq[i][t]);
            put_four(dkp + (16 * t + c) * L.dk_s[2], ch, dk, dkk[i][t]);
        }
    }
}

template <typename E, int DKP> hipError_t bwd(const DeltaLaunch& L, hipStream_t st)
{
    typedef Scans<E, DKP> Sc;
    constexpr size_t grad = sizeof(GradMem<E, DKP>);
    constexpr int threads = GradMem<E, DKP>::NT;
    static_assert(grad <= 160 * 1024, "one compute unit's LDS");
    const int slices = (L.dv + SLICE - 1) / SLICE;
    hipLaunchKernelGGL((sfda_delta_scans<E, DKP>), dim3(static_cast<unsigned>(L.heads) * slices, 2), dim3(Sc::THREADS), Sc::BYTES, st, L, slices);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || L.blocks == 0) return e;
    const unsigned keys = static_cast<unsigned>(L.heads / (L.H / L.Hk));
    hipLaunchKernelGGL((sfda_delta_grad<E, DKP>), dim3(keys * L.blocks), dim3(threads), grad, st, L);
    return hipGetLastError();
}
template <typename E> hipError_t bwd_any(const DeltaLaunch& L, hipStream_t st)
{
    return L.dk <= 64 ? bwd<E, 64>(L, st) : L.dk <= 128 ? bwd<E, 128>(L, st) : bwd<E, 256>(L, st);
}

}  // namespace
}  // namespace delta

hipError_t launch_delta_bwd(const DeltaLaunch& L, hipStream_t st)
{
    const hipError_t e = delta::prep(L, 2, st);
    if (e != hipSuccess) return e;
    return L.bf16 ? delta::bwd_any<uint16_t>(L, st) : delta::bwd_any<float>(L, st);
}

}  // namespace sfda
