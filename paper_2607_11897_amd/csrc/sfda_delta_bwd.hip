// The gated delta rule's backward (gfx950).  With the notation of the scan, u = beta R the writes and dv = beta du:
//   dbeta_i = du_i . R_i,   dq = c e dO S^T + (c D . dO u^T) K,
//   dk = w u U^T - e dv S^T + (c D . dO u^T)^T Q - (M + M^T) K,   M_ij = D_ij dv_i . u_j  (j < i).
// A log decay at token t scales what the outputs from t on read and what their writes cancel: with G the sum of the log decays,
// dL/dG_t = dO_t . o_t - v_t . dv_t, and what the state after the block carries on is S' . U, so that
//   dlog_decay_t = S' . U + sum_(s >= t, in the block) (dO_s . o_s - v_s . dv_s).
// Three launches after the inverses: the forward scan again, which records the states and the rows R, and the adjoint scan,
// which records U and du, side by side as roles of one; then all blocks at once form the products above.
#include "sfda_delta.h"

namespace sfda {
namespace delta {

hipError_t prep(const DeltaLaunch& L, int inverses, hipStream_t st);

namespace {

template <typename E, int DKP> constexpr size_t scan_bytes()
{
    return sizeof(Mem<E, DKP, RECORD>) > sizeof(Mem<E, DKP, ADJOINT>) ? sizeof(Mem<E, DKP, RECORD>) : sizeof(Mem<E, DKP, ADJOINT>);
}

template <typename E, int DKP> __global__ __launch_bounds__(NT) void sfda_delta_scans(DeltaLaunch L, int slices)
{
    extern __shared__ __align__(16) unsigned char smem[];
    long head;
    int sl;
    head_slice(blockIdx.x, slices, L.heads, head, sl);
    head = static_cast<long>(same_for_all(static_cast<uint64_t>(head)));
    sl = __builtin_amdgcn_readfirstlane(sl);
    if (blockIdx.y == 0) scan<E, DKP, RECORD>(L, head, sl, smem);
    else scan<E, DKP, ADJOINT>(L, head, sl, smem);
}

// ------------------------------------------------------------------ the blocks' gradients

constexpr int SLAB = 64;        // value columns at a time

template <typename E, int DKP> struct GradMem {
    typedef Block<E> B;
    static constexpr int C = B::C, P = B::P, SK = DKP + 8, SV = SLAB + 8, ST = C + 8;
    static constexpr int KPL = C * SK, VPL = C * SV, TPL = C * ST;
    union {
        struct { uint16_t o[P * VPL], v[P * VPL], u[P * VPL]; } row;    // dO, dv, u: [token][value column]
        struct { uint16_t k[P * KPL], q[P * KPL]; } key;
    };
    uint16_t w[P * TPL], m[P * TPL];                                    // c D . dO u^T, and -(M + M^T): [i][j]
    float e[C], wt[C], beta[C], gh[C], gl[C], db[C], vd[C], dot[NW];
};

// 4 neighbours of a row of n elements from column `col` on, zeros past them and where the row is not there
template <typename T> __device__ __forceinline__ f32x4 four(const T* row, int col, int n, bool there)
{
    f32x4 x = zero4();
    if (!there || col >= n) return x;
    if (col + 4 <= n) {
        if constexpr (sizeof(T) == 4) {
            memcpy(&x, row + col, 16);
        } else {
            u32x2 y;
            memcpy(&y, row + col, 8);
            x = f32x4{lo_f32(y[0]), hi_f32(y[0]), lo_f32(y[1]), hi_f32(y[1])};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (col + i < n) x[i] = value<T>(reinterpret_cast<const char*>(row + col + i));
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

// One workgroup for a block of a key head, its value heads one after the other.  A wave owns DKP / 64 tiles of 16 channels of dq and dk
// (rows; tokens are the columns), whose rows of the states it alone reads.
template <typename E, int DKP> __global__ __launch_bounds__(NT) void sfda_delta_grad(DeltaLaunch L)
{
    typedef Block<E> B;
    typedef GradMem<E, DKP> M_;
    constexpr int C = B::C, CT = B::CT, CF = B::CF, P = B::P, ES = sizeof(E), DW = DKP / 64;
    constexpr int SK = M_::SK, SV = M_::SV, ST = M_::ST, KPL = M_::KPL, VPL = M_::VPL, TPL = M_::TPL;
    constexpr int RPP = NT / (SLAB / 4), N = C / RPP, TW = CT * CT / NW;    // rows of a pass, passes, tiles of scores of a wave
    extern __shared__ __align__(16) unsigned char smem[];
    M_& M = *reinterpret_cast<M_*>(smem);

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned group = blockIdx.x / static_cast<unsigned>(L.blocks);
    const int blk = static_cast<int>(blockIdx.x - group * static_cast<unsigned>(L.blocks)), per = L.H / L.Hk;
    const long long key = L.first / per + group;
    const int b = __builtin_amdgcn_readfirstlane(static_cast<int>(key / L.Hk)), hk = __builtin_amdgcn_readfirstlane(static_cast<int>(key - static_cast<long long>(b) * L.Hk));
    const int len = __builtin_amdgcn_readfirstlane(seq_length(L.lengths, b, L.T));
    const int t0 = blk * C, rows = L.T - t0 < C ? L.T - t0 : C, cnt = len - t0 < 0 ? 0 : len - t0 < C ? len - t0 : C;
    const int dk = L.dk, dv = L.dv;
    const long long cells = static_cast<long long>(dk) * dv;

    E* const dqp = static_cast<E*>(L.dq) + b * L.dq_s[0] + hk * L.dq_s[1] + t0 * L.dq_s[2];
    E* const dkp = static_cast<E*>(L.dk_out) + b * L.dk_s[0] + hk * L.dk_s[1] + t0 * L.dk_s[2];
    f32x4 dq[DW][CT], dkk[DW][CT];
#pragma unroll
    for (int i = 0; i < DW; ++i)
#pragma unroll
        for (int t = 0; t < CT; ++t) dq[i][t] = dkk[i][t] = zero4();

#ifdef SFDA_LDS_POISON
    lds_poison(&M, sizeof(M_), tid, NT);
    __syncthreads();
#endif
    {   // the upper tiles of c D . dO u^T stay zero
        u32x4* z = reinterpret_cast<u32x4*>(M.w);
        const u32x4 zero = {0, 0, 0, 0};
        for (int i = tid; i < P * TPL / 8; i += NT) z[i] = zero;
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

        if (cnt == 0) {                 // nothing there: zeros
            for (int i = tid; i < rows * SLAB / 4; i += NT)
                for (int col = 4 * (i % (SLAB / 4)); col < dv; col += SLAB) put_four(dvp + (i / (SLAB / 4)) * L.dv_s[2], col, dv, zero4());
            if (tid < rows) dlp[tid * L.dl_s[2]] = dbp[tid * L.db_s[2]] = 0.f;
            continue;
        }
        RowTile<E, DKP, C, SK> tk, tq;
        tk.load(reinterpret_cast<const char*>(static_cast<const E*>(L.k) + b * L.k_s[0] + hk * L.k_s[1] + t0 * L.k_s[2]), static_cast<uint32_t>(L.k_s[2] * ES), cnt, dk, tid);
        tq.load(reinterpret_cast<const char*>(static_cast<const E*>(L.q) + b * L.q_s[0] + hk * L.q_s[1] + t0 * L.q_s[2]), static_cast<uint32_t>(L.q_s[2] * ES), cnt, dk, tid);

        __syncthreads();                // (the last head's tokens and keys are read)
        if (tid < C) {
            const float4 sc = L.scalars[row0 + tid];
            const float eh = __shfl(sc.x, C - 1), el = __shfl(sc.y, C - 1);
            M.gh[tid] = sc.x;
            M.gl[tid] = sc.y;
            M.beta[tid] = sc.z;
            M.e[tid] = expf(sc.x + sc.y);
            M.wt[tid] = expf((eh - sc.x) + (el - sc.y));
        }
        f32x4 de[DW][CT], dO[DW][CT], db[DW][CT], ws[TW], ms[TW], md[TW];
#pragma unroll
        for (int i = 0; i < DW; ++i)
#pragma unroll
            for (int t = 0; t < CT; ++t) de[i][t] = dO[i][t] = db[i][t] = zero4();
#pragma unroll
        for (int i = 0; i < TW; ++i) ws[i] = ms[i] = md[i] = zero4();
        float sdb[N] = {}, svd[N] = {}, dot = 0.f;

        for (int n0 = 0; n0 < dv; n0 += SLAB) {
            __syncthreads();            // (the last columns' rows are read, the tokens' factors written)
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int r = tid / (SLAB / 4) + u * RPP, col = n0 + 4 * (tid % (SLAB / 4));
                const bool there = r < cnt;
                f32x4 du = four(L.rec_du + (row0 + r) * dv, col, dv, there), R = four(L.rec_R + (row0 + r) * dv, col, dv, there);
                const f32x4 vv = four(vp + r * L.v_s[2], col, dv, there), go = four(gp + r * L.g_s[2], col, dv, there);
                const float be = M.beta[r];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sdb[u] = __builtin_fmaf(du[i], R[i], sdb[u]);
                    du[i] *= be;
                    R[i] *= be;
                    svd[u] = __builtin_fmaf(vv[i], du[i], svd[u]);
                }
                if (r < rows && col < dv) put_four(dvp + r * L.dv_s[2], col, dv, du);
                const int at = r * SV + 4 * (tid % (SLAB / 4));
                Ops<E>::put4(M.row.o + at, VPL, go);
                Ops<E>::put4(M.row.v + at, VPL, du);
                Ops<E>::put4(M.row.u + at, VPL, R);
            }
            __syncthreads();
#pragma unroll
            for (int f = 0; f < SLAB / 32; ++f) {
                if (n0 + 32 * f >= dv) break;
                const int at = 32 * f + 8 * g, col = n0 + at;
                // dq, dk from the states: a wave's channels
                Op<P> bo[CT], bv[CT], bu[CT];
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    bo[t] = op_rows<P>(M.row.o + (16 * t + c) * SV + at, VPL);
                    bv[t] = op_rows<P>(M.row.v + (16 * t + c) * SV + at, VPL);
                    bu[t] = op_rows<P>(M.row.u + (16 * t + c) * SV + at, VPL);
                }
#pragma unroll
                for (int i = 0; i < DW; ++i) {
                    const int ch = 16 * (w * DW + i) + c;
                    const bool there = ch < dk;
                    const long long off = there ? static_cast<long long>(ch) * dv : 0;
                    const f32x4 s0 = four(S + off, col, dv, there), s1 = four(S + off, col + 4, dv, there);
                    const f32x4 u0 = four(U + off, col, dv, there), u1 = four(U + off, col + 4, dv, there);
                    const f32x4 n1 = four(S + cells + off, col, dv, there), n2 = four(S + cells + off, col + 4, dv, there);
#pragma unroll
                    for (int r = 0; r < 4; ++r) dot = __builtin_fmaf(n1[r], u0[r], __builtin_fmaf(n2[r], u1[r], dot));
                    const Op<P> so = op_of<P>(s0, s1), uo = op_of<P>(u0, u1);
#pragma unroll
                    for (int x = 0; x < PAIRS<P, P>; ++x)
#pragma unroll
                        for (int t = 0; t < CT; ++t) {
                            mm<P, P>(x, dO[i][t], so, bo[t]);
                            mm<P, P>(x, de[i][t], so, bv[t]);
                            mm<P, P>(x, db[i][t], uo, bu[t]);
                        }
                }
                // scores (rows j, columns i): dO_i . u_j below the diagonal, dv_i . u_j on both sides of it
#pragma unroll
                for (int x = 0; x < TW; ++x) {
                    const int ti = (w + NW * x) / CT, tj = (w + NW * x) % CT;
                    const Op<P> uj = op_rows<P>(M.row.u + (16 * tj + c) * SV + at, VPL), vj = op_rows<P>(M.row.v + (16 * tj + c) * SV + at, VPL);
                    const Op<P> oi = op_rows<P>(M.row.o + (16 * ti + c) * SV + at, VPL), vi = op_rows<P>(M.row.v + (16 * ti + c) * SV + at, VPL);
                    const Op<P> ui = op_rows<P>(M.row.u + (16 * ti + c) * SV + at, VPL);
#pragma unroll
                    for (int y = 0; y < PAIRS<P, P>; ++y) {
                        if (ti >= tj) mm<P, P>(y, ws[x], uj, oi);
                        if (ti >= tj) mm<P, P>(y, ms[x], uj, vi);
                        if (ti <= tj) mm<P, P>(y, md[x], vj, ui);
                    }
                }
            }
        }
        __syncthreads();                // (the rows are read: keys and queries take their place)
        tk.store(M.key.k, cnt, dk, tid);
        tq.store(M.key.q, cnt, dk, tid);
#pragma unroll
        for (int x = 0; x < TW; ++x) {
            const int ti = (w + NW * x) / CT, tj = (w + NW * x) % CT, i = 16 * ti + c;
            f32x4 a, m;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int jj = 16 * tj + 4 * g + r, hi = i > jj ? i : jj, lo = i > jj ? jj : i;
                const float d = expf((M.gh[hi] - M.gh[lo]) + (M.gl[hi] - M.gl[lo]));
                a[r] = jj <= i ? ws[x][r] * (L.scale * d) : 0.f;
                m[r] = jj == i ? 0.f : -d * (jj < i ? ms[x][r] : md[x][r]);
            }
            if (ti >= tj) Ops<E>::put4(M.w + i * ST + 16 * tj + 4 * g, TPL, a);
            Ops<E>::put4(M.m + i * ST + 16 * tj + 4 * g, TPL, m);
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
                for (int p = 0; p < L.parts; ++p) x += L.odo[(head * L.parts + p) * (static_cast<long long>(L.blocks) * C) + t0 + tid];
                x -= M.vd[tid];
            }
#pragma unroll
            for (int d = 1; d < C; d *= 2) {
                const float y = __shfl_down(x, d);
                if (tid + d < C) x += y;
            }
            x += (M.dot[0] + M.dot[1]) + (M.dot[2] + M.dot[3]);
            if (tid < rows) {
                const bool there = tid < cnt;
                const float a = there ? L.log_decay[b * L.l_s[0] + h * L.l_s[1] + (t0 + tid) * L.l_s[2]] : 0.f;
                dlp[tid * L.dl_s[2]] = !there || a < -128.f ? 0.f : x;      // (such a decay is 0, and so is its gradient)
                dbp[tid * L.db_s[2]] = there ? M.db[tid] : 0.f;
            }
        }
        // the rows' factors, then the products over tokens
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const float fe = M.e[16 * t + c], fw = M.wt[16 * t + c];
#pragma unroll
            for (int i = 0; i < DW; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    dq[i][t][r] = __builtin_fmaf(L.scale * fe, dO[i][t][r], dq[i][t][r]);
                    dkk[i][t][r] += fw * db[i][t][r] - fe * de[i][t][r];
                }
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
                const Op<P> mt = op_rows<P>(M.m + (16 * t + c) * ST + 32 * f + 8 * g, TPL);
#pragma unroll
                for (int x = 0; x < PAIRS<P, P>; ++x)
#pragma unroll
                    for (int i = 0; i < DW; ++i) mm<P, P>(x, dkk[i][t], kc[i], mt);
                if (f <= t / 2) {
                    const Op<P> wt = op_rows<P>(M.w + (16 * t + c) * ST + 32 * f + 8 * g, TPL);
#pragma unroll
                    for (int x = 0; x < PAIRS<P, P>; ++x)
#pragma unroll
                        for (int i = 0; i < DW; ++i) mm<P, P>(x, dq[i][t], kc[i], wt);
                }
                if (f >= t / 2) {
                    const Op<P> wt = op_cols<P>(M.w + (32 * f + 8 * g + (c >> 2)) * ST + 16 * t + 4 * (c & 3), ST, TPL);
#pragma unroll
                    for (int x = 0; x < PAIRS<P, P>; ++x)
#pragma unroll
                        for (int i = 0; i < DW; ++i) mm<P, P>(x, dkk[i][t], qc[i], wt);
                }
            }
        }
    }
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
    constexpr size_t scans = scan_bytes<E, DKP>(), grad = sizeof(GradMem<E, DKP>);
    static_assert(scans <= 160 * 1024 && grad <= 160 * 1024, "one compute unit's LDS");
    const int slices = (L.dv + SLICE - 1) / SLICE;
    hipLaunchKernelGGL((sfda_delta_scans<E, DKP>), dim3(static_cast<unsigned>(L.heads) * slices, 2), dim3(NT), scans, st, L, slices);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || L.blocks == 0) return e;
    const unsigned keys = static_cast<unsigned>(L.heads / (L.H / L.Hk));
    hipLaunchKernelGGL((sfda_delta_grad<E, DKP>), dim3(keys * L.blocks), dim3(NT), grad, st, L);
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
