// Launch descriptors of the operators around the attention: linear attention with one decay for
// each head, rotary positions, group norm.  Arguments are already validated when these are filled in.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace sfda {

// One scan of a decay attention.  For queries q and keys k of da channels and values v of db:
//   S_i = lambda S_(i-1) + upd k_i v_i^T,   o_i = sum_(j <= i) intra lambda^(i-j) (q_i . k_j) v_j + (the start state's part),
// tokens in their order or, reversed, from a sequence's last to its first.  The start state enters o_i
// by inter lambda^(i+1) forward and inter lambda^i reversed, and the end state is lambda^n S + upd sum lambda^(n-1-j) k_j v_j^T
// forward, lambda^(n-j) reversed: dL/dS_t holds token t's own term before it meets a decay.
struct DecayRole {
    const void *q, *k, *v;
    void* o;
    const float* S0;         // may be null (zero state)
    float* S_T;              // may be null
    float* ws;               // states of the segments [segments][heads][da][db], null with one segment
    long long q_s[3], k_s[3], v_s[3], o_s[3];   // element strides of b, h, t
    int da, db;
    long long s_row, s_col;  // element strides of S0 and S_T inside a head (of da * db elements)
    int slices;              // workgroups over the value columns (set by the launcher)
    int reverse;
    float intra, inter, upd;
};

constexpr int DECAY_ROLES = 3;
struct DecayLaunch {
    DecayRole role[DECAY_ROLES];
    int roles;
    const float* log_decay;  // [H]
    const int* lengths;      // [B] or null
    int B, H, T;
    int seg_tokens;          // tokens of a segment (T or more: one segment)
    int segments;
    int cus;                 // compute units of the device
    bool bf16;
};
// value columns of a scan workgroup, and workgroups over db columns, for a state of da channels
constexpr int decay_slice(bool bf16, int da) { return bf16 || da <= 128 ? 64 : 32; }
constexpr int decay_slices(bool bf16, int da, int db) { return (db + decay_slice(bf16, da) - 1) / decay_slice(bf16, da); }
hipError_t launch_decay(const DecayLaunch& L, hipStream_t st);

struct DecayStepLaunch {
    const void *q, *k, *v;
    void* o;
    float* S;
    const float* log_decay;
    long long q_s[2], k_s[2], v_s[2], o_s[2];   // element strides of b, h
    int B, H, dk, dv;
    float scale;
    bool bf16;
};
hipError_t launch_decay_step(const DecayStepLaunch& L, hipStream_t st);

// The gated delta rule of value heads first .. first + heads - 1 (numbered over the batch), H / Hk of them for a key head.  The workspace's
// parts are counted from `first`; a sequence has room for `blocks` blocks of delta_block tokens.
struct DeltaLaunch {
    const void *q, *k, *v, *dO;
    void *o, *dq, *dk_out, *dv_out;
    const float *log_decay, *beta;
    float *dlog_decay, *dbeta;
    const float *S0, *dS_T;  // may be null (zero)
    float *S_T, *dS0;        // may be null
    long long q_s[3], k_s[3], v_s[3], o_s[3], g_s[3];           // element strides of b, h, t (g: dO)
    long long l_s[3], b_s[3];                                   // log_decay, beta
    long long dq_s[3], dk_s[3], dv_s[3], dl_s[3], db_s[3];
    const int* lengths;      // [B] or null
    int B, H, Hk, T, dk, dv;
    float scale;
    long long first;
    int heads, blocks;
    uint16_t *inv, *inv_back;       // [heads][blocks][3 parts][tiles of the lower triangle][16][16]
    uint16_t *scores, *scores_back;
    int score_parts;         // of the forward scan's scores that are read
    int segments, seg_blocks, slices;       // forward: of a sequence, blocks of one, workgroups over the value columns
    float *seg_N, *seg_M;    // [segments - 1][heads][dk][dv], [dk][dk]: a segment's end state is N + M times its start state (and behind N, S0)
    float4* scalars;         // [heads][blocks * block][2]: sum of the block's log decays (hi, lo), beta, e; w, w beta, the block's decay (hi, lo)
    float *rec_S, *rec_U;    // states before each block and after the last; their gradients after each block
    float *rec_R, *rec_du;   // [heads][blocks * block][dv]
    float* odo;              // [heads][parts][blocks * block]
    int parts;               // 16 columns each
    bool whole;              // value columns are whole fours, at 4-byte addresses where o is concerned
    bool bf16;
};
constexpr int delta_block(bool bf16) { return bf16 ? 64 : 32; }
constexpr int delta_tiles(bool bf16) { return bf16 ? 10 : 3; }
constexpr bool delta_segments(bool bf16, int dk) { return bf16 || dk <= 128; }      // whether sequences may be cut
hipError_t launch_delta_fwd(const DeltaLaunch& L, hipStream_t st);
hipError_t launch_delta_bwd(const DeltaLaunch& L, hipStream_t st);

struct DeltaStepLaunch {
    const void *q, *k, *v;
    void* o;
    float* S;
    const float *log_decay, *beta;
    long long q_s[2], k_s[2], v_s[2], o_s[2], l_s[2], b_s[2];   // element strides of b, h
    int B, H, Hk, dk, dv;
    float scale;
    bool bf16;
};
hipError_t launch_delta_step(const DeltaStepLaunch& L, hipStream_t st);

constexpr int ROTARY_AXES = 4, ROTARY_PAIRS = 2048;
struct RotaryLaunch {
    const void *q, *k;       // k may be null
    void *qo, *ko;
    long long q_s[3], k_s[3], qo_s[3], ko_s[3];
    const float *cos, *sin;  // [P, rot / 2]
    const void* positions;   // int32 or int64 [B or 1, T] ([axes, B or 1, T] with axes), or null: offset + t
    int pos64;
    long long pos_a, pos_b;  // element strides of positions over axes and b
    long long offset;
    int B, Hq, Hk, T, D, rot, P;
    int interleaved, inverse;
    int axes;                // 0: one position for a token
    unsigned axis[ROTARY_PAIRS / 16];       // each pair's axis, 2 bits
    bool bf16;
};
hipError_t launch_rotary(const RotaryLaunch& L, hipStream_t st);

struct NormLaunch {
    const void *x, *gate;    // gate may be null
    const void* dy;          // backward
    void *y, *dx, *dgate;
    const float *weight, *bias;     // may be null
    float *dweight, *dbias;
    float* partial;          // backward: [strips][2][H * D]
    long long x_s[3], dx_s[3];      // b, h, t
    long long g_s[2], dg_s[2], y_s[2];   // b, t (channel h * D + d)
    int B, H, T, D;
    int silu;
    float eps;
    bool bf16;
};
int norm_strips(long rows_bt, int H, int D, bool bf16);     // workgroups of a head
constexpr int NORM_MAX = 2048;          // channels of a group

// Rows x [B, T, D] (+ residual, rounded: total) normalised over D; backward, dx = the norm's gradient (+ dtotal).
struct LayerNormLaunch {
    const void *x, *residual;       // residual may be null
    const void *dy, *dtotal;        // backward; dtotal may be null
    void *y, *total, *dx;
    const float *weight, *bias;     // may be null
    float *dweight, *dbias;
    float* partial;          // backward: [strips][2][D]
    long long x_s[2], r_s[2], y_s[2], t_s[2], dy_s[2], dt_s[2], dx_s[2];     // element strides of b, t
    int B, T, D;
    float eps;
    bool bf16;
};
constexpr int LAYER_NORM_MAX = 16384;
int layer_norm_strips(long long rows, int D, bool bf16, bool bwd);    // workgroups
hipError_t launch_layer_norm(const LayerNormLaunch& L, hipStream_t st);
hipError_t launch_layer_norm_bwd(const LayerNormLaunch& L, hipStream_t st);
hipError_t launch_norm(const NormLaunch& L, hipStream_t st);
hipError_t launch_norm_bwd(const NormLaunch& L, hipStream_t st);

}  // namespace sfda
