// Launch descriptors of the operators around the attention: linear attention with one decay for
// each head, rotary positions, group norm.  Arguments are already validated when these are filled in.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>

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

struct RotaryLaunch {
    const void *q, *k;       // k may be null
    void *qo, *ko;
    long long q_s[3], k_s[3], qo_s[3], ko_s[3];
    const float *cos, *sin;  // [P, rot / 2]
    const void* positions;   // int32 or int64 [B or 1, T], or null: offset + t
    int pos64;
    long long pos_b;         // element stride of positions over b
    long long offset;
    int B, Hq, Hk, T, D, rot, P;
    int interleaved, inverse;
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
hipError_t launch_norm(const NormLaunch& L, hipStream_t st);
hipError_t launch_norm_bwd(const NormLaunch& L, hipStream_t st);

}  // namespace sfda
