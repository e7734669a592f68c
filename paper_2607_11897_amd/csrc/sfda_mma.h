// Matrix products of the operators around the attention (gfx950): operand fragments of bfloat16 parts from LDS, registers and
// accumulators, and rows of any alignment on their way to them.
#pragma once

#include "sfda_device.h"
#include "sfda_vec.h"

#include <string.h>

namespace sfda {
namespace mx {

using namespace vec;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// the first `cols` (fewer than fill them) elements of a row as 16 bytes, zeros behind them; a loop, for it is rare and the
// scan short of registers
template <typename E> __device__ __forceinline__ u32x4 short_row(const char* p, int cols)
{
    typedef unsigned long long u64;
    constexpr int BITS = 8 * sizeof(E);
    u64 lo = 0, hi = 0;
#pragma clang loop unroll(disable)
    for (int i = cols - 1; i >= 0; --i) {
        uint32_t u = 0;
        memcpy(&u, p + i * sizeof(E), sizeof(E));
        hi = hi << BITS | lo >> (64 - BITS);
        lo = lo << BITS | u;
    }
    return u32x4{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32)};
}

// What the element type decides.  The matrix cores take bfloat16 operands.  A float32 is the sum of three bfloat16 (its 24 bits,
// 8 in each), so float32 tensors lie in LDS as PL = 3 planes, and a product of two operands is the six products of parts
// that reach 2^-22 of it (the three left out are below that): 6 x 16 cycles for 16 x 16 x 32 on a SIMD, where the float32 matrix
// instruction takes 256.  B8 H16 T2048 d 128: float32 instructions take 1.40 times as long forward, 1.41 times backward; the LDS
// reads, the matrix instructions and the splitting of operands then take about a third of a block's time each.
// An infinity in float32 comes out as NaN where it is used (its parts are inf - inf).
//   VE: elements of a 16-byte vector;  KB: the contraction length of one operand fragment, 8 places in a lane;  KP, SP:
// elements that rows of keys and of the state in LDS are longer than their channels, so that what a read takes at a time
// lies on different banks (4 token rows of 32 bytes for the transposing read of keys, 8 rows of 16 bytes for the state).
// Lane l of a fragment has index c = l % 16 of the free axis and 8 places of the contraction for its
// group g = l / 16.  Sums over channels take 8 neighbours (rows: one 16-byte read); sums over tokens take
// the places 4 g .. 4 g + 3 of each 16, which is what an accumulator tile holds of its rows, so that scores become
// an operand without leaving their lane.
constexpr int KB = 32, KP = 16, SP = 8;

// row-major [free][contraction]
__device__ __forceinline__ bf16x8 plane_rows(const uint16_t* p) { return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p)); }
// row-major [contraction][free]: the transposing LDS read takes, from each group of 16 lanes,
// 4 rows of 16 (lane l: row l / 4, 4 elements) and gives lane l column l.  p: the lane's own 4 elements in
// row 4 g + c / 4
__device__ __forceinline__ bf16x8 plane_cols(const uint16_t* p, int stride)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * stride));
    u32x4 w;
    w.lo = __builtin_bit_cast(u32x2, a);
    w.hi = __builtin_bit_cast(u32x2, b);
    return __builtin_bit_cast(bf16x8, w);
}
// offset of the lane's own elements for plane_cols: 4 of column block c % 4 whose blocks are `step` apart
__device__ __forceinline__ int cols_at(int stride, int step, int c, int g) { return (4 * g + (c >> 2)) * stride + step * (c & 3); }
__device__ __forceinline__ void mfma(f32x4& d, bf16x8 a, bf16x8 b) { d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, d, 0, 0, 0); }

template <typename E> struct Ops;

template <> struct Ops<uint16_t> {
    static constexpr int VE = 8, PL = 1, QV = 1;        // QV: vectors of a fragment
    typedef bf16x8 Frag;
    static __device__ __forceinline__ Frag rows(const uint16_t* p, int) { return plane_rows(p); }
    static __device__ __forceinline__ Frag cols(const uint16_t* p, int stride, int) { return plane_cols(p, stride); }
    static __device__ __forceinline__ Frag frag(const u32x4* v) { return __builtin_bit_cast(Frag, v[0]); }
    // from the accumulator tiles t[0], t[1] whose rows are the contraction
    static __device__ __forceinline__ Frag acc(const f32x4* t)
    {
        u32x4 w = {pack2(t[0][0], t[0][1]), pack2(t[0][2], t[0][3]), pack2(t[1][0], t[1][1]), pack2(t[1][2], t[1][3])};
        return __builtin_bit_cast(Frag, w);
    }
    static constexpr int PAIRS = 1;
    static __device__ __forceinline__ void mma(int, f32x4& d, const Frag& a, const Frag& b) { mfma(d, a, b); }
    static __device__ __forceinline__ void put4(uint16_t* to, int, const f32x4& x)
    {
        *reinterpret_cast<u32x2*>(to) = u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
    }
    static __device__ __forceinline__ void put(uint16_t* to, int, u32x4 w) { *reinterpret_cast<u32x4*>(to) = w; }
    static __device__ __forceinline__ u32x4 pack8(const f32x4& x, const f32x4& y)
    {
        return u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(y[0], y[1]), pack2(y[2], y[3])};
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
                uint32_t p = pack2(a, b);
                asm("" : "+v"(p));      // (or the halves are converted once more, one by one)
                o[s][e] = p;
                if (s + 1 < PARTS) { a -= lo_f32(p); b -= hi_f32(p); }
            }
        }
#pragma unroll
        for (int s = 0; s < PARTS; ++s) out[s] = __builtin_bit_cast(Frag, o[s]);
    }
};

template <> struct Ops<float> {
    static constexpr int VE = 4, PL = 3, QV = 2;
    struct Frag { bf16x8 p[3]; };
    // a pair as parts, whose sum is exact.  The first ones are truncated (nothing overflows), the others to nearest, so that
    // the products left out have no sign of their own
    static __device__ __forceinline__ void split(uint32_t (&p)[3], float a, float b)
    {
        p[0] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
        a -= hi_f32(__float_as_uint(a));
        b -= hi_f32(__float_as_uint(b));
        p[1] = pack2(a, b);
        asm("" : "+v"(p[1]));       // (or the halves are converted once more, one by one)
        p[2] = pack2(a - lo_f32(p[1]), b - hi_f32(p[1]));
    }
    static __device__ __forceinline__ Frag split8(const float (&x)[8])
    {
        u32x4 w[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t p[3];
            split(p, x[2 * e], x[2 * e + 1]);
#pragma unroll
            for (int s = 0; s < 3; ++s) w[s][e] = p[s];
        }
        return Frag{{__builtin_bit_cast(bf16x8, w[0]), __builtin_bit_cast(bf16x8, w[1]), __builtin_bit_cast(bf16x8, w[2])}};
    }
    static __device__ __forceinline__ Frag rows(const uint16_t* p, int plane)
    {
        return Frag{{plane_rows(p), plane_rows(p + plane), plane_rows(p + 2 * plane)}};
    }
    static __device__ __forceinline__ Frag cols(const uint16_t* p, int stride, int plane)
    {
        return Frag{{plane_cols(p, stride), plane_cols(p + plane, stride), plane_cols(p + 2 * plane, stride)}};
    }
    static __device__ __forceinline__ Frag frag(const u32x4* v)
    {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(v[i / 4][i % 4]);
        return split8(x);
    }
    static __device__ __forceinline__ Frag acc(const f32x4* t)
    {
        const float x[8] = {t[0][0], t[0][1], t[0][2], t[0][3], t[1][0], t[1][1], t[1][2], t[1][3]};
        return split8(x);
    }
    // pair i of a product's parts, the small ones first: a loop over tiles inside one over pairs has no product wait for the last
    static constexpr int PAIRS = 6;
    static __device__ __forceinline__ void mma(int i, f32x4& d, const Frag& a, const Frag& b)
    {
        constexpr int A[PAIRS] = {2, 0, 1, 1, 0, 0}, B[PAIRS] = {0, 2, 1, 0, 1, 0};
        mfma(d, a.p[A[i]], b.p[B[i]]);
    }
    static __device__ __forceinline__ void put4(uint16_t* to, int plane, const f32x4& x)
    {
        uint32_t a[3], b[3];
        split(a, x[0], x[1]);
        split(b, x[2], x[3]);
#pragma unroll
        for (int s = 0; s < 3; ++s) *reinterpret_cast<u32x2*>(to + s * plane) = u32x2{a[s], b[s]};
    }
    static __device__ __forceinline__ void put(uint16_t* to, int plane, u32x4 w) { put4(to, plane, __builtin_bit_cast(f32x4, w)); }
    static __device__ __forceinline__ void store1(float* p, float x) { *p = x; }
    static constexpr int PARTS = 1;
    static __device__ __forceinline__ void weighted(Frag (&out)[PARTS], const Frag& v, const float (&w)[8])
    {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float f[3];
#pragma unroll
            for (int s = 0; s < 3; ++s) {
                const uint32_t u = __builtin_bit_cast(u32x4, v.p[s])[i / 2];
                f[s] = i & 1 ? hi_f32(u) : lo_f32(u);
            }
            x[i] = (f[0] + (f[1] + f[2])) * w[i];       // (the sum is the float32 that was taken apart)
        }
        out[0] = split8(x);
    }
};

__device__ __forceinline__ int seq_length(const int* lengths, int b, int T)
{
    if (lengths == nullptr) return T;
    const int n = lengths[b];
    return n < 0 ? 0 : n > T ? T : n;
}

__device__ __forceinline__ uint64_t same_for_all(uint64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x >> 32));
    return static_cast<uint64_t>(hi) << 32 | lo;
}
// 16 bytes at base + off + more, base and more the same for all lanes; less than 2^31 bytes from the base.  ALIGNED: to 4 bytes, by a
// buffer resource.
template <bool ALIGNED> struct From {
    const char* p;
    __device__ __forceinline__ explicit From(const char* base) : p(reinterpret_cast<const char*>(same_for_all(reinterpret_cast<uint64_t>(base)))) {}
    __device__ __forceinline__ u32x4 load(uint32_t off, uint32_t more) const { return load16(p + more + off); }
    __device__ __forceinline__ void store(uint32_t off, uint32_t more, u32x4 x) const { store16(const_cast<char*>(p) + more + off, x); }
};
template <> struct From<true> {
    __amdgpu_buffer_rsrc_t r;
    __device__ __forceinline__ explicit From(const char* base)
        : r(__builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(same_for_all(reinterpret_cast<uint64_t>(base))), 0, 0x7fffffff, 0x00020000)) {}
    __device__ __forceinline__ u32x4 load(uint32_t off, uint32_t more) const { return __builtin_amdgcn_raw_buffer_load_b128(r, off, more, 0); }
    __device__ __forceinline__ void store(uint32_t off, uint32_t more, u32x4 x) const { __builtin_amdgcn_raw_buffer_store_b128(x, r, off, more, 0); }
};

// 16 bytes `past` elements (fewer than they hold) down, zeros behind: words by selects, bfloat16 by 64-bit shifts, which take
// more time and fewer registers (B8 H16 T1024 d 127: shifts take 1.13 times as long in float32, as long in bfloat16)
template <typename E> __device__ __forceinline__ u32x4 move_down(u32x4 x, int past)
{
    if constexpr (sizeof(E) == 4) {
        const bool one = past & 1, two = past & 2;
        const uint32_t y0 = one ? x[1] : x[0], y1 = one ? x[2] : x[1], y2 = one ? x[3] : x[2], y3 = one ? 0 : x[3];
        return u32x4{two ? y2 : y0, two ? y3 : y1, two ? 0 : y2, two ? 0 : y3};
    } else {
        typedef unsigned long long u64;
        const u64 lo = static_cast<u64>(x[1]) << 32 | x[0], hi = static_cast<u64>(x[3]) << 32 | x[2];
        const int t = past * 16 & 63;
        const u64 l = lo >> t | hi << 1 << (63 - t), h = hi >> t;
        const u64 a = past < 4 ? l : h, b = past < 4 ? h : 0;
        return u32x4{static_cast<uint32_t>(a), static_cast<uint32_t>(a >> 32), static_cast<uint32_t>(b), static_cast<uint32_t>(b >> 32)};
    }
}

}  // namespace mx
}  // namespace sfda
