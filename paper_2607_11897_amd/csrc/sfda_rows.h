// Sums over the lanes that hold a row (gfx950).
#pragma once

#include <hip/hip_runtime.h>

namespace sfda {
namespace rows {

template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, false));
}
// sum over a group of `lpg` (a power of two) neighbouring lanes, the same for every lane of it.  Within 16 lanes by data-parallel
// moves: the quad's neighbours, then mirrored halves, whose lanes already hold equal sums.
__device__ __forceinline__ float group_sum(float x, int lpg)
{
    if (lpg > 1) x += dpp<0xB1>(x);         // quad [1, 0, 3, 2]
    if (lpg > 2) x += dpp<0x4E>(x);         // quad [2, 3, 0, 1]
    if (lpg > 4) x += dpp<0x141>(x);        // half row mirrored
    if (lpg > 8) x += dpp<0x140>(x);        // row mirrored
    if (lpg > 16) x += __shfl_xor(x, 16);
    if (lpg > 32) x += __shfl_xor(x, 32);
    return x;
}

// 1 / sqrt(x), x >= 0.  The hardware's instruction takes a subnormal for 0; a variance below 2^-126 (values of 1e-19) is one, and
// with eps = 0 it counts.  The scaling takes no time that shows (bfloat16 B8 H16 T4096 d 128, in turn: forward 95.4 us and 95.0
// without, backward 147.5 and 147.6).
__device__ __forceinline__ float inverse_root(float x)
{
    const bool small = x < 0x1p-100f;
    const float r = __builtin_amdgcn_rsqf(small ? x * 0x1p64f : x);
    return small ? r * 0x1p32f : r;
}

}  // namespace rows
}  // namespace sfda
