// gs_device.h -- what kernels of more than one translation unit share: bf16, the clip coefficient, sums across a workgroup.
#ifndef GS_DEVICE_H
#define GS_DEVICE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#pragma clang fp contract(off)

namespace gs {

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

// fp32 -> bf16, round to nearest even; NaN stays NaN (quiet bit forced).
__device__ __forceinline__ uint32_t f32_to_bf16_bits(float f)
{
    uint32_t u = __float_as_uint(f);
    uint32_t r = (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
    uint32_t nan = (u >> 16) | 0x0040u;
    return ((u & 0x7fffffffu) > 0x7f800000u) ? nan : r;
}

// Clip coefficient from the total squared norm (Sec. 2.1: global L2 norm for clipping).
__device__ __forceinline__ float clip_from(double sqnorm, float max_norm)
{
    float norm = (float)sqrt(sqnorm);
    float c = max_norm / (norm + 1e-6f);
    return c < 1.0f ? c : 1.0f;
}

// ---- block reduction used by the norm kernels ----------------------------------------------
// Per-lane fp64 partial (each square is exact in fp64) -> across the lanes of a wave -> LDS across the
// block's waves -> one partial per block; a second tiny kernel folds the block partials in a
// fixed order, so the result is deterministic.
// A small range waits for every step of this, so lanes are exchanged by DPP moves, a few cycles each, where
// shuffles go through the LDS hardware, and the waves' sums are added across lanes and not one after another
// (norm, 13 k / 200 k elements, k = 4 3.74/4.83 us against 3.99/5.14; fp32 norm, 13 k 2.32 against 2.66; staged norm, 520 k,
// k = 4 5.32 against 5.80).
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double add_dpp(double x)
{
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, ROWS, 0xf, false);
    return x + __hiloint2double(hi, lo);       // lanes outside ROWS add 0
}

// the sum of a row of 16 lanes, in all of them
__device__ __forceinline__ double row_sum(double x)
{
    x = add_dpp<0xb1>(x);                      // quad_perm [1,0,3,2]
    x = add_dpp<0x4e>(x);                      // quad_perm [2,3,0,1]
    x = add_dpp<0x141>(x);                     // row_half_mirror
    return add_dpp<0x140>(x);                  // row_mirror
}

// the sum of a wave, in its last lane
__device__ __forceinline__ double wave_sum(double x)
{
    x = row_sum(x);
    x = add_dpp<0x142, 0xa>(x);                // row_bcast:15 into rows 1 and 3
    return add_dpp<0x143, 0xc>(x);             // row_bcast:31 into rows 2 and 3
}

template <int BLOCK>
__device__ __forceinline__ double block_sum(double x, double *lds)
{
    constexpr int NW = BLOCK / 64;
    static_assert(NW >= 1 && NW <= 16, "the waves' sums lie in one row of lanes");
    x = wave_sum(x);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    double t = 0.0;
    if (wave == 0) t = row_sum(lane < NW ? lds[lane] : 0.0);
    return t;   // valid in thread 0
}

}  // namespace gs
#endif
