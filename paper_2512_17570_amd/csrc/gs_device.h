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

// Past the die's L2 too, which otherwise keeps the line dirty and sends it out later, in an order of its own.  No builtin gives this
// pair of cache bits.  A store of more than 64 bits goes on reading its registers for up to two cycles, in which none may be written:
// hence the s_nop.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void store_through(u32x4 *p, u32x4 v)
{
    asm volatile("global_store_dwordx4 %0, %1, off sc1 nt\n\ts_nop 1" ::"v"(p), "v"(v) : "memory");
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

// ---- the last of a launch's workgroups finishes it ----------------------------------------------
// Of a small launch a second one, for what its workgroups leave, is the larger part: 3.7 us of a stream's time each, whatever they
// do.  So each leaves W 32-bit words in the caller's workspace, then looks whether all n have, and the last to look sees that they have.
//   - Nothing has to be in the workspace before: a word lies beside a tag of this launch, in one 64-bit store, and counts only with
//     it.  Tags are the upper halves of signalling NaNs, which no sum in 64 bits has; who leaves other words there sees to it.
//   - Two may see all n: the one that takes the tag out of the first slot finishes; or both do, with the same result.
//   - Whoever finishes clears the slots, so a graph, whose launches have the same tag every time, finds none of its own.
//   - Nobody waits for another workgroup.
// The words go to memory and come from there by atomic accesses of the device's scope: the dies' caches do not see each other's
// lines.  A workgroup's own are there (vmcnt) before it looks at the others'.
struct Meeting {
    uint64_t *slots;
    uint32_t tag;
    int n;                        // 0: no meeting, another launch finishes
};
constexpr int MEET_MAX = 256;     // every workgroup reads the slots of all
// word q of slot i: those of a kind side by side, so that a wave's loads are whole lines
__device__ __forceinline__ uint64_t *word(const Meeting &M, int i, int q) { return M.slots + (int64_t)q * M.n + i; }

// by lane 0 of the wave that looks afterwards; alone, there is nothing to leave
template <int W>
__device__ __forceinline__ void leave(const Meeting &M, int me, const uint32_t (&w)[W])
{
    if (M.n == 1) return;
#pragma unroll
    for (int i = 0; i < W; ++i)
        __hip_atomic_store(word(M, me, i), (uint64_t)M.tag << 32 | w[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// By the whole wave, whose lane 0 has in w what it has left: true in the workgroup that finishes, with the words of slot `lane` in w;
// left_words() has those of later slots.  Up to 64 slots and with `again` (a result may be written twice) every one that sees all may, since it
// has all it needs.
template <int W>
__device__ __forceinline__ bool last_of(const Meeting &M, bool again, uint32_t (&w)[W])
{
    if (M.n == 1) {
        if ((threadIdx.x & 63) != 0)
#pragma unroll
            for (int q = 0; q < W; ++q) w[q] = 0;
        return true;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const int lane = threadIdx.x & 63;
    bool here = true;
#pragma unroll
    for (int q = 0; q < W; ++q) w[q] = 0;
#pragma unroll 1
    for (int i = lane; i < M.n; i += 64) {
        uint64_t x[W];
#pragma unroll
        for (int q = 0; q < W; ++q) x[q] = __hip_atomic_load(word(M, i, q), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int q = 0; q < W; ++q) {
            here = here && (uint32_t)(x[q] >> 32) == M.tag;
            if (i < 64) w[q] = (uint32_t)x[q];
        }
    }
    if (__ballot(here) != ~0ull) return false;
    if (M.n <= 64 && again) return true;
    uint32_t tag = 0;
    if (lane == 0) tag = (uint32_t)(__hip_atomic_fetch_and(M.slots, (uint64_t)0xffffffffu, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) >> 32);
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)tag) == M.tag;
}
template <int W>
__device__ __forceinline__ void left_words(const Meeting &M, int i, uint32_t (&w)[W])
{
#pragma unroll
    for (int q = 0; q < W; ++q) w[q] = (uint32_t)__hip_atomic_load(word(M, i, q), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <int W>
__device__ __forceinline__ void clear(const Meeting &M)
{
    if (M.n == 1) return;
    for (int i = threadIdx.x & 63; i < M.n * W; i += 64) __hip_atomic_store(M.slots + i, (uint64_t)0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// W / 2 doubles a slot, summed over all of them in a fixed order, in the wave's last lane
template <int W>
__device__ __forceinline__ void left_sums(const Meeting &M, uint32_t (&w)[W], double (&x)[W / 2])
{
#pragma unroll
    for (int q = 0; q < W / 2; ++q) x[q] = __hiloint2double((int)w[2 * q + 1], (int)w[2 * q]);       // 0 without a slot
#pragma unroll 1
    for (int i = (threadIdx.x & 63) + 64; i < M.n; i += 64) {
        left_words(M, i, w);
#pragma unroll
        for (int q = 0; q < W / 2; ++q) x[q] += __hiloint2double((int)w[2 * q + 1], (int)w[2 * q]);
    }
#pragma unroll
    for (int q = 0; q < W / 2; ++q) x[q] = wave_sum(x[q]);
}
__device__ __forceinline__ void halves(double x, uint32_t &lo, uint32_t &hi)
{
    lo = (uint32_t)__double2loint(x);
    hi = (uint32_t)__double2hiint(x);
}

}  // namespace gs
#endif
