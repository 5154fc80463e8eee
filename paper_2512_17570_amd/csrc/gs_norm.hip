// gs_norm.hip -- what a layer has around its products: layer norm of rows with its gradient, and dropout onto the residual stream.
//
// All of it is one pass over memory: read once, written once, so HBM is the bound; the arithmetic (ten operations an element, one eighth of
// a Philox block for dropout) goes on beside it.
//   * a row stays in the registers of its team (a wave, four or sixteen) from its first load to its last store; rows that none holds
//     are read again
//   * vectors of 16 bytes at any address the element type allows: the hardware takes them from wherever they lie
//
// 16384 x 8192 bf16: norm 94 us (5.7 TB/s), gradient 148 (5.4), dropout onto a residual 122 to 124 (6.6; a copy on this card 6.7).  One row of 8192 4.2 us,
// dropout of 257 x 1024 4.0, where a launch takes 3.7.  Pass after pass; in the first milliseconds of a load the clock moves, and the gradient takes up to 190.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "gs_device.h"
#include "gs_internal.h"

#pragma clang fp contract(off)

namespace gs {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// ---- an element type, and vectors of it at any of its addresses -----------------------------------
template <int ALIGN> struct Loose;
template <> struct Loose<2> { typedef u32x4 T __attribute__((aligned(2))); };
template <> struct Loose<4> { typedef u32x4 T __attribute__((aligned(4))); };
struct Bf16 {
    typedef uint16_t T;
    static constexpr int PER = 8;
    static __device__ __forceinline__ float load(const T *p) { return __uint_as_float((uint32_t)*p << 16); }
    static __device__ __forceinline__ void store(T *p, float f) { *p = (T)f32_to_bf16_bits(f); }
    static __device__ __forceinline__ void widen(u32x4 q, float (&z)[PER])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[2 * i] = bf16_lo(q[i]), z[2 * i + 1] = bf16_hi(q[i]);
    }
    static __device__ __forceinline__ u32x4 narrow(const float (&g)[PER])
    {
        u32x4 q;
#pragma unroll
        for (int i = 0; i < 4; ++i) {                 // rounded to nearest even, NaN stays NaN
            bf16x2 h = {(__bf16)g[2 * i], (__bf16)g[2 * i + 1]};
            q[i] = __builtin_bit_cast(uint32_t, h);
        }
        return q;
    }
};
struct F32 {
    typedef float T;
    static constexpr int PER = 4;
    static __device__ __forceinline__ float load(const T *p) { return *p; }
    static __device__ __forceinline__ void store(T *p, float f) { *p = f; }
    static __device__ __forceinline__ void widen(u32x4 q, float (&z)[PER])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = __uint_as_float(q[i]);
    }
    static __device__ __forceinline__ u32x4 narrow(const float (&g)[PER])
    {
        return u32x4{__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3])};
    }
};

template <typename E> __device__ __forceinline__ u32x4 load_vector(const typename E::T *p)
{
    return *reinterpret_cast<const typename Loose<sizeof(typename E::T)>::T *>(p);
}
// a stream's, which is read once
template <typename E> __device__ __forceinline__ u32x4 load_once(const typename E::T *p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const typename Loose<sizeof(typename E::T)>::T *>(p));
}
// Past the caches where a wave's vectors are whole lines; cut ones (an address off 16 bytes) are left to them to join (4095 x 5003 fp32, dropout: 36 us against 88).
template <typename E> __device__ __forceinline__ void store_vector(typename E::T *p, u32x4 q, bool through)
{
    if (through) store_through(reinterpret_cast<u32x4 *>(p), q);
    else *reinterpret_cast<typename Loose<sizeof(typename E::T)>::T *>(p) = q;
}
// whether rows of vectors all start on 16 bytes
static bool whole_lines(const void *p, int64_t stride_bytes) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)stride_bytes) & 15) == 0; }
// one element in its place of a vector
template <typename E> __device__ __forceinline__ u32x4 vector_of(const typename E::T (&e)[E::PER])
{
    u32x4 q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (E::PER == 8) q[i] = (uint32_t)e[2 * i] | (uint32_t)e[2 * i + 1] << 16;
        else q[i] = __float_as_uint(e[i]);
    }
    return q;
}
// Elements [c, c + PER) of an array that has `n`, as far as it has them; 0 for the others.  WHOLE: n is a multiple of PER.
template <typename E, bool ONCE, bool WHOLE = false> __device__ __forceinline__ u32x4 load_some(const typename E::T *p, int64_t c, int64_t n)
{
    if (WHOLE && c >= n) return u32x4{};
    if (WHOLE || c + E::PER <= n) return ONCE ? load_once<E>(p + c) : load_vector<E>(p + c);
    typename E::T e[E::PER];
#pragma unroll
    for (int i = 0; i < E::PER; ++i) e[i] = c + i < n ? p[c + i] : (typename E::T)0;
    return vector_of<E>(e);
}
template <typename E, bool WHOLE = false> __device__ __forceinline__ void store_some(typename E::T *p, int64_t c, int64_t n, const float (&z)[E::PER], bool through)
{
    if (WHOLE || c + E::PER <= n) {
        store_vector<E>(p + c, E::narrow(z), through);
    } else {
#pragma unroll
        for (int i = 0; i < E::PER; ++i)
            if (c + i < n) E::store(p + c + i, z[i]);
    }
}
// PER values of the scale or the shift, in a type of their own, as they lie there: `none` without an array
template <typename W, int PER, bool WHOLE = false> struct Weights {
    static constexpr int N = PER / W::PER ? PER / W::PER : 1;        // vectors; of bf16 beside fp32 rows, half of one
    u32x4 q[N];
    __device__ __forceinline__ void load(const void *w, int64_t c, int64_t n, float none)
    {
        const typename W::T *p = static_cast<const typename W::T *>(w);
        if (!p) {
            float f[W::PER];
#pragma unroll
            for (int i = 0; i < W::PER; ++i) f[i] = none;
#pragma unroll
            for (int v = 0; v < N; ++v) q[v] = W::narrow(f);
        } else if constexpr (W::PER <= PER) {
#pragma unroll
            for (int v = 0; v < N; ++v) q[v] = load_some<W, false, WHOLE>(p, c + v * W::PER, n);
        } else {
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            typedef u32x2 loose_u32x2 __attribute__((aligned(2)));
            if (WHOLE && c >= n) {
                q[0] = u32x4{};
            } else if (WHOLE || c + PER <= n) {
                const u32x2 h = *reinterpret_cast<const loose_u32x2 *>(p + c);
                q[0] = u32x4{h[0], h[1], 0, 0};
            } else {
                q[0] = load_some<W, false>(p, c, n);
            }
        }
    }
    __device__ __forceinline__ void get(float (&z)[PER]) const
    {
#pragma unroll
        for (int v = 0; v < N; ++v) {
            float f[W::PER];
            W::widen(q[v], f);
#pragma unroll
            for (int i = 0; i < W::PER && v * W::PER + i < PER; ++i) z[v * W::PER + i] = f[i];
        }
    }
};

// ---- sums of a team -----------------------------------------------------------------------------
template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ float add_dpp32(float x)
{
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float row_sum32(float x)
{
    x = add_dpp32<0xb1>(x);
    x = add_dpp32<0x4e>(x);
    x = add_dpp32<0x141>(x);
    return add_dpp32<0x140>(x);
}
// the sum of a wave, in all its lanes
__device__ __forceinline__ float wave_sum32(float x)
{
    x = row_sum32(x);
    x = add_dpp32<0x142, 0xa>(x);
    x = add_dpp32<0x143, 0xc>(x);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
// N sums over the lanes of a team, in all of them; `lds` has a place for each of the team's waves, used by this sum alone until the next barrier
template <int TEAM, int N> __device__ __forceinline__ void team_sums(float (&x)[N], float *lds)
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = wave_sum32(x[i]);
    if constexpr (TEAM > 64) {
        constexpr int NW = TEAM / 64;
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) lds[i * NW + wave] = x[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float t = row_sum32((lane & 15) < NW ? lds[i * NW + (lane & 15)] : 0.0f);
            x[i] = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(t)));
        }
    }
}

// Elements are kept as they came and widened each time: without this the compiler keeps the widened ones, in twice the registers (bf16).
__device__ __forceinline__ void as_it_came(u32x4 &q) { asm("" : "+v"(q)); }

// ---- forward -------------------------------------------------------------------------------------
struct NormArgs {
    const void *x;
    int64_t rows, cols, stride;
    const void *gamma, *beta;
    float eps;
    void *y;
    int64_t y_stride;
    float *stats;
    bool through;
};
// A row a team, NV vectors a lane; HELD: they hold the row, else it is read three times.  EARLY: scale and shift are on their way while the sums are taken, which
// is a trip to memory less where the time is a chain of them, and as many registers again (one row of 8192: 3.0 us against 4.6).
template <typename E, typename W, int TEAM, int NV, bool HELD, bool EARLY>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void k_norm(NormArgs A)
{
    constexpr int TEAMS = TEAM < 256 ? 256 / TEAM : 1, PER = E::PER;
    __shared__ float lds[2][TEAM / 64];
    const int64_t row = (int64_t)blockIdx.x * TEAMS + (TEAMS > 1 ? threadIdx.x / TEAM : 0);
    if (TEAMS > 1 && row >= A.rows) return;
    const int lane = TEAMS > 1 ? threadIdx.x % TEAM : threadIdx.x;
    const int64_t n = A.cols;
    const typename E::T *x = static_cast<const typename E::T *>(A.x) + row * A.stride;
    typename E::T *y = static_cast<typename E::T *>(A.y) + row * A.y_stride;
    u32x4 q[NV];
    Weights<W, PER> gamma[NV], beta[NV];
    float z[PER], sum[1] = {0.0f};
    const int64_t by = (int64_t)TEAM * PER;
    if constexpr (HELD) {
#pragma unroll
        for (int v = 0; v < NV; ++v) q[v] = load_some<E, true>(x, v * by + lane * PER, n);
#pragma unroll
        for (int v = 0; EARLY && v < NV; ++v) {
            gamma[v].load(A.gamma, v * by + lane * PER, n, 1.0f);
            beta[v].load(A.beta, v * by + lane * PER, n, 0.0f);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            E::widen(q[v], z);
#pragma unroll
            for (int i = 0; i < PER; ++i) sum[0] += z[i];
        }
    } else {
        for (int64_t c = lane * PER; c < n; c += by) {
            E::widen(load_some<E, false>(x, c, n), z);
#pragma unroll
            for (int i = 0; i < PER; ++i) sum[0] += z[i];
        }
    }
    team_sums<TEAM>(sum, lds[0]);
    const float mean = sum[0] / (float)n;
    sum[0] = 0.0f;
    auto squares = [&](int64_t c, u32x4 v) {
        E::widen(v, z);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const float d = z[i] - mean;
            if (c + i < n) sum[0] += d * d;
        }
    };
    if constexpr (HELD) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            as_it_came(q[v]);
            squares(v * by + lane * PER, q[v]);
        }
    } else {
        for (int64_t c = lane * PER; c < n; c += by) squares(c, load_some<E, false>(x, c, n));
    }
    team_sums<TEAM>(sum, lds[1]);
    const float rstd = 1.0f / sqrtf(sum[0] / (float)n + A.eps);
    if (A.stats && lane == 0) A.stats[2 * row] = mean, A.stats[2 * row + 1] = rstd;
    auto write = [&](int64_t c, u32x4 v, const Weights<W, PER> &gv, const Weights<W, PER> &bv) {
        float g[PER], b[PER];
        E::widen(v, z);
        gv.get(g);
        bv.get(b);
#pragma unroll
        for (int i = 0; i < PER; ++i) z[i] = (z[i] - mean) * rstd * g[i] + b[i];
        store_some<E>(y, c, n, z, A.through);
    };
    if constexpr (HELD) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = v * by + lane * PER;
            if (c >= n) continue;
            if (!EARLY) {
                gamma[v].load(A.gamma, c, n, 1.0f);
                beta[v].load(A.beta, c, n, 0.0f);
            }
            as_it_came(q[v]);
            write(c, q[v], gamma[v], beta[v]);
        }
    } else {
        for (int64_t c = lane * PER; c < n; c += by) {
            gamma[0].load(A.gamma, c, n, 1.0f);
            beta[0].load(A.beta, c, n, 0.0f);
            write(c, load_some<E, false>(x, c, n), gamma[0], beta[0]);
        }
    }
}

// The same for many rows: workgroups that stay, take rows in turn and have the next one on its way while one is worked on; scale and shift are read once.
// 16384 x 8192 bf16 94 us, where a workgroup a row takes 137 (its loads, its two sums and its stores follow one another).
template <typename E, typename W, int TEAM, int NV, bool WHOLE>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void k_norm_many(NormArgs A)
{
    constexpr int TEAMS = TEAM < 256 ? 256 / TEAM : 1, PER = E::PER;
    __shared__ float lds[2][2][TEAM / 64];
    const int team = TEAMS > 1 ? threadIdx.x / TEAM : 0, lane = TEAMS > 1 ? threadIdx.x % TEAM : threadIdx.x;
    const int64_t n = A.cols, by = (int64_t)TEAM * PER, step = (int64_t)gridDim.x * TEAMS;
    Weights<W, PER, WHOLE> gamma[NV], beta[NV];
    u32x4 q[2][NV];
    auto fetch = [&](int64_t row, int to) {
        const typename E::T *x = static_cast<const typename E::T *>(A.x) + row * A.stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) q[to][v] = load_some<E, true, WHOLE>(x, v * by + lane * PER, n);
    };
    auto work = [&](int64_t row, int at) {
        float z[PER], sum[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            E::widen(q[at][v], z);
#pragma unroll
            for (int i = 0; i < PER; ++i) sum[0] += z[i];
        }
        team_sums<TEAM>(sum, lds[at][0]);
        const float mean = sum[0] / (float)n;
        sum[0] = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            as_it_came(q[at][v]);
            E::widen(q[at][v], z);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float d = z[i] - mean;
                if (v * by + lane * PER + (WHOLE ? 0 : i) < n) sum[0] += d * d;
            }
        }
        team_sums<TEAM>(sum, lds[at][1]);
        const float rstd = 1.0f / sqrtf(sum[0] / (float)n + A.eps);
        if (A.stats && lane == 0) A.stats[2 * row] = mean, A.stats[2 * row + 1] = rstd;
        typename E::T *y = static_cast<typename E::T *>(A.y) + row * A.y_stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float g[PER], b[PER];
            as_it_came(q[at][v]);
#pragma unroll
            for (int i = 0; i < gamma[v].N; ++i) as_it_came(gamma[v].q[i]), as_it_came(beta[v].q[i]);
            E::widen(q[at][v], z);
            gamma[v].get(g);
            beta[v].get(b);
#pragma unroll
            for (int i = 0; i < PER; ++i) z[i] = (z[i] - mean) * rstd * g[i] + b[i];
            if (v * by + lane * PER < n) store_some<E, WHOLE>(y, v * by + lane * PER, n, z, A.through);
        }
    };
    int64_t row = (int64_t)blockIdx.x * TEAMS + team;
    if (row < A.rows) fetch(row, 0);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        gamma[v].load(A.gamma, v * by + lane * PER, n, 1.0f);
        beta[v].load(A.beta, v * by + lane * PER, n, 0.0f);
    }
    for (; row < A.rows; row += 2 * step) {
        if (row + step < A.rows) fetch(row + step, 1);
        work(row, 0);
        if (row + step >= A.rows) break;
        if (row + 2 * step < A.rows) fetch(row + 2 * step, 0);
        work(row + step, 1);
    }
}

// ---- backward ------------------------------------------------------------------------------------
struct NormGradArgs {
    const void *x, *dy;
    void *dx;
    int64_t rows, cols, stride, dy_stride, dx_stride;
    const void *gamma;
    const float *stats;
    float *partials;          // [workgroup][2][cols], or null
    bool through;
};
// Rows dealt in turn to the workgroups' teams, which add up dy xhat and dy of their own rows for each column; a workgroup's teams join theirs in LDS.  The next
// row is on its way while one is worked on, unless the registers of 1024 lanes have no room for it.  16384 x 8192 bf16 143 us (5.6 TB/s) of the gradient's 148, 1023 x 1001
// fp32 7 of 12; 8192 x 16384 bf16 152 with the fold, 8192 x 8192 fp32 141.
template <typename E, typename W, int TEAM, int NV, bool WHOLE>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void k_norm_grad(NormGradArgs A)
{
    constexpr int BLOCK = TEAM < 256 ? 256 : TEAM, TEAMS = BLOCK / TEAM, PER = E::PER, NW = TEAM / 64, BUFFERS = TEAM * NV > 1024 ? 1 : 2;
    __shared__ float lds[2][2 * NW];
    __shared__ float joint[TEAMS > 1 ? TEAMS * TEAM * NV * PER : 1];
    const int team = TEAMS > 1 ? threadIdx.x / TEAM : 0, lane = TEAMS > 1 ? threadIdx.x % TEAM : threadIdx.x;
    const int64_t n = A.cols, by = (int64_t)TEAM * PER, step = (int64_t)gridDim.x * TEAMS;
    Weights<W, PER, WHOLE> gamma[NV];
    float dgamma[NV][PER], dbeta[NV][PER];
    u32x4 x[BUFFERS][NV], dy[BUFFERS][NV];
    float2 stats[BUFFERS];
    auto fetch = [&](int64_t row, int to) {
        const typename E::T *xr = static_cast<const typename E::T *>(A.x) + row * A.stride, *dr = static_cast<const typename E::T *>(A.dy) + row * A.dy_stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            x[to][v] = load_some<E, true, WHOLE>(xr, v * by + lane * PER, n);
            dy[to][v] = load_some<E, true, WHOLE>(dr, v * by + lane * PER, n);
        }
        stats[to] = float2{A.stats[2 * row], A.stats[2 * row + 1]};
    };
    int turn = 0;
    auto work = [&](int64_t row, int at) {
        const float mean = stats[at].x, rstd = stats[at].y;
        float z[PER], d[PER], g[PER], sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            E::widen(x[at][v], z);
            E::widen(dy[at][v], d);
            gamma[v].get(g);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                z[i] = (z[i] - mean) * rstd;                 // behind the row d is 0
                dgamma[v][i] += d[i] * z[i];
                dbeta[v][i] += d[i];
                d[i] *= g[i];
                sum[0] += d[i];
                sum[1] += d[i] * z[i];
            }
            if (BUFFERS == 1) __builtin_amdgcn_sched_barrier(0);       // one vector's widened values at a time
        }
        team_sums<TEAM>(sum, lds[turn]);
        turn ^= 1;
        const float a = sum[0] / (float)n, b = sum[1] / (float)n;
        typename E::T *dx = static_cast<typename E::T *>(A.dx) + row * A.dx_stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            as_it_came(x[at][v]);
            as_it_came(dy[at][v]);
#pragma unroll
            for (int i = 0; i < gamma[v].N; ++i) as_it_came(gamma[v].q[i]);
            E::widen(x[at][v], z);
            E::widen(dy[at][v], d);
            gamma[v].get(g);
#pragma unroll
            for (int i = 0; i < PER; ++i) d[i] = rstd * (d[i] * g[i] - a - (z[i] - mean) * rstd * b);
            if (v * by + lane * PER < n) store_some<E, WHOLE>(dx, v * by + lane * PER, n, d, A.through);
            if (BUFFERS == 1) __builtin_amdgcn_sched_barrier(0);
        }
    };
    int64_t row = (int64_t)blockIdx.x * TEAMS + team;
    if (row < A.rows) fetch(row, 0);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        gamma[v].load(A.gamma, v * by + lane * PER, n, 1.0f);
#pragma unroll
        for (int i = 0; i < PER; ++i) dgamma[v][i] = dbeta[v][i] = 0.0f;
    }
    for (; BUFFERS == 1 && row < A.rows; row += step) {
        work(row, 0);
        if (row + step < A.rows) fetch(row + step, 0);
    }
    for (; row < A.rows; row += 2 * step) {
        if (row + step < A.rows) fetch(row + step, BUFFERS - 1);
        work(row, 0);
        if (row + step >= A.rows) break;
        if (row + 2 * step < A.rows) fetch(row + 2 * step, 0);
        work(row + step, BUFFERS - 1);
    }
    if (!A.partials) return;
    float *out = A.partials + (int64_t)blockIdx.x * 2 * n;
#pragma unroll
    for (int q = 0; q < 2; ++q, out += n) {
        if constexpr (TEAMS == 1) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int h = 0; h < PER; h += 4) {
                    const float *f = (q ? dbeta[v] : dgamma[v]) + h;
                    const float four[4] = {f[0], f[1], f[2], f[3]};
                    const int64_t c = v * by + lane * PER + h;
                    if (WHOLE ? c < n : c + 4 <= n) {
                        *reinterpret_cast<Loose<4>::T *>(out + c) = F32::narrow(four);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (c + i < n) out[c + i] = four[i];
                    }
                }
        } else {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < PER; ++i) joint[team * (TEAM * NV * PER) + v * by + lane * PER + i] = q ? dbeta[v][i] : dgamma[v][i];
            __syncthreads();
            for (int c = threadIdx.x; c < n; c += BLOCK) {
                float s = 0.0f;
                for (int t = 0; t < TEAMS; ++t) s += joint[t * (TEAM * NV * PER) + c];
                out[c] = s;
            }
        }
    }
}
// Rows that no team holds: dx from two readings, a row a workgroup (8192 x 16384 fp32, with the columns' sums and the fold, 571 us, 2.8 TB/s of what has to move; 8191 x 16383 bf16 484,
// 8191 x 8191 fp32 319);
template <typename E, typename W>
__global__ __launch_bounds__(1024) void k_norm_grad_long(NormGradArgs A)
{
    constexpr int PER = E::PER;
    __shared__ float lds[32];
    const int64_t row = blockIdx.x, n = A.cols;
    const typename E::T *x = static_cast<const typename E::T *>(A.x) + row * A.stride;
    const typename E::T *dy = static_cast<const typename E::T *>(A.dy) + row * A.dy_stride;
    typename E::T *dx = static_cast<typename E::T *>(A.dx) + row * A.dx_stride;
    const float mean = A.stats[2 * row], rstd = A.stats[2 * row + 1];
    float z[PER], d[PER], g[PER], sum[2] = {0.0f, 0.0f};
    Weights<W, PER> gamma;
    for (int64_t c = threadIdx.x * PER; c < n; c += 1024 * PER) {
        E::widen(load_some<E, false>(x, c, n), z);
        E::widen(load_some<E, false>(dy, c, n), d);
        gamma.load(A.gamma, c, n, 1.0f);
        gamma.get(g);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            d[i] *= g[i];
            sum[0] += d[i];
            sum[1] += d[i] * ((z[i] - mean) * rstd);
        }
    }
    team_sums<1024>(sum, lds);
    const float a = sum[0] / (float)n, b = sum[1] / (float)n;
    for (int64_t c = threadIdx.x * PER; c < n; c += 1024 * PER) {
        E::widen(load_some<E, false>(x, c, n), z);
        E::widen(load_some<E, false>(dy, c, n), d);
        gamma.load(A.gamma, c, n, 1.0f);
        gamma.get(g);
#pragma unroll
        for (int i = 0; i < PER; ++i) d[i] = rstd * (d[i] * g[i] - a - (z[i] - mean) * rstd * b);
        store_some<E>(dx, c, n, d, A.through);
    }
}
// and the columns' sums by themselves (before, since dx may lie where dy does): a lane PER columns, a workgroup a share of the rows
template <typename E>
__global__ __launch_bounds__(256) void k_norm_columns(NormGradArgs A, int64_t per)
{
    constexpr int PER = E::PER;
    const int64_t n = A.cols, c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * PER;
    if (c >= n) return;
    const int64_t from = blockIdx.y * per, to = from + per < A.rows ? from + per : A.rows;
    float dgamma[PER] = {}, dbeta[PER] = {};
    for (int64_t row = from; row < to; ++row) {
        float z[PER], d[PER];
        E::widen(load_some<E, false>(static_cast<const typename E::T *>(A.x) + row * A.stride, c, n), z);
        E::widen(load_some<E, false>(static_cast<const typename E::T *>(A.dy) + row * A.dy_stride, c, n), d);
        const float mean = A.stats[2 * row], rstd = A.stats[2 * row + 1];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            dgamma[i] += d[i] * ((z[i] - mean) * rstd);
            dbeta[i] += d[i];
        }
    }
    float *out = A.partials + (int64_t)blockIdx.y * 2 * n;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (c + i < n) out[c + i] = dgamma[i], out[n + c + i] = dbeta[i];
}
// Sums over the workgroups: a lane a column of one of the two, 16 waves that each take a share; joined in 64 bits.  A launch of its own
// (3.5 to 5 us), since it takes many workgroups: one alone reads 512 partials of 1024 columns in 30 us, 256 of 8192 in 148 (110 to 140 GB/s).
template <typename W>
__global__ __launch_bounds__(1024) void k_norm_fold(const float *partials, int parts, int64_t cols, void *dgamma, void *dbeta)
{
    __shared__ double part[16][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    double s = 0.0;
    if (c < 2 * cols) {
#pragma unroll 8
        for (int i = wave; i < parts; i += 16) s += (double)partials[(int64_t)i * 2 * cols + c];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= 2 * cols) return;
    s = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += part[i][lane];
    W::store(static_cast<typename W::T *>(c < cols ? dgamma : dbeta) + (c < cols ? c : c - cols), (float)s);
}

// ---- dropout -------------------------------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011): ten rounds of two 32 x 32 bit products.
__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c[0], b = (uint64_t)0xCD9E8D57u * c[2];
        const uint32_t n0 = (uint32_t)(b >> 32) ^ c[1] ^ k0, n2 = (uint32_t)(a >> 32) ^ c[3] ^ k1;
        c[0] = n0, c[1] = (uint32_t)b, c[2] = n2, c[3] = (uint32_t)a;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
}
struct DropoutArgs {
    const void *x, *residual;
    void *out;
    int64_t n;
    uint64_t offset, vectors;     // vectors by their first elements' numbers, the first and last perhaps in part
    uint32_t least;               // T
    float scale;                  // 1 / (1 - P)
    uint32_t k0, k1;
    const uint64_t *step;
    bool through;
};
constexpr int DROP_BLOCK = 256;
// A vector a lane: a block of the generator for eight bf16, half of one for four fp32 (two lanes make the same block, which costs less than accesses of half
// lines: 4095 x 5003 with a residual 40 us against 50).
template <typename E, bool RESIDUAL>
__global__ __launch_bounds__(DROP_BLOCK) void k_dropout(DropoutArgs A)
{
    constexpr int PER = E::PER;
    const uint64_t u = (uint64_t)blockIdx.x * DROP_BLOCK + threadIdx.x;
    if (u >= A.vectors) return;
    const uint64_t number = A.offset / PER + u;
    const int64_t at = (int64_t)(u * PER) - (int64_t)(A.offset % PER);       // of its first element, which may lie before the array
    const typename E::T *x = static_cast<const typename E::T *>(A.x), *res = static_cast<const typename E::T *>(A.residual);
    typename E::T *out = static_cast<typename E::T *>(A.out);
    const bool whole = at >= 0 && at + PER <= A.n;
    float z[PER], r[PER];
    if (whole) {
        E::widen(load_once<E>(x + at), z);
        if (RESIDUAL) E::widen(load_once<E>(res + at), r);
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int64_t e = at + i;
            const bool there = e >= 0 && e < A.n;
            z[i] = there ? E::load(x + e) : 0.0f;
            r[i] = RESIDUAL && there ? E::load(res + e) : 0.0f;
        }
    }
    const uint64_t step = A.step ? *A.step : 0, block = number * PER / 8;
    uint32_t c[4] = {(uint32_t)block, (uint32_t)(block >> 32), (uint32_t)step, (uint32_t)(step >> 32)};
    philox(c, A.k0, A.k1);
    if (PER == 4 && (number & 1)) c[0] = c[2], c[1] = c[3];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t bits = i & 1 ? c[i >> 1] >> 16 : c[i >> 1] & 0xffffu;
        z[i] = bits >= A.least ? z[i] * A.scale : 0.0f;
        if (RESIDUAL) z[i] += r[i];
    }
    if (whole) {
        store_vector<E>(out + at, E::narrow(z), A.through);
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int64_t e = at + i;
            if (e >= 0 && e < A.n) E::store(out + e, z[i]);
        }
    }
}

// ---- launches ------------------------------------------------------------------------------------
constexpr int64_t kMaxItems = 0xffffffffLL;      // HIP launches fewer than 2^32 work items at a time
// Rows of more than 1024 vectors are a workgroup's in any case (8192 x 8192 fp32 97 us, 5.5 TB/s, 8192 x 16384 bf16 105, of odd width 166); of more than 4096 they are read three
// times (8192 x 32768 bf16, the last that are held, 272).
// Rows up to which a row's own time counts: a workgroup a row (with more of them, the ones that stay: 512 x 4096 bf16 3.8 us, a workgroup a row 4.6; 768
// x 4096 4.1 and 6.3, 256 x 8192 3.9 and 3.8).
constexpr int64_t NORM_FEW = 256;
// Of workgroups that stay: 1024 a CU.  16384 x 8192 bf16, two of 512 lanes x 2 vectors 93.4 us, four of 256 x 4 93.1, one of 1024 x 1 102; with 2048
// lanes a CU 93.0.
constexpr int64_t NORM_LANES = 256 * 1024;
constexpr int NORM_PARTS = 512;                  // workgroups of a gradient, and partials of its columns (16384 x 8192 148 us, of 1024 154)

template <typename E, typename W, int TEAM, int NV, bool HELD, bool EARLY>
static hipError_t launch_norm_as(const NormArgs &A, hipStream_t stream)
{
    constexpr int BLOCK = TEAM < 256 ? 256 : TEAM, TEAMS = BLOCK / TEAM;
    const int64_t most = kMaxItems / BLOCK * TEAMS;
    for (int64_t r = 0; r < A.rows; r += most) {
        NormArgs B = A;
        B.x = static_cast<const typename E::T *>(A.x) + r * A.stride;
        B.y = static_cast<typename E::T *>(A.y) + r * A.y_stride;
        B.stats = A.stats ? A.stats + 2 * r : nullptr;
        B.rows = std::min(most, A.rows - r);
        k_norm<E, W, TEAM, NV, HELD, EARLY><<<(uint32_t)((B.rows + TEAMS - 1) / TEAMS), BLOCK, 0, stream>>>(B);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename E, typename W, int TEAM, int NV>
static hipError_t launch_norm_many(const NormArgs &A, hipStream_t stream)
{
    constexpr int BLOCK = TEAM < 256 ? 256 : TEAM, TEAMS = BLOCK / TEAM;
    const uint32_t grid = (uint32_t)std::min<int64_t>(NORM_LANES / BLOCK, (A.rows + TEAMS - 1) / TEAMS);
    if (A.cols % E::PER == 0) k_norm_many<E, W, TEAM, NV, true><<<grid, BLOCK, 0, stream>>>(A);
    else k_norm_many<E, W, TEAM, NV, false><<<grid, BLOCK, 0, stream>>>(A);
    return hipGetLastError();
}
template <typename E, typename W>
static hipError_t launch_norm(const NormArgs &A, hipStream_t stream)
{
    const int64_t v = (A.cols + E::PER - 1) / E::PER;
    if (v <= 64) return launch_norm_as<E, W, 64, 1, true, true>(A, stream);
    if (A.rows <= NORM_FEW && v <= 1024) {
        if (v <= 256) return launch_norm_as<E, W, 256, 1, true, true>(A, stream);
        return launch_norm_as<E, W, 1024, 1, true, true>(A, stream);
    }
    if (v <= 128) return launch_norm_many<E, W, 64, 2>(A, stream);
    if (v <= 256) return launch_norm_many<E, W, 256, 1>(A, stream);
    if (v <= 512) return launch_norm_many<E, W, 256, 2>(A, stream);
    if (v <= 1024) return launch_norm_many<E, W, 512, 2>(A, stream);
    if (v <= 2048) return launch_norm_as<E, W, 1024, 2, true, false>(A, stream);
    if (v <= 4096) return launch_norm_as<E, W, 1024, 4, true, false>(A, stream);
    return launch_norm_as<E, W, 1024, 1, false, false>(A, stream);
}

// Workgroups of a gradient over rows that are held: all that fit the chip at once, two a CU, or one of 1024 lanes.
template <typename E, typename W, int TEAM, int NV>
static hipError_t launch_norm_grad_as(const NormGradArgs &A, int &parts, hipStream_t stream)
{
    constexpr int BLOCK = TEAM < 256 ? 256 : TEAM, TEAMS = BLOCK / TEAM;
    parts = (int)std::min<int64_t>(BLOCK == 1024 ? NORM_PARTS / 2 : NORM_PARTS, (A.rows + TEAMS - 1) / TEAMS);
    if constexpr (TEAM * NV > 1024) k_norm_grad<E, W, TEAM, NV, true><<<parts, BLOCK, 0, stream>>>(A);
    else if (A.cols % E::PER == 0) k_norm_grad<E, W, TEAM, NV, true><<<parts, BLOCK, 0, stream>>>(A);
    else k_norm_grad<E, W, TEAM, NV, false><<<parts, BLOCK, 0, stream>>>(A);
    return hipGetLastError();
}
template <typename E, typename W>
static hipError_t launch_norm_grad(const NormGradArgs &A, void *dgamma, void *dbeta, hipStream_t stream)
{
    const int64_t v = (A.cols + E::PER - 1) / E::PER;
    int parts = 0;
    hipError_t e = hipSuccess;
    if (A.rows == 0) {
    } else if (v <= 64) e = launch_norm_grad_as<E, W, 64, 1>(A, parts, stream);
    else if (v <= 128) e = launch_norm_grad_as<E, W, 64, 2>(A, parts, stream);
    else if (v <= 256) e = launch_norm_grad_as<E, W, 256, 1>(A, parts, stream);
    else if (v <= 512) e = launch_norm_grad_as<E, W, 512, 1>(A, parts, stream);
    else if (v <= 1024) e = launch_norm_grad_as<E, W, 1024, 1>(A, parts, stream);
    else if (v <= 2048 && A.cols % E::PER == 0) e = launch_norm_grad_as<E, W, 1024, 2>(A, parts, stream);      // 1024 lanes have no registers for cut vectors
    else {
        if (A.partials) {
            const int64_t blocks = (v + 255) / 256, wanted = std::min<int64_t>(NORM_PARTS, std::max<int64_t>(1, 2048 / blocks)), per = (A.rows + wanted - 1) / wanted;
            parts = (int)((A.rows + per - 1) / per);
            k_norm_columns<E><<<dim3((uint32_t)blocks, (uint32_t)parts), 256, 0, stream>>>(A, per);
            e = hipGetLastError();
        }
        const int64_t most = kMaxItems / 1024;
        for (int64_t r = 0; r < A.rows && e == hipSuccess; r += most) {
            NormGradArgs B = A;
            B.x = static_cast<const typename E::T *>(A.x) + r * A.stride;
            B.dy = static_cast<const typename E::T *>(A.dy) + r * A.dy_stride;
            B.dx = static_cast<typename E::T *>(A.dx) + r * A.dx_stride;
            B.stats = A.stats + 2 * r;
            k_norm_grad_long<E, W><<<(uint32_t)std::min(most, A.rows - r), 1024, 0, stream>>>(B);
            e = hipGetLastError();
        }
    }
    if (e != hipSuccess || !A.partials) return e;
    k_norm_fold<W><<<(uint32_t)((2 * A.cols + 63) / 64), 1024, 0, stream>>>(A.partials, parts, A.cols, dgamma, dbeta);
    return hipGetLastError();
}

template <typename E>
static hipError_t launch_dropout(DropoutArgs A, hipStream_t stream)
{
    const int64_t most = kMaxItems / DROP_BLOCK * DROP_BLOCK, size = sizeof(typename E::T);       // vectors of a launch
    A.through = whole_lines(static_cast<char *>(A.out) - A.offset % E::PER * size, 0);
    for (uint64_t left = (A.offset % E::PER + (uint64_t)A.n + E::PER - 1) / E::PER; left; left -= A.vectors) {
        A.vectors = std::min<uint64_t>(most, left);
        const uint32_t grid = (uint32_t)((A.vectors + DROP_BLOCK - 1) / DROP_BLOCK);
        if (A.residual) k_dropout<E, true><<<grid, DROP_BLOCK, 0, stream>>>(A);
        else k_dropout<E, false><<<grid, DROP_BLOCK, 0, stream>>>(A);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        // the next launch's first vector begins with the next element
        const int64_t elements = (int64_t)(A.vectors * E::PER - A.offset % E::PER);
        A.x = static_cast<const typename E::T *>(A.x) + elements;
        if (A.residual) A.residual = static_cast<const typename E::T *>(A.residual) + elements;
        A.out = static_cast<typename E::T *>(A.out) + elements;
        A.n -= elements;
        A.offset += elements;
    }
    return hipSuccess;
}

// ---- checks -------------------------------------------------------------------------------------
static bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static bool good(const void *p, uintptr_t to) { return p && aligned(p, to); }
static bool good_type(int32_t t) { return t == GS_BF16 || t == GS_F32; }
static int64_t size_of(int32_t dtype) { return dtype == GS_BF16 ? 2 : 4; }
static bool good_norm_sizes(int64_t rows, int64_t cols) { return rows >= 0 && rows <= (int64_t)1 << 31 && cols >= 1 && cols <= (int64_t)1 << 24; }
// bytes from a matrix's first element to behind its last one; -1 if they do not fit an address
static int64_t extent(int64_t rows, int64_t cols, int64_t stride, int64_t size)
{
    int64_t n;
    if (rows <= 1) return rows * cols * size;
    if (__builtin_mul_overflow(rows - 1, stride, &n) || __builtin_add_overflow(n, cols, &n) || __builtin_mul_overflow(n, size, &n)) return -1;
    return n;
}
static bool good_rows(const gs_matrix &x, const void *p, int64_t stride)
{
    if (x.rows == 0) return true;
    return good(p, size_of(x.dtype)) && (x.rows == 1 || stride >= x.cols) && extent(x.rows, x.cols, stride, size_of(x.dtype)) >= 0;
}
static bool good_matrix(const gs_matrix *x) { return x && good_type(x->dtype) && good_norm_sizes(x->rows, x->cols) && good_rows(*x, x->data, x->row_stride); }
static Range matrix_range(const gs_matrix &x, const void *p, int64_t stride, bool out) { return range_of(p, extent(x.rows, x.cols, stride, size_of(x.dtype)), out); }
static bool apart(const Range *s, int n, bool skip = false, int a = -1, int b = -1)
{
    for (int i = 0; i < n; ++i)
        for (int j = i + 1; j < n; ++j)
            if ((s[i].out || s[j].out) && !(skip && i == a && j == b) && overlap(s[i], s[j])) return false;
    return true;
}
static bool same(const gs_matrix &x, const void *p, int64_t p_stride, const void *q, int64_t q_stride) { return p == q && (x.rows == 1 || p_stride == q_stride); }
template <typename F> static hipError_t by_types(int32_t x, int32_t w, F f)
{
    if (x == GS_BF16) return w == GS_BF16 ? f(Bf16{}, Bf16{}) : f(Bf16{}, F32{});
    return w == GS_BF16 ? f(F32{}, Bf16{}) : f(F32{}, F32{});
}

}  // namespace gs

using namespace gs;

extern "C" {

gs_status gs_layer_norm(const gs_matrix *x, const void *gamma, const void *beta, int32_t weight_dtype, float eps, void *y, int64_t y_stride,
                        float *row_stats, void *stream)
{
    if (!good_matrix(x) || !good_type(weight_dtype) || !(eps >= 0.0f) || !std::isfinite(eps)) return GS_ERR_INVALID_ARG;
    const int64_t wsize = size_of(weight_dtype);
    if (!aligned(gamma, wsize) || !aligned(beta, wsize) || !good_rows(*x, y, y_stride) || !aligned(row_stats, 4)) return GS_ERR_INVALID_ARG;
    if (x->rows == 0) return GS_OK;
    const Range s[] = {matrix_range(*x, x->data, x->row_stride, false), matrix_range(*x, y, y_stride, true), range_of(gamma, x->cols * wsize, false),
                       range_of(beta, x->cols * wsize, false), range_of(row_stats, x->rows * 8, true)};
    if (!apart(s, 5, same(*x, x->data, x->row_stride, y, y_stride), 0, 1)) return GS_ERR_INVALID_ARG;
    const NormArgs A = {x->data, x->rows, x->cols, x->rows > 1 ? x->row_stride : x->cols, gamma, beta, eps, y, x->rows > 1 ? y_stride : x->cols, row_stats,
                        whole_lines(y, (x->rows > 1 ? y_stride : 0) * size_of(x->dtype))};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e = by_types(x->dtype, weight_dtype, [&](auto t, auto w) { return launch_norm<decltype(t), decltype(w)>(A, st); });
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_layer_norm launch");
}

size_t gs_layer_norm_workspace_bytes(int64_t rows, int64_t cols)
{
    if (!good_norm_sizes(rows, cols)) return 0;
    return (size_t)std::max<int64_t>(1, std::min<int64_t>(rows, NORM_PARTS)) * 2 * cols * sizeof(float);
}

gs_status gs_layer_norm_grad(const gs_matrix *x, const void *gamma, int32_t weight_dtype, const float *row_stats, const void *dy,
                             int64_t dy_stride, void *dx, int64_t dx_stride, void *dgamma, void *dbeta, void *d_workspace,
                             size_t workspace_bytes, void *stream)
{
    if (!good_matrix(x) || !good_type(weight_dtype)) return GS_ERR_INVALID_ARG;
    const int64_t wsize = size_of(weight_dtype);
    if (!aligned(gamma, wsize) || !aligned(dgamma, wsize) || !aligned(dbeta, wsize) || !dgamma != !dbeta) return GS_ERR_INVALID_ARG;
    if (!good_rows(*x, dy, dy_stride) || !good_rows(*x, dx, dx_stride) || (x->rows && !good(row_stats, 4))) return GS_ERR_INVALID_ARG;
    if (dgamma && (!good(d_workspace, 256) || workspace_bytes < gs_layer_norm_workspace_bytes(x->rows, x->cols))) return GS_ERR_WORKSPACE;
    if (x->rows == 0 && !dgamma) return GS_OK;
    const Range s[] = {matrix_range(*x, dy, dy_stride, false), matrix_range(*x, dx, dx_stride, true), matrix_range(*x, x->data, x->row_stride, false),
                       range_of(gamma, x->cols * wsize, false), range_of(row_stats, x->rows * 8, false), range_of(dgamma, x->cols * wsize, true),
                       range_of(dbeta, x->cols * wsize, true), range_of(dgamma ? d_workspace : nullptr, (int64_t)workspace_bytes, true)};
    if (!apart(s, 8, x->rows && same(*x, dy, dy_stride, dx, dx_stride), 0, 1)) return GS_ERR_INVALID_ARG;
    const bool many = x->rows > 1;
    const NormGradArgs A = {x->data, dy, dx, x->rows, x->cols, many ? x->row_stride : x->cols, many ? dy_stride : x->cols, many ? dx_stride : x->cols,
                            gamma, row_stats, dgamma ? static_cast<float *>(d_workspace) : nullptr, whole_lines(dx, (many ? dx_stride : 0) * size_of(x->dtype))};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e = by_types(x->dtype, weight_dtype, [&](auto t, auto w) { return launch_norm_grad<decltype(t), decltype(w)>(A, dgamma, dbeta, st); });
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_layer_norm_grad launch");
}

gs_status gs_dropout(const void *x, const void *residual, void *out, int64_t n, int32_t dtype, float p, uint64_t seed, uint64_t offset,
                     const uint64_t *d_step, void *stream)
{
    if (!good_type(dtype) || n < 0 || n > (int64_t)1 << 40 || !(p >= 0.0f && p <= 1.0f) || !aligned(d_step, 8)) return GS_ERR_INVALID_ARG;
    if (n && offset > UINT64_MAX - (uint64_t)(n - 1)) return GS_ERR_INVALID_ARG;
    if (n == 0) return GS_OK;
    const int64_t size = size_of(dtype);
    if (!good(x, size) || !aligned(residual, size) || !good(out, size)) return GS_ERR_INVALID_ARG;
    const Range s[] = {range_of(x, n * size, false), range_of(residual, n * size, false), range_of(out, n * size, true), range_of(d_step, 8, false)};
    for (int i = 0; i < 4; ++i)
        if (i != 2 && !(i < 2 && s[i].lo == s[2].lo) && overlap(s[i], s[2])) return GS_ERR_INVALID_ARG;
    DropoutArgs A = {};
    A.x = x;
    A.residual = residual;
    A.out = out;
    A.n = n;
    A.offset = offset;
    A.least = (uint32_t)std::lround((double)p * 65536.0);
    A.scale = A.least < 65536 ? (float)(65536.0 / (65536.0 - A.least)) : 0.0f;
    A.k0 = (uint32_t)seed;
    A.k1 = (uint32_t)(seed >> 32);
    A.step = d_step;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e = dtype == GS_BF16 ? launch_dropout<Bf16>(A, st) : launch_dropout<F32>(A, st);
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_dropout launch");
}

}  // extern "C"
