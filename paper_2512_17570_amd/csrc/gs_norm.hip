// gs_norm.hip -- what a layer has around its products: layer norm of rows with its gradient, and dropout onto the residual stream.
//
// All of it is one pass over memory: read once, written once, so HBM is the bound; the arithmetic (ten operations an element, one eighth of
// a Philox block for dropout) goes on beside it.
//   * a row stays in the registers of its team (a wave, four or sixteen) from its first load to its last store; rows that none holds
//     are read again
//   * vectors of 16 bytes at any address the element type allows: the hardware takes them from wherever they lie
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
// Elements [c, c + PER) of an array that has `n`, as far as it has them; 0 for the others.
template <typename E> __device__ __forceinline__ void load_some(const typename E::T *p, int64_t c, int64_t n, float (&z)[E::PER])
{
    if (c + E::PER <= n) {
        E::widen(load_vector<E>(p + c), z);
    } else {
#pragma unroll
        for (int i = 0; i < E::PER; ++i) z[i] = c + i < n ? E::load(p + c + i) : 0.0f;
    }
}
template <typename E> __device__ __forceinline__ void store_some(typename E::T *p, int64_t c, int64_t n, const float (&z)[E::PER])
{
    if (c + E::PER <= n) {
        *reinterpret_cast<typename Loose<sizeof(typename E::T)>::T *>(p + c) = E::narrow(z);
    } else {
#pragma unroll
        for (int i = 0; i < E::PER; ++i)
            if (c + i < n) E::store(p + c + i, z[i]);
    }
}
// PER values of the scale or the shift, in a type of their own
template <typename W, int PER> __device__ __forceinline__ void load_weights(const void *w, int64_t c, int64_t n, float none, float (&z)[PER])
{
    const typename W::T *p = static_cast<const typename W::T *>(w);
    if (!p) {
#pragma unroll
        for (int i = 0; i < PER; ++i) z[i] = none;
    } else if (PER % W::PER == 0 && c + PER <= n) {
        constexpr int N = PER / W::PER ? PER / W::PER : 1;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            float f[W::PER];
            W::widen(load_vector<W>(p + c + q * W::PER), f);
#pragma unroll
            for (int i = 0; i < W::PER; ++i) z[q * W::PER + i] = f[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) z[i] = c + i < n ? W::load(p + c + i) : 0.0f;
    }
}

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

// ---- forward -------------------------------------------------------------------------------------
struct NormArgs {
    const void *x;
    int64_t rows, cols, stride;
    const void *gamma, *beta;
    float eps;
    void *y;
    int64_t y_stride;
    float *stats;
};
// A row a team, NV vectors a lane; HELD: they hold the row, else it is read three times.
template <typename E, typename W, int TEAM, int NV, bool HELD>
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
    float z[NV][PER], sum[1] = {0.0f};
    const int64_t by = (int64_t)TEAM * PER;
    if constexpr (HELD) {
#pragma unroll
        for (int v = 0; v < NV; ++v) load_some<E>(x, v * by + lane * PER, n, z[v]);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < PER; ++i) sum[0] += z[v][i];
    } else {
        for (int64_t c = lane * PER; c < n; c += by) {
            load_some<E>(x, c, n, z[0]);
#pragma unroll
            for (int i = 0; i < PER; ++i) sum[0] += z[0][i];
        }
    }
    team_sums<TEAM>(sum, lds[0]);
    const float mean = sum[0] / (float)n;
    sum[0] = 0.0f;
    if constexpr (HELD) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                z[v][i] -= mean;
                if (v * by + lane * PER + i < n) sum[0] += z[v][i] * z[v][i];
            }
    } else {
        for (int64_t c = lane * PER; c < n; c += by) {
            load_some<E>(x, c, n, z[0]);
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (c + i < n) sum[0] += (z[0][i] - mean) * (z[0][i] - mean);
        }
    }
    team_sums<TEAM>(sum, lds[1]);
    const float rstd = 1.0f / sqrtf(sum[0] / (float)n + A.eps);
    if (A.stats && lane == 0) A.stats[2 * row] = mean, A.stats[2 * row + 1] = rstd;
    auto write = [&](int64_t c, float (&d)[PER]) {
        float g[PER], b[PER];
        load_weights<W, PER>(A.gamma, c, n, 1.0f, g);
        load_weights<W, PER>(A.beta, c, n, 0.0f, b);
#pragma unroll
        for (int i = 0; i < PER; ++i) d[i] = d[i] * rstd * g[i] + b[i];
        store_some<E>(y, c, n, d);
    };
    if constexpr (HELD) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (v * by + lane * PER < n) write(v * by + lane * PER, z[v]);
    } else {
        for (int64_t c = lane * PER; c < n; c += by) {
            load_some<E>(x, c, n, z[0]);
#pragma unroll
            for (int i = 0; i < PER; ++i) z[0][i] -= mean;
            write(c, z[0]);
        }
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
};
// Rows dealt in turn to the workgroups' teams, which add up dy xhat and dy of their own rows for each column; a workgroup's teams join theirs in LDS.
template <typename E, typename W, int TEAM, int NV>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void k_norm_grad(NormGradArgs A)
{
    constexpr int BLOCK = TEAM < 256 ? 256 : TEAM, TEAMS = BLOCK / TEAM, PER = E::PER, NW = TEAM / 64;
    __shared__ float lds[2][2 * NW];
    __shared__ float joint[TEAMS > 1 ? TEAMS * TEAM * NV * PER : 1];
    const int team = TEAMS > 1 ? threadIdx.x / TEAM : 0, lane = TEAMS > 1 ? threadIdx.x % TEAM : threadIdx.x;
    const int64_t n = A.cols, by = (int64_t)TEAM * PER;
    float gamma[NV][PER], dgamma[NV][PER], dbeta[NV][PER];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        load_weights<W, PER>(A.gamma, v * by + lane * PER, n, 1.0f, gamma[v]);
#pragma unroll
        for (int i = 0; i < PER; ++i) dgamma[v][i] = dbeta[v][i] = 0.0f;
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < A.rows; row += (int64_t)gridDim.x * TEAMS, turn ^= 1) {
        const typename E::T *x = static_cast<const typename E::T *>(A.x) + row * A.stride;
        const typename E::T *dy = static_cast<const typename E::T *>(A.dy) + row * A.dy_stride;
        typename E::T *dx = static_cast<typename E::T *>(A.dx) + row * A.dx_stride;
        const float mean = A.stats[2 * row], rstd = A.stats[2 * row + 1];
        float z[NV][PER], d[NV][PER], sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            load_some<E>(x, v * by + lane * PER, n, z[v]);
            load_some<E>(dy, v * by + lane * PER, n, d[v]);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                z[v][i] = (z[v][i] - mean) * rstd;                 // behind the row d is 0
                dgamma[v][i] += d[v][i] * z[v][i];
                dbeta[v][i] += d[v][i];
                d[v][i] *= gamma[v][i];
                sum[0] += d[v][i];
                sum[1] += d[v][i] * z[v][i];
            }
        team_sums<TEAM>(sum, lds[turn]);
        const float a = sum[0] / (float)n, b = sum[1] / (float)n;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int i = 0; i < PER; ++i) d[v][i] = rstd * (d[v][i] - a - z[v][i] * b);
            if (v * by + lane * PER < n) store_some<E>(dx, v * by + lane * PER, n, d[v]);
        }
    }
    if (!A.partials) return;
    float *out = A.partials + (int64_t)blockIdx.x * 2 * n;
#pragma unroll
    for (int q = 0; q < 2; ++q, out += n) {
        if constexpr (TEAMS == 1) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (v * by + lane * PER + i < n) out[v * by + lane * PER + i] = q ? dbeta[v][i] : dgamma[v][i];
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
// Rows that no team holds: dx from two readings, a row a workgroup;
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
    for (int64_t c = threadIdx.x * PER; c < n; c += 1024 * PER) {
        load_some<E>(x, c, n, z);
        load_some<E>(dy, c, n, d);
        load_weights<W, PER>(A.gamma, c, n, 1.0f, g);
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
        load_some<E>(x, c, n, z);
        load_some<E>(dy, c, n, d);
        load_weights<W, PER>(A.gamma, c, n, 1.0f, g);
#pragma unroll
        for (int i = 0; i < PER; ++i) d[i] = rstd * (d[i] * g[i] - a - (z[i] - mean) * rstd * b);
        store_some<E>(dx, c, n, d);
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
        load_some<E>(static_cast<const typename E::T *>(A.x) + row * A.stride, c, n, z);
        load_some<E>(static_cast<const typename E::T *>(A.dy) + row * A.dy_stride, c, n, d);
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
// Sums over the workgroups: a lane a column of one of the two, 16 waves that each take a share; joined in 64 bits.
template <typename W>
__global__ __launch_bounds__(1024) void k_norm_fold(const float *partials, int parts, int64_t cols, void *dgamma, void *dbeta)
{
    __shared__ double part[16][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    double s = 0.0;
    if (c < 2 * cols)
        for (int i = wave; i < parts; i += 16) s += (double)partials[(int64_t)i * 2 * cols + c];
    part[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= 2 * cols) return;
    s = 0.0;
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
    uint64_t offset, blocks;      // blocks of 8 elements by their numbers, the first and last perhaps in part
    uint32_t least;               // T
    float scale;                  // 1 / (1 - P)
    uint32_t k0, k1;
    const uint64_t *step;
};
constexpr int DROP_BLOCK = 256;
// Eight elements a lane: one block of the generator.
template <typename E, bool RESIDUAL>
__global__ __launch_bounds__(DROP_BLOCK) void k_dropout(DropoutArgs A)
{
    constexpr int V = 8 / E::PER;
    const uint64_t b = (uint64_t)blockIdx.x * DROP_BLOCK + threadIdx.x;
    if (b >= A.blocks) return;
    const uint64_t number = (A.offset >> 3) + b;
    const int64_t at = (int64_t)(b * 8) - (int64_t)(A.offset & 7);       // of its first element, which may lie before the array
    const typename E::T *x = static_cast<const typename E::T *>(A.x), *res = static_cast<const typename E::T *>(A.residual);
    typename E::T *out = static_cast<typename E::T *>(A.out);
    const bool whole = at >= 0 && at + 8 <= A.n;
    float z[V][E::PER], r[V][E::PER];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (whole) {
            E::widen(load_vector<E>(x + at + v * E::PER), z[v]);
            if (RESIDUAL) E::widen(load_vector<E>(res + at + v * E::PER), r[v]);
        } else {
#pragma unroll
            for (int i = 0; i < E::PER; ++i) {
                const int64_t e = at + v * E::PER + i;
                const bool there = e >= 0 && e < A.n;
                z[v][i] = there ? E::load(x + e) : 0.0f;
                r[v][i] = RESIDUAL && there ? E::load(res + e) : 0.0f;
            }
        }
    }
    const uint64_t step = A.step ? *A.step : 0;
    uint32_t c[4] = {(uint32_t)number, (uint32_t)(number >> 32), (uint32_t)step, (uint32_t)(step >> 32)};
    philox(c, A.k0, A.k1);
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int i = 0; i < E::PER; ++i) {
            const int e = v * E::PER + i;
            const uint32_t bits = e & 1 ? c[e >> 1] >> 16 : c[e >> 1] & 0xffffu;
            z[v][i] = bits >= A.least ? z[v][i] * A.scale : 0.0f;
            if (RESIDUAL) z[v][i] += r[v][i];
        }
        if (whole) {
            *reinterpret_cast<typename Loose<sizeof(typename E::T)>::T *>(out + at + v * E::PER) = E::narrow(z[v]);
        } else {
#pragma unroll
            for (int i = 0; i < E::PER; ++i) {
                const int64_t e = at + v * E::PER + i;
                if (e >= 0 && e < A.n) E::store(out + e, z[v][i]);
            }
        }
    }
}

// ---- launches ------------------------------------------------------------------------------------
constexpr int64_t kMaxItems = 0xffffffffLL;      // HIP launches fewer than 2^32 work items at a time
constexpr int NORM_PARTS = 512;                  // workgroups of a gradient, and partials of its columns

template <typename E, typename W, int TEAM, int NV, bool HELD>
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
        k_norm<E, W, TEAM, NV, HELD><<<(uint32_t)((B.rows + TEAMS - 1) / TEAMS), BLOCK, 0, stream>>>(B);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename E, typename W>
static hipError_t launch_norm(const NormArgs &A, hipStream_t stream)
{
    const int64_t v = (A.cols + E::PER - 1) / E::PER;
    if (v <= 64) return launch_norm_as<E, W, 64, 1, true>(A, stream);
    if (v <= 128) return launch_norm_as<E, W, 64, 2, true>(A, stream);
    if (v <= 256) return launch_norm_as<E, W, 64, 4, true>(A, stream);
    if (v <= 512) return launch_norm_as<E, W, 256, 2, true>(A, stream);
    if (v <= 1024) return launch_norm_as<E, W, 256, 4, true>(A, stream);
    if (v <= 2048) return launch_norm_as<E, W, 1024, 2, true>(A, stream);
    if (v <= 4096) return launch_norm_as<E, W, 1024, 4, true>(A, stream);
    return launch_norm_as<E, W, 1024, 1, false>(A, stream);
}

// Workgroups of a gradient over rows that are held: all that fit the chip at once, two a CU.
template <typename E, typename W, int TEAM, int NV>
static hipError_t launch_norm_grad_as(const NormGradArgs &A, int &parts, hipStream_t stream)
{
    constexpr int BLOCK = TEAM < 256 ? 256 : TEAM, TEAMS = BLOCK / TEAM;
    parts = (int)std::min<int64_t>(NORM_PARTS, (A.rows + TEAMS - 1) / TEAMS);
    k_norm_grad<E, W, TEAM, NV><<<parts, BLOCK, 0, stream>>>(A);
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
    else if (v <= 512) e = launch_norm_grad_as<E, W, 256, 2>(A, parts, stream);
    else if (v <= 1024) e = launch_norm_grad_as<E, W, 256, 4>(A, parts, stream);
    else if (v <= 2048) e = launch_norm_grad_as<E, W, 1024, 2>(A, parts, stream);
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
static hipError_t launch_dropout(const DropoutArgs &A, hipStream_t stream)
{
    const int64_t most = kMaxItems / DROP_BLOCK * DROP_BLOCK;       // blocks of a launch
    DropoutArgs B = A;
    for (uint64_t done = 0; done < A.blocks; done += most) {
        B.blocks = std::min<uint64_t>(most, A.blocks - done);
        const uint32_t grid = (uint32_t)((B.blocks + DROP_BLOCK - 1) / DROP_BLOCK);
        if (A.residual) k_dropout<E, true><<<grid, DROP_BLOCK, 0, stream>>>(B);
        else k_dropout<E, false><<<grid, DROP_BLOCK, 0, stream>>>(B);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        // the next launch's first block begins with the next element
        const int64_t elements = most * 8 - (int64_t)(B.offset & 7);
        B.x = static_cast<const typename E::T *>(B.x) + elements;
        if (B.residual) B.residual = static_cast<const typename E::T *>(B.residual) + elements;
        B.out = static_cast<typename E::T *>(B.out) + elements;
        B.n -= elements;
        B.offset += elements;
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
    const NormArgs A = {x->data, x->rows, x->cols, x->rows > 1 ? x->row_stride : x->cols, gamma, beta, eps, y, x->rows > 1 ? y_stride : x->cols, row_stats};
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
                            gamma, row_stats, dgamma ? static_cast<float *>(d_workspace) : nullptr};
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
    A.blocks = ((offset & 7) + (uint64_t)n + 7) / 8;
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
