// gs_head.hip -- a linear head's token log-probabilities and cross entropy without its logits: z = x W^T + b is made a tile at a
// time in registers, leaves a maximum and a sum of exponentials, and is gone.  The gradient makes it again, a piece of the
// vocabulary at a time, as dz in bf16, which two more products take to the hidden states and to the weights; where z is small (kKeptBytes) a loss leaves it
// in memory instead.
//
// All the work is in products of matrices: 2 N V H operations for the log-probabilities and 8 N V H with the gradient (2 of them to make
// z again), on the matrix cores.  rows x hidden x vocabulary: 8192 x 2048 x 50304 scored in 1.28 to 1.34 ms (1260 to 1315 TFLOP/s), 8192 x 4096 x 131072 with its
// gradients 26.0 to 26.5 ms (1330 to 1350 TFLOP/s), 4095 x 2048 x 50001 with a bias, of whose rows 3075 count, 2.28 to 2.34 ms; with few rows memory is the bound: one of
// 4096 x 131072 scored in 161 us (7.0 TB/s of weights), 64 x 4096 x 32000 with gradients 212 to 222 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "gs_device.h"
#include "gs_internal.h"

#pragma clang fp contract(off)

namespace gs {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896340736f;

// a value that all lanes of a wave have, in scalar registers
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b)
{
    bf16x2 h = {(__bf16)a, (__bf16)b};             // rounded to nearest even, NaN stays NaN
    return __builtin_bit_cast(uint32_t, h);
}

// ---- a tile of a product -----------------------------------------------------------------------
// C[m][n] = sum_k A[m][k] B[n][k] over a tile of BM x BN, WM x WN waves of MI x NI blocks of 16 x 16 each.  The operands come to LDS
// BK of k at a time by loads that go there without passing registers, STAGES of them in turn, one worked on while the others are on their way.
// An operand is either rows of k (ALONG: k is contiguous) or rows of m or n (k is the distance between rows); the second kind is read from
// LDS by the transposing load.
//
// What bounds it is power: the chip holds its clock (1.9 GHz here, of 2.4) to what the matrix cores, LDS and loads draw together, and each adds to
// the time.  16 x 16 x 32 products draw least (alone, of random values, 2160 TFLOP/s; 32 x 32 x 16, whose sums go through the registers twice as
// often, 1900); rows of 128 bytes are whole lines of the caches (64 bytes a row, four stages: 1190 TFLOP/s against 1300 for 8192 x 4096 x 16384, both steps
// together).  Four waves of 128 x 128, which read a third less LDS: level, they wait where eight do not.  Of 8192 x 4096 x 16384 (0.82 ms, 1340 TFLOP/s;
// the library's 8192 x 131072 x 4096 1490) the products alone take 0.53 ms, with the reads 0.65, with the loads but not the reads 0.65.
constexpr int BK = 64, PART = 32, PARTS = BK / PART;
template <int BM_, int BN_, int WM_, int WN_, int STAGES_> struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WAVES = WM * WN, BLOCK = WAVES * 64, STAGES = STAGES_;
    static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;
    static constexpr int STAGE = (BM + BN) * BK * 2, LDS = STAGES * STAGE;
};
// One operand: `rows` rows (of m or n, or of k), `cols` elements each that may be read, a multiple of 8 and aligned to 16 bytes; stride < 2^23.
struct Operand {
    const uint16_t *p;
    int64_t stride;
    int64_t rows, cols;
};

// 16 bytes a lane from base + offset to LDS (from `lds` + AT on), one lane's behind another's.  By hand because the compiler holds every transposing read back until all loads on
// their way to LDS have come; nothing is returned in registers, and who reads waits for vmcnt and a barrier.  m0 is none of the registers that the compiler has values in, and
// it takes no note of it as written (it is reserved): it would have it for uses of its own, of which these kernels have none (a test looks).
template <int AT>
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base), "n"(AT) : "memory", "scc");
}

// ALONG: LDS has W rows of 128 bytes, whose eight 16-byte chunks are exchanged by the row's bits 1 to 3, so that 16 lanes that read a chunk
// of 16 rows find each bank once.  Else BK rows (k) of 2 W bytes, whose 32-byte slots are exchanged by the row's bits 0, 1 and 3 for the
// same reason.  Positions beyond the operand's rows or columns read its last ones; what comes of those is not used, or meets zeros.  Rows of k may end
// within the last step if ENDS is set.
template <int W, int WAVES, int FRAGS, bool ALONG, bool ENDS> struct Side {
    static constexpr int LOADS = W / 8 / WAVES;
    static_assert(LOADS >= 1 && W * BK * 2 == LOADS * WAVES * 1024, "whole loads of each wave");
    static_assert((FRAGS & (FRAGS - 1)) == 0 && (ALONG || W >= 128), "blocks are told apart by bits of an address");
    const char *next;                     // of the tile, in the step that is loaded next
    int64_t step_by;                      // bytes from a step to the next
    uint32_t at[LOADS], beyond[LOADS];    // bytes from the base; of them, what the last step's rows of k lie behind the operand's last one
    uint32_t frag;                        // of the wave's first block in a stage
    uint32_t place;                       // in the stage of this wave's first load

    static __device__ __forceinline__ int slot(int row) { return 2 * (row & 3) | ((row >> 3) & 1); }
    __device__ __forceinline__ void start(const Operand &X, int64_t first, int64_t k0, int steps, int wave, int lane, int sub)
    {
        place = (uint32_t)(wave * LOADS * 1024);
        step_by = 2 * (ALONG ? BK : BK * X.stride);
        next = reinterpret_cast<const char *>(uniform(reinterpret_cast<int64_t>(X.p + (ALONG ? first * X.stride + k0 : k0 * X.stride + first))));
        const uint32_t stride = (uint32_t)X.stride * 2;
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
            const int i = wave * LOADS + q;
            if constexpr (ALONG) {
                const int row = i * 8 + (lane >> 3), most = (int)min(X.rows - 1 - first, (int64_t)W);
                at[q] = (uint32_t)min(row, most) * stride + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
            } else {
                constexpr int LANES = W / 8, PER = 64 / LANES;        // lanes a row, rows a load
                const int row = i * PER + lane / LANES, p = lane % LANES, most = (int)min(X.cols - 8 - first, (int64_t)W);
                at[q] = (uint32_t)row * stride + min((((p >> 1) ^ slot(row)) << 4) + (p & 1) * 8, most) * 2;
                if constexpr (ENDS) beyond[q] = (uint32_t)max(row - (int)min(X.rows - 1 - k0 - (int64_t)(steps - 1) * BK, (int64_t)BK), 0) * stride;
            }
        }
        if constexpr (ALONG) {
            frag = (uint32_t)((sub * FRAGS * 16 + (lane & 15)) * 128 + (((lane >> 4) ^ ((lane >> 1) & 7)) << 4));
        } else {
            const int row = 8 * (lane >> 4) + ((lane & 15) >> 2);
            frag = (uint32_t)(row * (2 * W) + (((sub * FRAGS) ^ slot(row)) << 5) + (lane & 3) * 8);
        }
    }
    template <int Q> __device__ __forceinline__ void load(uint32_t stage, bool end) const
    {
        uint32_t offset = at[Q];
        if constexpr (ENDS) offset -= end ? beyond[Q] : 0;
        load_to_lds<Q * 1024>(next, offset, stage + place);
    }
    // block f's operand of part s of a stage
    __device__ __forceinline__ bf16x8 read(uint32_t stage, int s, int f) const
    {
        typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
        if constexpr (ALONG) {
            return *reinterpret_cast<lds_bf16x8 *>((uintptr_t)((stage + frag) ^ (s << 6)) + f * 2048);
        } else {
            const uint32_t p = ((stage + frag) ^ (f << 5)) + s * (PART * 2 * W);
            union {
                i16x4 h[2];
                bf16x8 v;
            } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_i16x4 *>((uintptr_t)p));
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_i16x4 *>((uintptr_t)(p + 4 * 2 * W)));
            return u.v;
        }
    }
};

// all loads of this wave but the last N have come, and every LDS read is back
template <int N> __device__ __forceinline__ void wait_loads()
{
    static_assert(N < 64, "what the counter holds");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }

// f(0) ... f(N - 1), each a constant of its own
template <int N, typename F> __device__ __forceinline__ void each(F f)
{
    if constexpr (N > 0) {
        each<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// acc = the tile's product over `steps` steps of BK from k0 on.  Every access lies in the operands, whatever `steps` is: loads ahead of the end
// repeat the last step's.  At the end every wave has passed a barrier and no load is on its way, so the LDS can be used again.
//
// A step is two parts of 32 of k.  While a part is multiplied, the next one is read from LDS: the last part's reads are of the next stage, and before
// them lies the step's one barrier, at which that stage has come and every wave has read all of its own, whose place the stage STAGES steps
// ahead then takes.
template <typename T, bool A_ALONG, bool B_ALONG, bool A_ENDS>
__device__ __forceinline__ void product(const Operand &A, const Operand &B, int64_t m0, int64_t n0, int64_t k0, int steps, char *lds,
                                        f32x4 (&acc)[T::MI][T::NI])
{
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    Side<T::BM, T::WAVES, T::MI, A_ALONG, A_ENDS> a;
    Side<T::BN, T::WAVES, T::NI, B_ALONG, false> b;
    a.start(A, m0, k0, steps, wave, lane, wave / T::WN);
    b.start(B, n0, k0, steps, wave, lane, wave % T::WN);
    constexpr int A_LOADS = decltype(a)::LOADS, L = A_LOADS + decltype(b)::LOADS, MN = T::MI * T::NI;
#pragma unroll
    for (int i = 0; i < T::MI; ++i)
#pragma unroll
        for (int j = 0; j < T::NI; ++j) acc[i][j] = f32x4{};
    if (steps <= 0) return;
    const int end = steps - 1;
    // What the wave's loads and reads go by is kept from step to step in scalar registers, a few additions each: between two products there is room for
    // three other instructions.
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds), lds_last = lds0 + (T::STAGES - 1) * T::STAGE;
    auto behind = [&](uint32_t stage) { return stage == lds_last ? lds0 : stage + (uint32_t)T::STAGE; };
    int loading = 0;                       // the step that is loaded, and the stage that it takes
    uint32_t to = lds0;
    auto load = [&](auto q) {
        if constexpr (q < A_LOADS) a.template load<q>(to, loading >= end);
        else b.template load<q - A_LOADS>(to + T::BM * BK * 2, loading >= end);
        if constexpr (q == L - 1) {
            if (loading < end) a.next += a.step_by, b.next += b.step_by;
            ++loading;
            to = behind(to);
        }
    };
    bf16x8 fa[T::MI], fb[2][T::NI];
    uint32_t from = lds0;                  // the stage that is read
    auto read_a = [&](int s, int i) { fa[i] = a.read(from, s, i); };
    auto read_b = [&](int s, int j) { fb[s & 1][j] = b.read(from + T::BM * BK * 2, s, j); };
    // A part's products, with a read or a load behind some, so that none of them keeps the matrix cores waiting: a row of blocks' operand is read again as
    // soon as its last product has begun.  Loads begin behind the barrier and end half a step later.  The order is held as it stands here.
    constexpr int BAR = T::NI;                              // products of the last part in front of the barrier
    constexpr int EACH = MN * PARTS / 2 / L, FIRST = (MN - BAR) / EACH < L ? (MN - BAR) / EACH : L;      // products to a load; loads in the last part
    static_assert(EACH >= 1 && BAR + T::NI <= MN, "a place for each load and read");
    auto part = [&](auto part_of) {
        constexpr int s = part_of, next = s == PARTS - 1 ? 0 : s + 1;
        constexpr bool last = s == PARTS - 1;
        each<MN>([&](auto p) {
            if constexpr (last && p == BAR) {
                wait_loads<(T::STAGES - 2) * L>();
                barrier();
                from = behind(from);
            }
            constexpr int i = p / T::NI, j = p % T::NI;
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb[s & 1][j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (j == 0 && i > 0) read_a(next, i - 1);
            if constexpr (p == MN - 1) read_a(next, i);
            if constexpr (p >= BAR && p - BAR < T::NI) read_b(next, p - BAR);
            if constexpr (last) {
                if constexpr (p >= BAR && (p - BAR) % EACH == 0 && (p - BAR) / EACH < FIRST) load(std::integral_constant<int, (p - BAR) / EACH>{});
            } else {
                constexpr int g = s * MN + p;
                if constexpr (g % EACH == 0 && FIRST + g / EACH < L) load(std::integral_constant<int, FIRST + g / EACH>{});
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    };
#pragma unroll
    for (int t = 0; t < T::STAGES - 1; ++t) each<L>([&](auto q) { load(q); });
    wait_loads<(T::STAGES - 2) * L>();
    barrier();
    each<FIRST>([&](auto q) { load(q); });
#pragma unroll
    for (int f = 0; f < T::NI; ++f) read_b(0, f);
#pragma unroll
    for (int f = 0; f < T::MI; ++f) read_a(0, f);
    for (int t = 0; t < steps; ++t) each<PARTS>([&](auto s) { part(s); });
    wait_loads<0>();
    barrier();
}
// where element r of a wave's block lies: row of m, column of n
__device__ __forceinline__ int row_of(int r, int lane) { return 4 * (lane >> 4) + r; }
__device__ __forceinline__ int column_of(int lane) { return lane & 15; }

// Tiles in groups along the first dimension, dealt so that each of the 8 dies has neighbours: its 32 CUs work on about 4 x 8 tiles at a time, whose
// operands its L2 holds.  (8 at a time 1 % behind; where all the work is to write rows of results, 4 are 4 % behind.)  false: no tile.
template <int GROUP>
__host__ __device__ __forceinline__ bool deal(uint32_t id, int64_t tiles1, int64_t tiles2, uint32_t &t1, uint32_t &t2)
{
    // a launch has fewer than 2^32 work items, and so fewer than 2^24 tiles
    const uint32_t second = (uint32_t)tiles2, all = (uint32_t)tiles1 * second, per = (all + 7) / 8, t = (id & 7) * per + (id >> 3);
    if ((id >> 3) >= per || t >= all) return false;
    const uint32_t group = t / (GROUP * second), in = t - group * GROUP * second, left = (uint32_t)tiles1 - group * GROUP, width = left < GROUP ? left : GROUP;
    t1 = group * GROUP + in % width;
    t2 = in / width;
    return true;
}
// Of the rows only the tiles that have some that count, wherever the batch ends: those lie in front, so with the others dealt too whole dies would have nothing to do
// (losses of 8192 x 4096 x 32000 of which a half and a quarter count 3250 and 1987 us against 3952 and 2740).  `rows`: of the packed batch; if one tile has them
// all, nothing of this has to wait for the count.
template <typename T> __host__ __device__ __forceinline__ int64_t live_tiles(int64_t rows, int count) { return rows <= T::BN ? 1 : (count + T::BN - 1) / T::BN; }
// a tile of z: words, rows; and of the sums to the rows: rows, columns of the hidden state
template <typename T> __host__ __device__ __forceinline__ bool tile_of_z(uint32_t id, int64_t words, int64_t rows, int count, uint32_t &tw, uint32_t &tr)
{
    return deal<4>(id, (words + T::BM - 1) / T::BM, live_tiles<T>(rows, count), tw, tr) && count > 0;
}
template <typename T> __host__ __device__ __forceinline__ bool tile_of_rows(uint32_t id, int64_t hidden, int64_t rows, int count, uint32_t &tr, uint32_t &th)
{
    return deal<4>(id, live_tiles<T>(rows, count), (hidden + T::BM - 1) / T::BM, tr, th) && count > 0;
}
// the same in scalar registers
__device__ __forceinline__ int64_t scalar(uint32_t x) { return __builtin_amdgcn_readfirstlane((int)x); }

// A wave's blocks as rows of bf16: `value(i, j, r)` of element (m, n) goes to out[n * stride + m] for n < rows, m < cols, counted from the wave's first.
// A lane has four neighbours of m; through LDS (a place of its wave alone) they become rows of whole lines, 16 bytes a lane.  Any alignment of two.
typedef u32x4 loose_u32x4 __attribute__((aligned(2)));
template <typename T, typename F>
__device__ __forceinline__ void store_rows(char *lds, int wave, int lane, F value, uint16_t *out, int64_t stride, int rows, int cols)
{
    constexpr int WIDTH = T::MI * 32, PITCH = WIDTH + 16, PASS = T::NI < 2 ? 1 : 2, CHUNKS = WIDTH / 16, AT_ONCE = 64 / CHUNKS;      // bytes of a row; blocks of n a time
    static_assert(T::WAVES * PASS * 16 * PITCH <= T::LDS && T::NI % PASS == 0 && AT_ONCE * CHUNKS == 64, "");
    char *mine = lds + wave * (PASS * 16 * PITCH);
#pragma unroll
    for (int j0 = 0; j0 < T::NI; j0 += PASS) {
#pragma unroll
        for (int j = 0; j < PASS; ++j)
#pragma unroll
            for (int i = 0; i < T::MI; ++i)
                *reinterpret_cast<u32x2 *>(mine + (j * 16 + column_of(lane)) * PITCH + (i * 16 + row_of(0, lane)) * 2) =
                    u32x2{two_bf16(value(i, j0 + j, 0), value(i, j0 + j, 1)), two_bf16(value(i, j0 + j, 2), value(i, j0 + j, 3))};
        asm volatile("" ::: "memory");
#pragma unroll
        for (int q = 0; q < PASS * 16; q += AT_ONCE) {        // a wave's own accesses to LDS stay in order
            const int n = q + lane / CHUNKS, m = lane % CHUNKS * 8, row = j0 * 16 + n;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(mine + n * PITCH + m * 2);
            if (row >= rows || m >= cols) continue;
            uint16_t *to = out + row * stride + m;
            if (m + 8 <= cols) {
                *reinterpret_cast<loose_u32x4 *>(to) = v;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (m + e < cols) to[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
            }
        }
        asm volatile("" ::: "memory");
    }
}

// ---- the kernels -------------------------------------------------------------------------------
// Rows that count, one after another: the rows with a token (and a factor other than 0).
struct Live {
    int32_t *count;
    int32_t *index;        // the batch's row that is the j-th to count
    int32_t *place;        // of a row of the batch among those; -1: it does not count
    int32_t *token;        // of the j-th
};
constexpr int LIVE_BLOCK = 1024;
// Rows that do not count get logp 0 and statistics (0, 1) here, where there are any to write.
__global__ __launch_bounds__(LIVE_BLOCK) void k_head_live(const int64_t *targets, const float *factor, int rows, int vocab, Live L, float *logp, float *row_stats)
{
    __shared__ int waves[LIVE_BLOCK / 64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < rows; base += LIVE_BLOCK) {
        const int r = base + threadIdx.x;
        bool live = false;
        int64_t t = -1;
        if (r < rows) {
            t = targets[r];
            live = t >= 0 && t < vocab && (!factor || factor[r] != 0.0f);
            if (!live && logp) logp[r] = 0.0f;
            if (!live && row_stats) row_stats[2 * r] = 0.0f, row_stats[2 * r + 1] = 1.0f;
        }
        const uint64_t mask = __ballot(live);
        if (lane == 0) waves[wave] = __popcll(mask);
        __syncthreads();
        int at = before, sum = 0;
        for (int w = 0; w < LIVE_BLOCK / 64; ++w) {
            if (w < wave) at += waves[w];
            sum += waves[w];
        }
        at += __popcll(mask & ((1ull << lane) - 1));
        if (live) L.index[at] = r, L.token[at] = (int32_t)t;
        if (r < rows) L.place[r] = live ? at : -1;
        before += sum;
        __syncthreads();
    }
    if (threadIdx.x == 0) *L.count = before;
}

// Elements of a row, and zeros up to `width` (a multiple of 8); `there`: whether there is such a row.
template <bool WIDE>
__device__ __forceinline__ void copy_row(const uint16_t *f, int64_t cols, bool there, uint16_t *to, int64_t width)
{
    u32x4 *t = reinterpret_cast<u32x4 *>(to);
    for (int64_t c = threadIdx.x; c < width / 8; c += 256) {
        u32x4 q = {};
        if (there) {
            if (WIDE && c * 8 + 8 <= cols) {
                q = *reinterpret_cast<const u32x4 *>(f + c * 8);
            } else {
                uint32_t e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = c * 8 + i < cols ? f[c * 8 + i] : 0;
                q = u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
            }
        }
        t[c] = q;
    }
}
// Row j of `to` (stride `width`, a multiple of 8): row index[j] of `from` (row j without an index), zeros behind its `cols` elements and in rows from count on.
template <bool WIDE>
__global__ __launch_bounds__(256) void k_head_pack(const uint16_t *from, int64_t stride, int64_t cols, const Live L, int64_t rows, uint16_t *to, int64_t width)
{
    const int64_t j = blockIdx.x;
    const bool there = L.count ? j < *L.count : j < rows;
    copy_row<WIDE>(from + (there ? (L.index ? (int64_t)L.index[j] : j) : 0) * stride, cols, there, to + j * width, width);
}
// Both for up to GATHER_MAX rows, in one launch: every workgroup counts the rows that count by itself, which is less than another launch takes (5 us,
// where the two take 4 and 7 for 512 rows; counting 8192 rows takes one workgroup 12 us, beside a product of 1.4 ms).
constexpr int GATHER_MAX = 1024;
template <bool WIDE>
__global__ __launch_bounds__(256) void k_head_gather(const int64_t *targets, const float *factor, int rows, int vocab, Live L, float *logp, float *row_stats,
                                                     const uint16_t *from, int64_t stride, int64_t cols, uint16_t *to, int64_t width)
{
    __shared__ int waves[4], found;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, j = blockIdx.x;
    constexpr int EACH = GATHER_MAX / 256;
    uint64_t masks[EACH];
    int before = 0;
    if (threadIdx.x == 0) found = -1;
    // wave w has rows [256 w, 256 w + 256), 64 at a time
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
        const int r = wave * (64 * EACH) + q * 64 + lane;
        bool live = false;
        if (r < rows) {
            const int64_t t = targets[r];
            live = t >= 0 && t < vocab && (!factor || factor[r] != 0.0f);
        }
        masks[q] = __ballot(live);
        before += __popcll(masks[q]);
    }
    if (lane == 0) waves[wave] = before;
    __syncthreads();
    int at = 0, count = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) at += waves[w];
        count += waves[w];
    }
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
        const int r = wave * (64 * EACH) + q * 64 + lane, mine = at + __popcll(masks[q] & ((1ull << lane) - 1));
        const bool live = masks[q] >> lane & 1;
        if (live && mine == j) found = r;
        if (j == 0 && r < rows) {
            if (live) L.index[mine] = r, L.token[mine] = (int32_t)targets[r];
            L.place[r] = live ? mine : -1;
            if (!live && logp) logp[r] = 0.0f;
            if (!live && row_stats) row_stats[2 * r] = 0.0f, row_stats[2 * r + 1] = 1.0f;
        }
        at += __popcll(masks[q]);
    }
    if (j == 0 && threadIdx.x == 0) *L.count = count;
    __syncthreads();
    copy_row<WIDE>(from + (int64_t)max(found, 0) * stride, cols, found >= 0, to + j * width, width);
}

// What the tiles of z leave, or take.  Columns of a tile (n) are rows of the batch, its rows (m) are words.
struct Logit {
    const uint16_t *bias;
    Live live;
    int64_t rows;             // of the packed batch
    int64_t word0, words;     // this piece of the vocabulary; tiles' words are counted from word0
    int64_t vocab;
    float k;                  // log2(e) / temperature
    float2 *partials;         // [tile of words][rows]: maximum, sum
    float *target_logit;      // [rows]
    float *z;                 // null, or [rows][z_stride], this piece's: z is kept, in 32 bits
    const float4 *row;        // [rows]: M, 1 / S, the gradient's factor over `unit`, unit
    uint16_t *dz;             // [rows][stride]
    int64_t stride, z_stride;
};

// Words of a lane's elements, counted from its wave's first one on; `before` are of the first element of a block.
__device__ __forceinline__ int words_before(int lane) { return row_of(0, lane); }
__device__ __forceinline__ constexpr int word_of(int i, int r) { return i * 16 + r; }

template <typename T>
__device__ __forceinline__ void add_bias(const Logit &G, int64_t w0, int lane, f32x4 (&acc)[T::MI][T::NI])
{
    if (!G.bias) return;
    const int64_t first = w0 + words_before(lane), last = G.vocab - 1;
#pragma unroll
    for (int i = 0; i < T::MI; ++i) {
        float b[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) b[r] = __uint_as_float((uint32_t)G.bias[min(first + word_of(i, r), last)] << 16);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < T::NI; ++j) acc[i][j][r] += b[r];
        asm volatile("" ::: "memory");        // not all of a wave's biases at once
    }
}
// a lane's words that there are, and the place of a target among them (-1: not here)
__device__ __forceinline__ int words_left(const Logit &G, int64_t w0, int lane)
{
    return (int)min(max(G.vocab - w0 - words_before(lane), (int64_t)0), (int64_t)4096);
}
__device__ __forceinline__ int place_of(int64_t target, int64_t w0, int lane)
{
    const int64_t p = target - w0 - words_before(lane);
    return p >= 0 && p < 4096 ? (int)p : -1;
}
// of the four lanes that have a column's elements
__device__ __forceinline__ float column_max(float x) { x = fmaxf(x, __shfl_xor(x, 16)); return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ float column_sum(float x) { x += __shfl_xor(x, 16); return x + __shfl_xor(x, 32); }
// what exponentials are taken from: of nothing but -inf they sum to 0
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
// (m, s) joined with another maximum and sum
__device__ __forceinline__ void join(float k, float &m, float &s, float2 q)
{
    const float top = fmaxf(m, q.x), base = base_of(top);
    s = s * __builtin_amdgcn_exp2f(k * (m - base)) + q.y * __builtin_amdgcn_exp2f(k * (q.x - base));
    m = top;
}

// Maximum and sum of exponentials of each row of the batch over a tile of words.  8192 x 4096 x 32768 1.60 ms (1380 TFLOP/s);
// 64 x 4096 x 32000 62 us with the weights in the memory-side cache, 90 from HBM.
template <typename T>
__global__ __launch_bounds__(T::BLOCK, 2) void k_head_stats(Operand W, Operand X, int steps, Logit G)
{
    __shared__ __attribute__((aligned(128))) char lds[T::LDS];
    uint32_t id1, id2;
    const int count = *G.live.count;
    if (!tile_of_z<T>(blockIdx.x, G.words, G.rows, count, id1, id2)) return;
    const int64_t tw = scalar(id1), tr = scalar(id2);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / T::WN, wn = wave % T::WN;
    const int64_t w0 = G.word0 + tw * T::BM + wm * T::MI * 16;
    int target[T::NI];                     // on its way during the product
#pragma unroll
    for (int j = 0; j < T::NI; ++j) target[j] = G.live.token[tr * T::BN + (wn * T::NI + j) * 16 + column_of(lane)];
    f32x4 acc[T::MI][T::NI];
    product<T, true, true, false>(W, X, tw * T::BM, tr * T::BN, 0, steps, lds, acc);
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
        asm volatile("" : "+v"(target[j]));          // not looked at before
        target[j] = tr * T::BN + (wn * T::NI + j) * 16 + column_of(lane) < count ? place_of(target[j], w0, lane) : -1;
    }
    add_bias<T>(G, w0, lane, acc);
    const int left = words_left(G, w0, lane);
    float2 *joint = reinterpret_cast<float2 *>(lds);        // [WM][BN]
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
        const int n = (wn * T::NI + j) * 16 + column_of(lane);
        const int64_t row = tr * T::BN + n;
        float m = -INFINITY, z = 0.0f;
        bool here = false;
        if (G.z) {
            float *out = G.z + row * G.z_stride + (w0 - G.word0) + words_before(lane);
#pragma unroll
            for (int i = 0; i < T::MI; ++i) *reinterpret_cast<f32x4 *>(out + word_of(i, 0)) = acc[i][j];
        }
#pragma unroll
        for (int i = 0; i < T::MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (word_of(i, r) >= left) acc[i][j][r] = -INFINITY;
                if (word_of(i, r) == target[j]) z = acc[i][j][r], here = true;
                m = fmaxf(m, acc[i][j][r]);
            }
        if (here) G.target_logit[row] = z;
        m = column_max(m);
        const float base = base_of(m);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < T::MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s += __builtin_amdgcn_exp2f(G.k * (acc[i][j][r] - base));
        s = column_sum(s);
        if (lane < 16) joint[wm * T::BN + n] = float2{m, s};
    }
    __syncthreads();
    for (int n = threadIdx.x; n < T::BN; n += T::BLOCK) {
        float m = joint[n].x, s = joint[n].y;
        for (int q = 1; q < T::WM; ++q) join(G.k, m, s, joint[q * T::BN + n]);
        G.partials[(G.word0 / T::BM + tw) * G.rows + tr * T::BN + n] = float2{m, s};
    }
}

// dz of an element
__device__ __forceinline__ float dz_of(const Logit &G, const float4 &R, float z, bool target)
{
    return R.z * ((target ? 1.0f : 0.0f) - __builtin_amdgcn_exp2f(G.k * (z - R.x)) * R.y);
}
// dz of a tile of words (8192 x 4096 x 32768 1.72 ms), rounded to bf16, since it is an operand of the two products that follow; each of its roundings is
// independent (`unit_of` sees to that) and they meet in sums of thousands: 2e-3 of a gradient's norm, of which its own rounding to bf16 is 1.7e-3. Zeros
// in rows from count on and for words behind the vocabulary, which products that follow meet
template <typename T>
__global__ __launch_bounds__(T::BLOCK, 2) void k_head_dz(Operand W, Operand X, int steps, Logit G)
{
    __shared__ __attribute__((aligned(128))) char lds[T::LDS];
    uint32_t id1, id2;
    const int count = *G.live.count;
    if (!tile_of_z<T>(blockIdx.x, G.words, G.rows, count, id1, id2)) return;
    const int64_t tw = scalar(id1), tr = scalar(id2);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / T::WN, wn = wave % T::WN;
    const int64_t w0 = G.word0 + tw * T::BM + wm * T::MI * 16;
    int targets[T::NI];                    // on their way during the product
    f32x4 rows[T::NI];
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
        const int64_t row = tr * T::BN + (wn * T::NI + j) * 16 + column_of(lane);
        targets[j] = G.live.token[row];
        rows[j] = *reinterpret_cast<const f32x4 *>(G.row + row);
    }
    f32x4 acc[T::MI][T::NI];
    product<T, true, true, false>(W, X, tw * T::BM, tr * T::BN, 0, steps, lds, acc);
    add_bias<T>(G, w0, lane, acc);
    const int left = words_left(G, w0, lane);
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
        const int64_t row = tr * T::BN + (wn * T::NI + j) * 16 + column_of(lane);
        asm volatile("" : "+v"(targets[j]), "+v"(rows[j]));          // not looked at before
        const int words = row < count ? left : 0, target = row < count ? place_of(targets[j], w0, lane) : -1;
        const float4 R = {rows[j][0], rows[j][1], rows[j][2], rows[j][3]};
#pragma unroll
        for (int i = 0; i < T::MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] = word_of(i, r) < words ? dz_of(G, R, acc[i][j][r], word_of(i, r) == target) : 0.0f;
    }
    uint16_t *out = G.dz + (tr * T::BN + wn * T::NI * 16) * G.stride + (w0 - G.word0);
    store_rows<T>(lds, wave, lane, [&](int i, int j, int r) { return acc[i][j][r]; }, out, G.stride, T::NI * 16, T::MI * 16);
}
// loss (+)= sum of weights times -logp over the rows that count, by one workgroup
struct Loss {
    const float *logp, *weights;
    float *loss;              // null: none
    int accumulate;
};
__device__ __forceinline__ void loss_of(const Live &live, const Loss &L)
{
    __shared__ double lds[4];
    const int count = *live.count;
    double s = 0.0;
    for (int j = threadIdx.x; j < count; j += 256) {
        const int r = live.index[j];
        s -= (double)(L.weights ? L.weights[r] : 1.0f) * (double)L.logp[r];
    }
    s = block_sum<256>(s, lds);
    if (threadIdx.x == 0) *L.loss = (float)(s + (L.accumulate ? (double)*L.loss : 0.0));
}
__global__ __launch_bounds__(256) void k_head_loss(Live live, Loss L) { loss_of(live, L); }
// dz from z that was kept: a lane four words; the workgroup behind the rows' has the loss, which is a launch less (64 x 32000 5 us)
__global__ __launch_bounds__(256) void k_head_dz_kept(Logit G, Loss L)
{
    const int64_t row = blockIdx.x, w = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
    if (row >= G.rows) {
        if (blockIdx.y == 0 && L.loss) loss_of(G.live, L);
        return;
    }
    const int count = *G.live.count;
    if (row >= (count + 255) / 256 * 256 || w >= (G.words + 255) / 256 * 256) return;
    float d[4] = {};
    if (row < count) {
        const float4 R = G.row[row];
        const f32x4 z = *reinterpret_cast<const f32x4 *>(G.z + row * G.z_stride + w);
        const int64_t target = G.live.token[row] - G.word0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (w + i < G.words) d[i] = dz_of(G, R, z[i], w + i == target);
    }
    *reinterpret_cast<u32x2 *>(G.dz + row * G.stride + w) = u32x2{two_bf16(d[0], d[1]), two_bf16(d[2], d[3])};
}

// sum[split][row][h] (+)= dz W over a piece of the vocabulary; W is read as it lies, k across its rows (8192 x 4096 x 32768 1.64 ms)
struct ToRows {
    Live live;
    int64_t rows, hidden;
    float *sum;
    int first;                // of the pieces
    int splits, steps;        // steps: of the piece
};
template <typename T>
__device__ __forceinline__ void dx_tile(const Operand &W, const Operand &DZ, const ToRows &G, uint32_t id, int split, char *lds)
{
    uint32_t id1, id2;
    if (!tile_of_rows<T>(id, G.hidden, G.rows, *G.live.count, id1, id2)) return;
    const int64_t tr = scalar(id1), th = scalar(id2);
    const int per = (G.steps + G.splits - 1) / G.splits, from = split * per, mine = G.steps - from < per ? G.steps - from : per;
    f32x4 acc[T::MI][T::NI];
    product<T, false, true, true>(W, DZ, th * T::BM, tr * T::BN, (int64_t)from * BK, mine, lds, acc);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / T::WN, wn = wave % T::WN;
    const int64_t h0 = th * T::BM + wm * T::MI * 16 + row_of(0, lane);
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
        const int64_t row = tr * T::BN + (wn * T::NI + j) * 16 + column_of(lane);
        float *out = G.sum + ((int64_t)split * G.rows + row) * G.hidden;          // hidden: of the sums' rows, a multiple of 4
#pragma unroll
        for (int i = 0; i < T::MI; ++i) {
            const int64_t h = h0 + i * 16;
            if (h >= G.hidden) continue;
            f32x4 *to = reinterpret_cast<f32x4 *>(out + h);
            *to = G.first ? acc[i][j] : *to + acc[i][j];
        }
    }
}
template <typename T>
__global__ __launch_bounds__(T::BLOCK, 2) void k_head_dx(Operand W, Operand DZ, ToRows G)
{
    __shared__ __attribute__((aligned(128))) char lds[T::LDS];
    dx_tile<T>(W, DZ, G, blockIdx.x, (int)blockIdx.y, lds);
}

// dW[word][h] = dz^T x of a piece of the vocabulary; of both k lies across the rows (8192 x 4096 x 32768 1.61 ms, 1360 TFLOP/s)
struct ToWeights {
    Live live;
    int64_t word0, words, hidden;
    uint16_t *dw;
    int64_t stride;
    const float4 *row;
};
template <typename T>
__device__ __forceinline__ void dw_tile(const Operand &X, const Operand &DZ, const ToWeights &G, uint32_t id, char *lds)
{
    uint32_t id1, id2;
    if (!deal<8>(id, (G.words + T::BN - 1) / T::BN, (G.hidden + T::BM - 1) / T::BM, id1, id2)) return;
    const int64_t tw = scalar(id1), th = scalar(id2);
    f32x4 acc[T::MI][T::NI];
    const int count = *G.live.count;
    product<T, false, false, false>(X, DZ, th * T::BM, tw * T::BN, 0, (count + BK - 1) / BK, lds, acc);
    const float unit = count ? G.row[0].w : 1.0f;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / T::WN, wn = wave % T::WN;
    const int64_t w0 = tw * T::BN + wn * T::NI * 16, h0 = th * T::BM + wm * T::MI * 16;
    store_rows<T>(lds, wave, lane, [&](int i, int j, int r) { return acc[i][j][r] * unit; }, G.dw + (G.word0 + w0) * G.stride + h0, G.stride,
                  (int)min(G.words - w0, (int64_t)4096), (int)min(G.hidden - h0, (int64_t)4096));
}
template <typename T>
__global__ __launch_bounds__(T::BLOCK, 2) void k_head_dw(Operand X, Operand DZ, ToWeights G)
{
    __shared__ __attribute__((aligned(128))) char lds[T::LDS];
    dw_tile<T>(X, DZ, G, blockIdx.x, lds);
}
// Both of few rows, in one launch: the sums to the rows read all weights and write little, those to the weights read little and write as much.  The
// first `dx` workgroups (`dx` / splits of each part) have the rows, about one on each CU; the others come and go beside them.  Losses, us, against
// two launches: 64 x 4096 x 32000 212/221, 128 x 4096 x 50304 361/384, 120 x 2048 x 8192 65/77, 70 x 512 x 1152 31/36, 1 x 4864 x 7680 93/102, 300 x
// 8192 x 10000 290/285.  With up to 512 workgroups for the rows the first two take 222 and 373, with the rows' dealt evenly between the others 233
// and 429.  Large tiles leave no room on a CU for another workgroup.
template <typename TX, typename TW>
__global__ __launch_bounds__(TX::BLOCK, 2) void k_head_dx_dw(Operand W, Operand X, Operand DZ, ToRows R, ToWeights G, uint32_t dx)
{
    static_assert(TX::BLOCK == TW::BLOCK, "one launch");
    __shared__ __attribute__((aligned(128))) char lds[TX::LDS > TW::LDS ? TX::LDS : TW::LDS];
    if (blockIdx.x < dx) {
        const uint32_t per = dx / (uint32_t)R.splits, split = blockIdx.x / per;
        dx_tile<TX>(W, DZ, R, blockIdx.x - split * per, (int)split, lds);
    } else {
        dw_tile<TW>(X, DZ, G, blockIdx.x - dx, lds);
    }
}

// db[word] = sum over rows of dz, of the same one in bf16 that dW takes (db is dW of a state that is 1 in every row): a lane two words, a wave a share of the rows; dz is read
// once more (3075 rows that count x 50001 59 us, 5.2 TB/s)
__global__ __launch_bounds__(1024) void k_head_db(const uint16_t *dz, int64_t dz_stride, Live live, int64_t words, const float4 *row, uint16_t *db)
{
    __shared__ float part[16][128];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 128 + lane * 2;           // a piece's rows have whole tiles of words
    const int count = *live.count;
    float a = 0.0f, b = 0.0f;
#pragma unroll 8
    for (int r = wave; r < count; r += 16) {
        const uint32_t q = *reinterpret_cast<const uint32_t *>(dz + (int64_t)r * dz_stride + w);
        a += bf16_lo(q);
        b += bf16_hi(q);
    }
    part[wave][2 * lane] = a;
    part[wave][2 * lane + 1] = b;
    __syncthreads();
    if (threadIdx.x < 128) {
        float s = 0.0f;
        for (int i = 0; i < 16; ++i) s += part[i][threadIdx.x];
        const int64_t at = (int64_t)blockIdx.x * 128 + threadIdx.x;
        if (at < words) db[at] = (uint16_t)f32_to_bf16_bits(count ? s * row[0].w : 0.0f);
    }
}

// What of the rows' factors dz does without: a value in [1, 2), the first one's significand, which the sums are multiplied by at the end.  A mean over
// tokens gives all rows one factor, and dz of a target is nearly that: divided by it, it is a power of two and loses nothing in bf16, where else
// all of them would be rounded the same way (gradients off by up to 2^-8 of themselves, all in one direction).  Divided by its own significand a
// factor is a power of two exactly.
__device__ __forceinline__ float unit_of(float factor)
{
    const uint32_t u = __float_as_uint(factor) & 0x7fffffffu;
    return u >= 0x00800000u && u < 0x7f800000u ? __uint_as_float((u & 0x007fffffu) | 0x3f800000u) : 1.0f;
}
// Rows' maxima and sums, joined over the tiles of words: R rows a workgroup, 256 / R lanes a row.
struct Join {
    const float2 *partials;
    const float *target_logit;
    int64_t tiles, rows;       // rows: of the packed batch, or of the batch without a list of those that count
    float k, it;
    float *logp, *row_stats;   // of the batch
    const float *weights;      // of the rows, or null for ones: factors of a loss's gradient are -weights / temperature
    float4 *row;               // null: no gradient follows
    Live live;
    const int64_t *targets;    // without such a list
    int vocab;
};
template <int R>
__global__ __launch_bounds__(256) void k_head_join(Join J)
{
    constexpr int LANES = 256 / R;
    __shared__ float2 part[LANES][R];
    const int n = threadIdx.x % R, slice = threadIdx.x / R;
    const int64_t j = (int64_t)blockIdx.x * R + n;
    const int64_t count = J.live.count ? *J.live.count : J.rows;
    if ((int64_t)blockIdx.x * R >= count) return;
    float m = -INFINITY, s = 0.0f;
#pragma unroll 4
    for (int64_t t = slice; t < J.tiles; t += LANES) join(J.k, m, s, J.partials[t * J.rows + j]);
    part[slice][n] = float2{m, s};
#pragma unroll
    for (int h = LANES / 2; h; h /= 2) {
        __syncthreads();
        if (slice < h) {
            join(J.k, m, s, part[slice + h][n]);
            part[slice][n] = float2{m, s};
        }
    }
    if (slice != 0 || j >= count) return;
    int64_t r = j;
    if (J.live.count) {
        r = J.live.index[j];
    } else if (const int64_t t = J.targets[j]; t < 0 || t >= J.vocab) {
        J.logp[r] = 0.0f;
        if (J.row_stats) J.row_stats[2 * r] = 0.0f, J.row_stats[2 * r + 1] = 1.0f;
        return;
    }
    J.logp[r] = J.it * (J.target_logit[j] - m) - logf(s);
    if (J.row_stats) J.row_stats[2 * r] = m, J.row_stats[2 * r + 1] = s;
    if (!J.row) return;
    const float unit = unit_of(J.it * (J.weights ? J.weights[J.live.index[0]] : 1.0f));
    J.row[j] = float4{m, 1.0f / s, -J.it * (J.weights ? J.weights[r] : 1.0f) / unit, unit};
}
// rows' data for a gradient from statistics that the caller has
__global__ __launch_bounds__(256) void k_head_rows(Live live, const float *row_stats, const float *dlogp, float it, float4 *row)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= *live.count) return;
    const int64_t r = live.index[j];
    const float unit = unit_of(it * dlogp[live.index[0]]);
    row[j] = float4{row_stats[2 * r], 1.0f / row_stats[2 * r + 1], it * dlogp[r] / unit, unit};
}

// dx of the rows that count from their sums, zeros in the others: a lane four elements
__global__ __launch_bounds__(256) void k_head_rows_out(Live live, const float *sum, int splits, int64_t rows, int64_t width, int64_t hidden, const float4 *row,
                                                       uint16_t *dx, int64_t stride)
{
    const int64_t r = blockIdx.x, h = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
    if (h >= hidden) return;
    const int64_t j = live.place[r];
    f32x4 s = {};
    if (j >= 0) {
        const float *from = sum + j * width + h;
#pragma unroll 8
        for (int i = 0; i < splits; ++i) s += *reinterpret_cast<const f32x4 *>(from + i * rows * width);
        s *= row[j].w;
    }
    uint16_t *out = dx + r * stride + h;
    const u32x2 q = {two_bf16(s[0], s[1]), two_bf16(s[2], s[3])};
    if (h + 4 <= hidden) {
        typedef u32x2 loose_u32x2 __attribute__((aligned(2)));
        *reinterpret_cast<loose_u32x2 *>(out) = q;
    } else {
        for (int e = 0; e < 4; ++e)
            if (h + e < hidden) out[e] = (uint16_t)(q[e >> 1] >> (16 * (e & 1)));
    }
}

// ---- up to 16 rows, scored -----------------------------------------------------------------------
// Every weight is read once and meets few rows: HBM is the bound, and the weights go from there to registers.  A workgroup takes FEW_WORDS words, its four waves take
// turns along k, 128 at a time; the matrix cores' other columns are idle.  Rows of the batch that there are not repeat the last one.
constexpr int FEW_ROWS = 16, FEW_WORDS = 32, FEW_WAVES = 4, FEW_K = 128;
template <bool VEC>
__device__ __forceinline__ bf16x8 load_k(const uint16_t *p, int64_t k, int64_t n)
{
    if (VEC && k + 8 <= n) return *reinterpret_cast<const bf16x8 *>(p + k);
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = k + i < n ? p[k + i] : 0;
    return __builtin_bit_cast(bf16x8, u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16});
}
struct Few {
    const uint16_t *x, *w, *bias;
    int64_t x_stride, w_stride, hidden, vocab;
    int rows;
    const int64_t *targets;
    float k;
    float2 *partials;          // [workgroup][rows]
    float *target_logit;
};
template <bool VEC>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_head_few(Few G)
{
    constexpr int MI = FEW_WORDS / 16, KI = FEW_K / 32;
    __shared__ f32x4 part[FEW_WAVES - 1][MI][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n = lane & 15;
    const int64_t w0 = (int64_t)blockIdx.x * FEW_WORDS, H = G.hidden;
    const uint16_t *x = G.x + min(n, G.rows - 1) * G.x_stride, *w[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) w[i] = G.w + min(w0 + i * 16 + n, G.vocab - 1) * G.w_stride;
    f32x4 acc[MI] = {};
    auto some = [&](int64_t k0, auto whole) {
        bf16x8 fw[MI][KI], fx[KI];
#pragma unroll
        for (int q = 0; q < KI; ++q) {
            const int64_t k = k0 + q * 32 + (lane >> 4) * 8;
#pragma unroll
            for (int i = 0; i < MI; ++i) fw[i][q] = load_k<VEC>(w[i], k, whole ? k + 8 : H);
            if (VEC && (whole || k + 8 <= H)) fx[q] = *reinterpret_cast<const bf16x8 *>(x + k);
            else fx[q] = load_k<false>(x, k, H);
        }
#pragma unroll
        for (int q = 0; q < KI; ++q)
#pragma unroll
            for (int i = 0; i < MI; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[i][q], fx[q], acc[i], 0, 0, 0);
    };
    int64_t k0 = wave * FEW_K;
    for (; VEC && k0 + FEW_K <= H; k0 += FEW_WAVES * FEW_K) some(k0, std::true_type{});
    for (; k0 < H; k0 += FEW_WAVES * FEW_K) some(k0, std::false_type{});
    if (wave > 0) {
#pragma unroll
        for (int i = 0; i < MI; ++i) part[wave - 1][i][lane] = acc[i];
    }
    __syncthreads();
    if (wave > 0) return;
    const int64_t left = G.vocab - w0 - row_of(0, lane), target = n < G.rows ? G.targets[n] - w0 - row_of(0, lane) : -1;
    float m = -INFINITY, s = 0.0f;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
#pragma unroll
        for (int q = 0; q < FEW_WAVES - 1; ++q) acc[i] += part[q][i][lane];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (G.bias) acc[i][r] += __uint_as_float((uint32_t)G.bias[min(w0 + i * 16 + row_of(r, lane), G.vocab - 1)] << 16);
            if (i * 16 + r >= left) acc[i][r] = -INFINITY;
            if (i * 16 + r == target) G.target_logit[n] = acc[i][r];
            m = fmaxf(m, acc[i][r]);
        }
    }
    m = column_max(m);
    const float base = base_of(m);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) s += __builtin_amdgcn_exp2f(G.k * (acc[i][r] - base));
    s = column_sum(s);
    if (lane < G.rows && lane < 16) G.partials[(int64_t)blockIdx.x * G.rows + lane] = float2{m, s};
}

// The sum of a wave, in all its lanes.
template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ float add_dpp32(float x)
{
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum32(float x)
{
    x = add_dpp32<0xb1>(x);
    x = add_dpp32<0x4e>(x);
    x = add_dpp32<0x141>(x);
    x = add_dpp32<0x140>(x);
    x = add_dpp32<0x142, 0xa>(x);
    x = add_dpp32<0x143, 0xc>(x);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
// Up to R <= 4 rows: a wave's lanes lie along k, so that each load is whole lines of one word's weights, where the matrix cores' operand is 64 bytes of each of 16
// words; products of pairs are added up in 32 bits.  SPLIT waves share a word, each with NC parts of 512 of k, for which it keeps the rows in
// registers: as few as those allow, since the sum over a wave's lanes costs as much as 900 products.
constexpr int DOT_ROWS = 4, DOT_K = 512, DOT_HIDDEN = FEW_WAVES * DOT_K * 4;
template <int R, int NC, int SPLIT>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_head_dot(Few G)
{
    constexpr int WORDS = FEW_WORDS * SPLIT / FEW_WAVES, AT_ONCE = 16 / NC < WORDS ? 16 / NC : WORDS;        // words of a wave: all, on their way at a time
    static_assert(WORDS % AT_ONCE == 0 && R <= 2 * FEW_WAVES, "");
    __shared__ float part[SPLIT][R][FEW_WORDS];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, share = wave % SPLIT, first = wave / SPLIT * WORDS;
    const int64_t w0 = (int64_t)blockIdx.x * FEW_WORDS;
    const int k0 = share * DOT_K + lane * 8;
    u32x4 x[R][NC];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int k = k0 + c * (SPLIT * DOT_K);
            x[r][c] = k < G.hidden ? *reinterpret_cast<const u32x4 *>(G.x + min(r, G.rows - 1) * G.x_stride + k) : u32x4{};
        }
#pragma unroll 1
    for (int b = first; b < first + WORDS; b += AT_ONCE) {
        u32x4 w[AT_ONCE][NC];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const uint16_t *p = G.w + min(w0 + b + i, G.vocab - 1) * G.w_stride;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int k = k0 + c * (SPLIT * DOT_K);
                w[i][c] = k < G.hidden ? __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p + k)) : u32x4{};
            }
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float s = 0.0f;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)w[i][c][e]), __builtin_bit_cast(bf16x2, (uint32_t)x[r][c][e]), s, false);
                s = wave_sum32(s);
                if (lane == 0) part[share][r][b + i] = s;
            }
    }
    __syncthreads();
    const int n = lane / FEW_WORDS + 2 * wave, w = lane % FEW_WORDS;        // half a wave a row
    if (n >= G.rows) return;
    float z = part[0][n][w];
#pragma unroll
    for (int q = 1; q < SPLIT; ++q) z += part[q][n][w];
    if (G.bias) z += __uint_as_float((uint32_t)G.bias[min(w0 + w, G.vocab - 1)] << 16);
    if (w0 + w >= G.vocab) z = -INFINITY;
    if (w0 + w == G.targets[n]) G.target_logit[n] = z;
    float m = z;
#pragma unroll
    for (int h = 16; h; h /= 2) m = fmaxf(m, __shfl_xor(m, h));
    float s = __builtin_amdgcn_exp2f(G.k * (z - base_of(m)));
#pragma unroll
    for (int h = 16; h; h /= 2) s += __shfl_xor(s, h);
    if (w == 0) G.partials[(int64_t)blockIdx.x * G.rows + n] = float2{m, s};
}

// ---- the plan of a call ------------------------------------------------------------------------
// Many rows; up to 128, or too few for the others; up to 64, where the weights' way from memory is all the time there is.  Scoring, us, hidden x
// vocabulary 4096 x 131072, 2048 x 50304, 4096 x 32000, 8192 x 32000, 1024 x 32000: Mid of 128 rows 201/66/79/153/31, with a third stage, which leaves a
// CU one workgroup of it fewer, 215/72/69/136/28, and of 256 rows (the last four) 98/97/175/37 against 108/105/190/42; Slim 187/57/67/129/24, with six
// stages 195/64/67/129/25, of 256 words 186/62/87/170/32.
typedef Tile<256, 256, 2, 4, 2> Big;
typedef Tile<128, 128, 2, 2, 2> Mid;
typedef Tile<128, 64, 4, 1, 3> Slim;
typedef Tile<64, 64, 2, 2, 3> Tiny;           // up to 64 rows and so few words that those would leave CUs without work

constexpr int64_t kMaxRows = 1 << 20, kMaxHidden = 1 << 17, kMaxVocab = 1 << 30;
constexpr int64_t kPieceBytes = 512 << 20;          // of dz: 8192 x 4096 x 131072 25.9 ms, with 256 MB 26.1, 128 MB 26.0, 64 MB 27.1; 4095 x 2048 x 50001 2.33, 2.43, 2.69, 2.82
// Of z, in 32 bits: what a call may take beside dz.  A bound on memory, not where time turns; a loss in us, kept and made again: 64 x 4096 x 32000 222/243, 1000 x 2048 x 32000
// 446/500, 1024 x 4096 x 131072 3013/3641, and of more, with a limit of 1 GiB, 2600 x 2048 x 50304 1742/1990, 4095 x 2048 x 50001 2430/2777, 8192 x 512 x 32000 1255/1198.
constexpr int64_t kKeptBytes = 512 << 20;
static_assert(kKeptBytes <= 2 * kPieceBytes, "of a batch whose z is kept, dz is one piece");
// Of the hidden state from which z is kept, us kept and made again: 1354 x 320 x 39296 355/324; of 512 few rows gain, 500 x 50304 195/206, 128 rows of 1024 x 50304
// 107/119, and many lose, 4000 x 512 x 32000 673/635.
constexpr int64_t kKeptWidth = 512;
constexpr int64_t kPackedBytes = 128 << 20;         // of weights that cannot be read where they lie
// Large tiles up to which a product is done in small ones, four times as many, all of which run at once, two on each of the 256 CUs.  Scored, us, large
// against small: 256 rows of 4096 x 32000 (125 tiles) 117/99, of 2048 x 50304 (197) 79/96, 200 of 4096 x 50304 (197) 133/172, 512 of 4096 x 32000 (250)
// 126/184.  To the weights, a loss: 1024 x 4096 x 8192 (512) 252/253, 4096 x 2048 x 50304 2772/3038.
constexpr int64_t MID_TILES = 128;
// The same up to 64 rows: 64 x 4096 x 16000 (125 tiles of 128 words) scored in 48 us against 40, 64 x 4096 x 8000 29/25, 1 x 4864 x 7680 a loss of 93/83; 32 x 4096 x 24000 (188) 54/57,
// 64 x 4096 x 32000 (250) level.
constexpr int64_t TINY_WORDS = MID_TILES * Slim::BM;

struct Plan {
    int64_t rows;            // of the packed batch
    int64_t width;           // of its rows, of packed weights and of sums to the rows
    int64_t piece;           // words
    int64_t packed;          // words of a piece where weights have to be packed
    int64_t tiles;           // of 256 words
    int64_t joined;          // maxima and sums of a row
    int splits;              // of the sums to the rows
    int words, side;         // of a tile: words (or hidden columns), rows
    int dx, dw;              // rows of the tiles of the sums to the rows, words of those to the weights
    bool kept;
    size_t index, x, partials, target, row, z, dz, sum, w, all;      // places in the workspace, and its size
};
static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
// A call without a gradient; with one, from the caller's statistics; with one behind a forward pass of its own, which is what can keep z.
enum Work { SCORES, GRADIENT, LOSS };
// Packed weights are reckoned with in any case: their alignment is not known when the size is asked for.
static Plan plan_of(int64_t rows, int64_t hidden, int64_t vocab, Work work)
{
    const bool gradient = work != SCORES;
    Plan P = {};
    P.side = rows <= Slim::BN ? Slim::BN : rows <= Mid::BN || up(rows, Big::BN) / Big::BN * (up(vocab, Big::BM) / Big::BM) <= MID_TILES ? Mid::BN : Big::BN;
    P.words = P.side == Big::BN ? Big::BM : P.side == Slim::BN && vocab <= TINY_WORDS ? Tiny::BM : Slim::BM;
    P.rows = up(std::max<int64_t>(rows, 1), P.side);
    P.width = up(hidden, 64);
    P.tiles = up(vocab, 256) / 256;
    P.joined = up(vocab, P.words) / P.words;
    const int64_t most = std::max<int64_t>(1, kPieceBytes / (2 * P.rows * 256));
    P.kept = work == LOSS && P.width >= kKeptWidth && P.rows * P.tiles * 256 * 4 <= kKeptBytes;
    P.piece = std::min(P.tiles, most) * 256;              // all of them where z is kept
    P.packed = std::min(P.piece, std::max<int64_t>(1, kPackedBytes / (2 * P.width * 256)) * 256);
    // Tiles of 256 columns of the hidden state where it has more than 128 (loss of 4096 x 320 x 32000 544 us, of 128 columns 548; 640 814 and 841, 896
    // 919 and 1027).
    const bool wide = hidden > 128;
    P.dx = P.side == Slim::BN ? Slim::BN : wide && P.side == Big::BN ? Big::BN : Mid::BN;
    P.dw = wide && up(hidden, Big::BM) / Big::BM * (up(std::min(P.piece, vocab), Big::BN) / Big::BN) > MID_TILES ? Big::BN : Mid::BN;
    // The sums to the rows in parts of k that fill the chip: the fewest of those whose tiles take least, a step each and 24 for what a tile has to do
    // besides (a loss of 1000 x 2048 x 32000 450 us, in one part 938; 4096 x 2048 x 50304 2772 and 3145).
    const int64_t out = P.rows / P.dx * (up(hidden, P.dx == Big::BN ? Big::BM : Slim::BM) / (P.dx == Big::BN ? Big::BM : Slim::BM)), at_once = 256;
    const int64_t steps = up(std::min(P.piece, vocab), BK) / BK;
    int64_t least = INT64_MAX;
    for (int s = 1; s <= 32 && s * 4 <= std::max<int64_t>(steps, 4); ++s) {
        const int64_t time = up(out * s, at_once) / at_once * ((steps + s - 1) / s + 24);
        if (time * 20 < least * 19 || s == 1) least = time, P.splits = s;
    }
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += (size_t)up(bytes, 256);
        return here;
    };
    P.index = take((3 * P.rows + 64) * 4);
    P.x = take(P.rows * P.width * 2);
    P.partials = take(std::max(P.joined * P.rows, rows <= FEW_ROWS ? up(vocab, FEW_WORDS) / FEW_WORDS * FEW_ROWS : 0) * 8);
    P.target = take(P.rows * 4);
    P.row = take(P.rows * 16);
    P.dz = gradient ? take(P.rows * P.piece * 2) : at;
    P.sum = gradient ? take(P.splits * P.rows * P.width * 4) : at;
    P.w = take(P.packed * P.width * 2);
    P.z = P.kept ? take(P.rows * P.tiles * 256 * 4) : at;
    P.all = at;
    return P;
}

struct Call {
    gs_head h;
    Plan P;
    char *ws;
    const int64_t *targets;
    float it;
    Live live;
    hipStream_t stream;
    bool packed;             // the weights cannot be read where they lie
    uint16_t *x() const { return reinterpret_cast<uint16_t *>(ws + P.x); }
    uint16_t *w() const { return reinterpret_cast<uint16_t *>(ws + P.w); }
    uint16_t *dz() const { return reinterpret_cast<uint16_t *>(ws + P.dz); }
    float *sum() const { return reinterpret_cast<float *>(ws + P.sum); }
    float2 *partials() const { return reinterpret_cast<float2 *>(ws + P.partials); }
    float *target() const { return reinterpret_cast<float *>(ws + P.target); }
    float4 *row() const { return reinterpret_cast<float4 *>(ws + P.row); }
};

static bool multiple16(const void *p, int64_t stride) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(stride * 2)) & 15) == 0; }

static Call call_of(const gs_head &h, const int64_t *targets, float temperature, Work work, void *ws, void *stream)
{
    Call C = {};
    C.h = h;
    if (h.rows <= 1) C.h.x_stride = h.hidden;
    if (h.vocab <= 1) C.h.w_stride = h.hidden;
    C.P = plan_of(h.rows, h.hidden, h.vocab, work);
    C.ws = static_cast<char *>(ws);
    C.targets = targets;
    C.it = 1.0f / temperature;
    int32_t *index = reinterpret_cast<int32_t *>(C.ws + C.P.index);
    C.live = {index, index + 64, index + 64 + C.P.rows, index + 64 + 2 * C.P.rows};
    C.stream = static_cast<hipStream_t>(stream);
    C.packed = h.hidden % 64 != 0 || !multiple16(h.w, C.h.w_stride) || C.h.w_stride >= 1 << 23;
    return C;
}

static hipError_t pack(const Call &C, const uint16_t *from, int64_t stride, const Live &live, int64_t there, int64_t rows, uint16_t *to)
{
    if (multiple16(from, stride)) k_head_pack<true><<<(uint32_t)rows, 256, 0, C.stream>>>(from, stride, C.h.hidden, live, there, to, C.P.width);
    else k_head_pack<false><<<(uint32_t)rows, 256, 0, C.stream>>>(from, stride, C.h.hidden, live, there, to, C.P.width);
    return hipGetLastError();
}
// the rows that count, packed
static hipError_t pack_rows(const Call &C, const float *factor, float *logp, float *row_stats)
{
    const gs_head &h = C.h;
    if (C.P.rows <= GATHER_MAX) {
        auto *kernel = multiple16(h.x, h.x_stride) ? k_head_gather<true> : k_head_gather<false>;
        kernel<<<(uint32_t)C.P.rows, 256, 0, C.stream>>>(C.targets, factor, (int)h.rows, (int)h.vocab, C.live, logp, row_stats, h.x, h.x_stride, h.hidden, C.x(), C.P.width);
        return hipGetLastError();
    }
    k_head_live<<<1, LIVE_BLOCK, 0, C.stream>>>(C.targets, factor, (int)h.rows, (int)h.vocab, C.live, logp, row_stats);
    return pack(C, h.x, h.x_stride, C.live, C.P.rows, C.P.rows, C.x());
}
static Logit logit_of(const Call &C, int64_t word0, int64_t words)
{
    Logit G = {};
    G.bias = C.h.bias;
    G.live = C.live;
    G.rows = C.P.rows;
    G.word0 = word0;
    G.words = words;
    G.vocab = C.h.vocab;
    G.k = kLog2e * C.it;
    G.partials = C.partials();
    G.target_logit = C.target();
    G.z = C.P.kept ? reinterpret_cast<float *>(C.ws + C.P.z) + word0 : nullptr;
    G.z_stride = C.P.tiles * 256;
    G.row = C.row();
    G.dz = C.dz();
    G.stride = C.P.piece;
    return G;
}
static uint32_t grid_of(int64_t tiles) { return (uint32_t)(up(tiles, 8)); }

// each(first word, words, their weights) of every piece; have_w: weights packed as one piece are there already; reads_w: whether weights are read at all
template <typename F> static hipError_t pieces(const Call &C, bool have_w, bool reads_w, F each)
{
    const bool packed = C.packed && reads_w;
    const int64_t piece = packed ? C.P.packed : C.P.piece;
    for (int64_t w = 0; w < C.h.vocab; w += piece) {
        const int64_t words = std::min(piece, C.h.vocab - w);
        Operand W = {C.h.w + w * C.h.w_stride, C.h.w_stride, words, C.h.hidden};
        if (packed) {
            if (!(have_w && piece >= C.h.vocab))
                if (hipError_t e = pack(C, W.p, W.stride, Live{}, words, words, C.w()); e != hipSuccess) return e;
            W = {C.w(), C.P.width, words, C.P.width};
        }
        if (hipError_t e = each(w, words, W); e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
static hipError_t forward(const Call &C, float *logp, float *row_stats, const float *row_weights, bool gradient)
{
    const Operand X = {C.x(), C.P.width, C.P.rows, C.P.width};
    hipError_t e = pieces(C, false, true, [&](int64_t w, int64_t words, const Operand &W) {
        k_head_stats<T><<<grid_of(up(words, T::BM) / T::BM * (C.P.rows / T::BN)), T::BLOCK, 0, C.stream>>>(W, X, (int)(C.P.width / BK), logit_of(C, w, words));
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    const Join J = {C.partials(), C.target(), C.P.joined, C.P.rows, kLog2e * C.it, C.it, logp, row_stats, row_weights, gradient ? C.row() : nullptr, C.live, nullptr, 0};
    if (C.P.side < Big::BN) k_head_join<1><<<(uint32_t)C.P.rows, 256, 0, C.stream>>>(J);
    else k_head_join<32><<<(uint32_t)(C.P.rows / 32), 256, 0, C.stream>>>(J);
    return hipGetLastError();
}
static hipError_t forward(const Call &C, float *logp, float *row_stats, const float *row_weights, bool gradient)
{
    return (C.P.words == Tiny::BM ? forward<Tiny> : C.P.side == Slim::BN ? forward<Slim> : C.P.side == Mid::BN ? forward<Mid> : forward<Big>)(C, logp, row_stats, row_weights, gradient);
}
template <int R> static void launch_dot(const Few &G, uint32_t grid, hipStream_t stream)
{
    if (G.hidden <= DOT_K) k_head_dot<R, 1, 1><<<grid, FEW_WAVES * 64, 0, stream>>>(G);
    else if (G.hidden <= 2 * DOT_K) k_head_dot<R, 2, 1><<<grid, FEW_WAVES * 64, 0, stream>>>(G);
    else if (G.hidden <= 4 * DOT_K) k_head_dot<R, 4, 1><<<grid, FEW_WAVES * 64, 0, stream>>>(G);
    else if (G.hidden <= 8 * DOT_K) k_head_dot<R, 4, 2><<<grid, FEW_WAVES * 64, 0, stream>>>(G);
    else k_head_dot<R, 4, 4><<<grid, FEW_WAVES * 64, 0, stream>>>(G);
}
static void launch_dot(const Few &G, uint32_t grid, hipStream_t stream)
{
    if (G.rows == 1) launch_dot<1>(G, grid, stream);
    else launch_dot<DOT_ROWS>(G, grid, stream);
}
// Rows that are scored without LDS: up to 4 in any case, up to 16 while the weights are few (us, against tiles, 16 rows: 2^25 values 21/24, 2^27 57/57, 2^28 123/129,
// 2^29 267/187: half lines, but more workgroups).
static bool few_rows(int64_t rows, int64_t hidden, int64_t vocab)
{
    if (vocab > (int64_t)1 << 28) return false;            // of whose workgroups a launch does not take as many
    return rows <= DOT_ROWS || (rows <= FEW_ROWS && hidden * vocab <= (int64_t)1 << 28);
}
static hipError_t forward_few(const Call &C, float *logp, float *row_stats)
{
    const gs_head &h = C.h;
    const Few G = {h.x, h.w, h.bias, h.x_stride, h.w_stride, h.hidden, h.vocab, (int)h.rows, C.targets, kLog2e * C.it, C.partials(), C.target()};
    const int64_t tiles = up(h.vocab, FEW_WORDS) / FEW_WORDS;
    const bool whole = multiple16(h.x, h.x_stride) && multiple16(h.w, h.w_stride);
    if (whole && h.hidden % 8 == 0 && h.hidden <= DOT_HIDDEN && h.rows <= DOT_ROWS) launch_dot(G, (uint32_t)tiles, C.stream);
    else if (whole) k_head_few<true><<<(uint32_t)tiles, FEW_WAVES * 64, 0, C.stream>>>(G);
    else k_head_few<false><<<(uint32_t)tiles, FEW_WAVES * 64, 0, C.stream>>>(G);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const Join J = {C.partials(), C.target(), tiles, h.rows, kLog2e * C.it, C.it, logp, row_stats, nullptr, nullptr, Live{}, C.targets, (int)h.vocab};
    k_head_join<1><<<(uint32_t)h.rows, 256, 0, C.stream>>>(J);
    return hipGetLastError();
}

template <typename T> static void launch_dx(const Call &C, const Operand &W, const Operand &DZ, const ToRows &R)
{
    k_head_dx<T><<<dim3(grid_of(C.P.rows / T::BN * (up(C.P.width, T::BM) / T::BM)), (uint32_t)C.P.splits), T::BLOCK, 0, C.stream>>>(W, DZ, R);
}
template <typename T> static void launch_dw(const Call &C, const Operand &X, const Operand &DZ, const ToWeights &R)
{
    k_head_dw<T><<<grid_of(up(R.words, T::BN) / T::BN * (up(R.hidden, T::BM) / T::BM)), T::BLOCK, 0, C.stream>>>(X, DZ, R);
}
template <typename T> static void launch_dx_dw(const Call &C, const Operand &W, const Operand &X, const Operand &DZ, const ToRows &R, const ToWeights &G)
{
    const uint32_t dx = grid_of(C.P.rows / T::BN * (up(C.P.width, T::BM) / T::BM)) * (uint32_t)C.P.splits;
    k_head_dx_dw<T, Mid><<<dx + grid_of(up(G.words, Mid::BN) / Mid::BN * (up(G.hidden, Mid::BM) / Mid::BM)), T::BLOCK, 0, C.stream>>>(W, X, DZ, R, G, dx);
}
template <typename T> static void launch_dz(const Call &C, const Operand &W, const Operand &X, const Logit &G)
{
    k_head_dz<T><<<grid_of(up(G.words, T::BM) / T::BM * (C.P.rows / T::BN)), T::BLOCK, 0, C.stream>>>(W, X, (int)(C.P.width / BK), G);
}
// after_forward: z, if it is kept, and weights packed as one piece are there from the forward pass, whose loss is still to be summed
static hipError_t backward(const Call &C, const gs_head_grads &D, bool after_forward, const Loss &loss)
{
    const Plan &P = C.P;
    const bool have_z = after_forward && P.kept;
    if (loss.loss && !have_z) k_head_loss<<<1, 256, 0, C.stream>>>(C.live, loss);
    const Operand X = {C.x(), P.width, P.rows, P.width};
    hipError_t e = pieces(C, after_forward, !have_z || D.dx, [&](int64_t w, int64_t words, const Operand &W) {
        const Logit G = logit_of(C, w, words);
        if (have_z) k_head_dz_kept<<<dim3((uint32_t)P.rows + 1, (uint32_t)((words + 1023) / 1024)), 256, 0, C.stream>>>(G, w == 0 ? loss : Loss{});
        else (P.words == Tiny::BM ? launch_dz<Tiny> : P.side == Slim::BN ? launch_dz<Slim> : P.side == Mid::BN ? launch_dz<Mid> : launch_dz<Big>)(C, W, X, G);
        const Operand DZ = {C.dz(), P.piece, P.rows, P.piece};
        const ToRows R = {C.live, P.rows, P.width, C.sum(), w == 0, P.splits, (int)(up(words, BK) / BK)};
        const ToWeights E = {C.live, w, words, C.h.hidden, D.dw, C.h.vocab > 1 ? D.dw_stride : C.h.hidden, C.row()};
        if (D.dx && D.dw && P.side < Big::BN) {
            (P.dx == Slim::BN ? launch_dx_dw<Slim> : launch_dx_dw<Mid>)(C, W, X, DZ, R, E);
        } else if (D.dx) {
            (P.dx == Slim::BN ? launch_dx<Slim> : P.dx == Mid::BN ? launch_dx<Mid> : launch_dx<Big>)(C, W, DZ, R);
        }
        if (D.dw && !(D.dx && P.side < Big::BN)) (P.dw == Mid::BN ? launch_dw<Mid> : launch_dw<Big>)(C, X, DZ, E);
        if (D.dbias) k_head_db<<<(uint32_t)((words + 127) / 128), 1024, 0, C.stream>>>(C.dz(), P.piece, C.live, words, C.row(), D.dbias + w);
        return hipGetLastError();
    });
    if (e != hipSuccess || !D.dx || !C.h.rows) return e;
    k_head_rows_out<<<dim3((uint32_t)C.h.rows, (uint32_t)((C.h.hidden + 1023) / 1024)), 256, 0, C.stream>>>(C.live, C.sum(), P.splits, P.rows, P.width, C.h.hidden, C.row(), D.dx,
                                                                                                          C.h.rows > 1 ? D.dx_stride : C.h.hidden);
    return hipGetLastError();
}

// ---- checks -------------------------------------------------------------------------------------
static bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static bool good(const void *p, uintptr_t to) { return p && aligned(p, to); }
// bytes from a matrix's first element to behind its last one; -1 if they do not fit an address
static int64_t extent(int64_t rows, int64_t cols, int64_t stride)
{
    int64_t n;
    if (rows <= 1) return rows * cols * 2;
    if (__builtin_mul_overflow(rows - 1, stride, &n) || __builtin_add_overflow(n, cols, &n) || __builtin_mul_overflow(n, (int64_t)2, &n)) return -1;
    return n;
}
static bool good_rows(const void *p, int64_t rows, int64_t cols, int64_t stride)
{
    return good(p, 2) && (rows <= 1 || stride >= cols) && extent(rows, cols, stride) >= 0;
}
static bool good_sizes(int64_t rows, int64_t hidden, int64_t vocab)
{
    return rows >= 0 && rows <= kMaxRows && hidden >= 1 && hidden <= kMaxHidden && vocab >= 1 && vocab <= kMaxVocab;
}
static bool good_head(const gs_head *h)
{
    if (!h || !good_sizes(h->rows, h->hidden, h->vocab)) return false;
    if (!good_rows(h->w, h->vocab, h->hidden, h->w_stride) || !aligned(h->bias, 2)) return false;
    return h->rows == 0 || good_rows(h->x, h->rows, h->hidden, h->x_stride);
}
static bool good_grads(const gs_head &h, const gs_head_grads *D)
{
    if (!D) return false;
    if (D->dx && h.rows && !good_rows(D->dx, h.rows, h.hidden, D->dx_stride)) return false;
    if (D->dw && !good_rows(D->dw, h.vocab, h.hidden, D->dw_stride)) return false;
    return aligned(D->dbias, 2);
}
static bool good_temperature(float t) { return t >= 1e-4f && t <= 1e4f; }

struct Ranges {
    Range r[16];
    int n = 0;
    void add(const void *p, int64_t bytes, bool out) { r[n++] = range_of(p, bytes, out); }
    void add(const gs_head &h)
    {
        add(h.x, extent(h.rows, h.hidden, h.x_stride), false);
        add(h.w, extent(h.vocab, h.hidden, h.w_stride), false);
        add(h.bias, h.vocab * 2, false);
    }
    void add(const gs_head &h, const gs_head_grads &D)
    {
        add(D.dx, extent(h.rows, h.hidden, D.dx_stride), true);
        add(D.dw, extent(h.vocab, h.hidden, D.dw_stride), true);
        add(D.dbias, h.vocab * 2, true);
    }
    bool apart() const
    {
        for (int i = 0; i < n; ++i)
            for (int j = i + 1; j < n; ++j)
                if ((r[i].out || r[j].out) && overlap(r[i], r[j])) return false;
        return true;
    }
};

}  // namespace gs

using namespace gs;

extern "C" {

size_t gs_head_workspace_bytes(int64_t rows, int64_t hidden, int64_t vocab, int gradient)
{
    if (!good_sizes(rows, hidden, vocab)) return 0;
    return plan_of(rows, hidden, vocab, gradient ? LOSS : SCORES).all;
}

size_t gs_head_logp_grad_workspace_bytes(int64_t rows, int64_t hidden, int64_t vocab)
{
    if (!good_sizes(rows, hidden, vocab)) return 0;
    return plan_of(rows, hidden, vocab, GRADIENT).all;
}

gs_status gs_head_logp(const gs_head *head, const int64_t *targets, float temperature, float *logp, float *row_stats, void *d_workspace,
                       size_t workspace_bytes, void *stream)
{
    if (!good_head(head) || !good_temperature(temperature)) return GS_ERR_INVALID_ARG;
    const int64_t rows = head->rows;
    if (rows && (!good(targets, 8) || !good(logp, 4) || !aligned(row_stats, 4))) return GS_ERR_INVALID_ARG;
    if (!good(d_workspace, 256) || workspace_bytes < gs_head_workspace_bytes(rows, head->hidden, head->vocab, 0)) return GS_ERR_WORKSPACE;
    if (rows == 0) return GS_OK;
    Ranges R;
    R.add(*head);
    R.add(targets, rows * 8, false);
    R.add(logp, rows * 4, true);
    R.add(row_stats, rows * 8, true);
    R.add(d_workspace, (int64_t)workspace_bytes, true);
    if (!R.apart()) return GS_ERR_INVALID_ARG;
    const Call C = call_of(*head, targets, temperature, SCORES, d_workspace, stream);
    hipError_t e;
    if (few_rows(rows, head->hidden, head->vocab)) {
        e = forward_few(C, logp, row_stats);
    } else {
        e = pack_rows(C, nullptr, logp, row_stats);
        if (e == hipSuccess) e = forward(C, logp, row_stats, nullptr, false);
    }
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_head_logp launch");
}

gs_status gs_head_logp_grad(const gs_head *head, const int64_t *targets, float temperature, const float *row_stats, const float *dlogp,
                            const gs_head_grads *grads, void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!good_head(head) || !good_temperature(temperature) || !good_grads(*head, grads)) return GS_ERR_INVALID_ARG;
    const int64_t rows = head->rows;
    if (rows && (!good(targets, 8) || !good(row_stats, 4) || !good(dlogp, 4))) return GS_ERR_INVALID_ARG;
    if (!good(d_workspace, 256) || workspace_bytes < gs_head_logp_grad_workspace_bytes(rows, head->hidden, head->vocab)) return GS_ERR_WORKSPACE;
    Ranges R;
    R.add(*head);
    R.add(*head, *grads);
    R.add(targets, rows * 8, false);
    R.add(row_stats, rows * 8, false);
    R.add(dlogp, rows * 4, false);
    R.add(d_workspace, (int64_t)workspace_bytes, true);
    if (!R.apart()) return GS_ERR_INVALID_ARG;
    const Call C = call_of(*head, targets, temperature, GRADIENT, d_workspace, stream);
    hipError_t e = pack_rows(C, dlogp, nullptr, nullptr);
    if (e == hipSuccess) {
        k_head_rows<<<(uint32_t)((C.P.rows + 255) / 256), 256, 0, C.stream>>>(C.live, row_stats, dlogp, C.it, C.row());
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = backward(C, *grads, false, Loss{});
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_head_logp_grad launch");
}

gs_status gs_head_cross_entropy(const gs_head *head, const int64_t *targets, const float *weights, float temperature, float *logp,
                                const gs_head_grads *grads, float *d_loss, int accumulate, void *d_workspace, size_t workspace_bytes,
                                void *stream)
{
    if (!good_head(head) || !good_temperature(temperature) || (grads && !good_grads(*head, grads))) return GS_ERR_INVALID_ARG;
    const int64_t rows = head->rows;
    if (rows && (!good(targets, 8) || !aligned(weights, 4) || !good(logp, 4))) return GS_ERR_INVALID_ARG;
    if (!good(d_loss, 4)) return GS_ERR_INVALID_ARG;
    if (!good(d_workspace, 256) || workspace_bytes < gs_head_workspace_bytes(rows, head->hidden, head->vocab, grads != nullptr)) return GS_ERR_WORKSPACE;
    Ranges R;
    R.add(*head);
    if (grads) R.add(*head, *grads);
    R.add(targets, rows * 8, false);
    R.add(weights, rows * 4, false);
    R.add(logp, rows * 4, true);
    R.add(d_loss, 4, true);
    R.add(d_workspace, (int64_t)workspace_bytes, true);
    if (!R.apart()) return GS_ERR_INVALID_ARG;
    const Call C = call_of(*head, targets, temperature, grads ? LOSS : SCORES, d_workspace, stream);
    hipError_t e = pack_rows(C, weights, logp, nullptr);
    if (e == hipSuccess) e = forward(C, logp, nullptr, weights, grads != nullptr);
    const Loss loss = {logp, weights, d_loss, accumulate};
    if (e == hipSuccess && grads) e = backward(C, *grads, true, loss);
    if (e == hipSuccess && !grads) {
        k_head_loss<<<1, 256, 0, C.stream>>>(C.live, loss);
        e = hipGetLastError();
    }
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_head_cross_entropy launch");
}

}  // extern "C"
