// gs_head.hip -- a linear head's token log-probabilities and cross entropy without its logits: z = x W^T + b is made a tile at a
// time in registers, leaves a maximum and a sum of exponentials, and is gone.  The gradient makes it again, a piece of the
// vocabulary at a time, as dz in bf16, which two more products take to the hidden states and to the weights.
//
// All the work is in products of matrices: 2 N V H operations for the log-probabilities and 8 N V H with the gradient (2 of them to make
// z again), on the matrix cores.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

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
// BK of k at a time by loads that go there without passing registers, one stage on its way while another is worked on.
// An operand is either rows of k (ALONG: k is contiguous) or rows of m or n (k is the distance between rows); the second kind is read from
// LDS by the transposing load.
//
// What bounds it is power: the chip holds its clock (1.9 GHz here, of 2.4) to what the matrix cores, LDS and loads draw together, and each adds to
// the time.  16 x 16 x 32 products draw least (alone, of random values, 2160 TFLOP/s; 32 x 32 x 16, whose sums go through the registers twice as
// often, 1900); rows of 128 bytes are whole lines of the caches (64 bytes a row, four stages: 1190 TFLOP/s against 1300 for 8192 x 4096 x 16384, both steps
// together).  Four waves of 128 x 128, which read a third less LDS: level, they wait where eight do not.
constexpr int BK = 64, PART = 32, PARTS = BK / PART, STAGES = 2;
template <int BM_, int BN_, int WM_, int WN_> struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WAVES = WM * WN, BLOCK = WAVES * 64;
    static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;
    static constexpr int STAGE = (BM + BN) * BK * 2;
};
// One operand: `rows` rows (of m or n, or of k), `cols` elements each that may be read, a multiple of 8 and aligned to 16 bytes; stride < 2^23.
struct Operand {
    const uint16_t *p;
    int64_t stride;
    int64_t rows, cols;
};

// 16 bytes a lane from base + offset to LDS, one lane's behind another's.  By hand because the compiler holds every transposing read back until all loads on
// their way to LDS have come; nothing is returned in registers, and who reads waits for vmcnt and a barrier.
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t offset, char *lds)
{
    const uint32_t to = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}

// ALONG: LDS has W rows of 128 bytes, whose eight 16-byte chunks are exchanged by the row's bits 1 to 3, so that 16 lanes that read a chunk
// of 16 rows find each bank once.  Else BK rows (k) of 2 W bytes, whose 32-byte slots are exchanged by the row's bits 0, 1 and 3 for the
// same reason.  Positions beyond the operand's rows or columns read its last ones; what comes of those is not used, or meets zeros.  Rows of k may end
// within the last step if ENDS is set.
template <int W, int WAVES, int FRAGS, bool ALONG, bool ENDS> struct Side {
    static constexpr int LOADS = W / 8 / WAVES;
    static_assert(LOADS >= 1 && W * BK * 2 == LOADS * WAVES * 1024, "whole loads of each wave");
    static_assert((FRAGS & (FRAGS - 1)) == 0 && W >= 128, "blocks are told apart by bits of an address");
    const char *base;                     // of the tile
    int64_t step_by;                      // bytes from a step to the next
    uint32_t at[LOADS], beyond[LOADS];    // bytes from the base; of them, what the last step's rows of k lie behind the operand's last one
    uint32_t frag;                        // of the wave's first block in a stage
    int place;                            // in the stage of this wave's first load

    static __device__ __forceinline__ int slot(int row) { return 2 * (row & 3) | ((row >> 3) & 1); }
    __device__ __forceinline__ void start(const Operand &X, int64_t first, int64_t k0, int steps, int wave, int lane, int sub)
    {
        place = wave * LOADS * 1024;
        step_by = 2 * (ALONG ? BK : BK * X.stride);
        base = reinterpret_cast<const char *>(uniform(reinterpret_cast<int64_t>(X.p + (ALONG ? first * X.stride + k0 : k0 * X.stride + first))));
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
    __device__ __forceinline__ void load(char *stage, int q, int step, bool end) const
    {
        uint32_t offset = at[q];
        if constexpr (ENDS) offset -= end ? beyond[q] : 0;
        load_to_lds(base + step * step_by, offset, stage + place + q * 1024);
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

// every load of this wave has come, and every LDS read is back
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }

// acc = the tile's product over `steps` steps of BK from k0 on.  Every access lies in the operands, whatever `steps` is: loads ahead of the end
// repeat the last step's.  At the end every wave has passed a barrier and no load is on its way, so the LDS can be used again.
//
// A step is two parts of 32 of k.  While a part is multiplied, the next one is read from LDS: the last part's reads are of the next stage, and before
// them lies the step's one barrier, at which that stage has come and every wave has read all of its own, whose place the stage after
// the next one then takes.
template <typename T, bool A_ALONG, bool B_ALONG, bool B_ENDS>
__device__ __forceinline__ void product(const Operand &A, const Operand &B, int64_t m0, int64_t n0, int64_t k0, int steps, char *lds,
                                        f32x4 (&acc)[T::MI][T::NI])
{
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    Side<T::BM, T::WAVES, T::MI, A_ALONG, false> a;
    Side<T::BN, T::WAVES, T::NI, B_ALONG, B_ENDS> b;
    a.start(A, m0, k0, steps, wave, lane, wave / T::WN);
    b.start(B, n0, k0, steps, wave, lane, wave % T::WN);
    constexpr int A_LOADS = decltype(a)::LOADS, L = A_LOADS + decltype(b)::LOADS, MN = T::MI * T::NI;
#pragma unroll
    for (int i = 0; i < T::MI; ++i)
#pragma unroll
        for (int j = 0; j < T::NI; ++j) acc[i][j] = f32x4{};
    if (steps <= 0) return;
    const int end = steps - 1;
    auto load = [&](int t, int q) {
        char *stage = lds + (t & 1) * T::STAGE;
        const int s = t < end ? t : end;
        if (q < A_LOADS) a.load(stage, q, s, s == end);
        else b.load(stage + T::BM * BK * 2, q - A_LOADS, s, s == end);
    };
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds);
    bf16x8 fa[T::MI], fb[2][T::NI];
    auto read_a = [&](int t, int s, int i) { fa[i] = a.read(lds0 + (t & 1) * T::STAGE, s, i); };
    auto read_b = [&](int t, int s, int j) { fb[s & 1][j] = b.read(lds0 + (t & 1) * T::STAGE + T::BM * BK * 2, s, j); };
    // A part's products, with a read or a load behind some, so that none of them keeps the matrix cores waiting: a row of blocks' operand is read again as
    // soon as its last product has begun.  Loads begin behind the barrier and end half a step later.  The order is held as it stands here.
    constexpr int BAR = T::NI;                              // products of the last part in front of the barrier
    constexpr int EACH = MN * PARTS / 2 / L, FIRST = (MN - BAR) / EACH < L ? (MN - BAR) / EACH : L;      // products to a load; loads in the last part
    static_assert(EACH >= 1 && BAR + T::NI <= MN, "a place for each load and read");
    auto part = [&](int t, int s) {
        const bool last = s == PARTS - 1;
        const int tr = last ? t + 1 : t, sr = last ? 0 : s + 1;
#pragma unroll
        for (int p = 0; p < MN; ++p) {
            if (last && p == BAR) {
                wait_loads();
                barrier();
            }
            const int i = p / T::NI, j = p % T::NI;
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb[s & 1][j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (j == 0 && i > 0) read_a(tr, sr, i - 1);
            if (p == MN - 1) read_a(tr, sr, i);
            if (p >= BAR && p - BAR < T::NI) read_b(tr, sr, p - BAR);
            if (last) {
                if (p >= BAR && (p - BAR) % EACH == 0 && (p - BAR) / EACH < FIRST) load(t + 2, (p - BAR) / EACH);
            } else {
                const int g = s * MN + p;
                if (g % EACH == 0 && FIRST + g / EACH < L) load(t + 1, FIRST + g / EACH);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll
    for (int q = 0; q < L; ++q) load(0, q);
    wait_loads();
    barrier();
#pragma unroll
    for (int q = 0; q < FIRST; ++q) load(1, q);
#pragma unroll
    for (int f = 0; f < T::NI; ++f) read_b(0, 0, f);
#pragma unroll
    for (int f = 0; f < T::MI; ++f) read_a(0, 0, f);
    for (int t = 0; t < steps; ++t) {
#pragma unroll
        for (int s = 0; s < PARTS; ++s) part(t, s);
    }
    wait_loads();
    barrier();
}
// where element r of a wave's block lies: row of m, column of n
__device__ __forceinline__ int row_of(int r, int lane) { return 4 * (lane >> 4) + r; }
__device__ __forceinline__ int column_of(int lane) { return lane & 15; }

// Tiles in groups of 8 along the first dimension, dealt so that each of the 8 dies has neighbours: its 32 CUs work on about 8 x 4 tiles at a
// time, whose operands its L2 holds.  false: no tile.
__device__ __forceinline__ bool my_tile(int64_t tiles1, int64_t tiles2, int64_t &t1, int64_t &t2)
{
    // a launch has fewer than 2^32 work items, and so fewer than 2^24 tiles
    const uint32_t second = (uint32_t)tiles2, all = (uint32_t)tiles1 * second, per = (all + 7) / 8, id = blockIdx.x, t = (id & 7) * per + (id >> 3);
    if ((id >> 3) >= per || t >= all) return false;
    const uint32_t group = t / (8 * second), in = t - group * 8 * second, left = (uint32_t)tiles1 - group * 8, width = left < 8 ? left : 8;
    t1 = __builtin_amdgcn_readfirstlane((int)(group * 8 + in % width));
    t2 = __builtin_amdgcn_readfirstlane((int)(in / width));
    return true;
}

// ---- the kernels -------------------------------------------------------------------------------
// Rows that count, one after another: the rows with a token (and a factor other than 0).
struct Live {
    int32_t *index;        // the batch's row that is the j-th to count
    int32_t *count;
};
constexpr int LIVE_BLOCK = 1024;
__global__ __launch_bounds__(LIVE_BLOCK) void k_head_live(const int64_t *targets, const float *factor, int rows, int vocab, Live L)
{
    __shared__ int waves[LIVE_BLOCK / 64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < rows; base += LIVE_BLOCK) {
        const int r = base + threadIdx.x;
        bool live = false;
        if (r < rows) {
            const int64_t t = targets[r];
            live = t >= 0 && t < vocab && (!factor || factor[r] != 0.0f);
        }
        const uint64_t mask = __ballot(live);
        if (lane == 0) waves[wave] = __popcll(mask);
        __syncthreads();
        int at = before, sum = 0;
        for (int w = 0; w < LIVE_BLOCK / 64; ++w) {
            if (w < wave) at += waves[w];
            sum += waves[w];
        }
        if (live) L.index[at + __popcll(mask & ((1ull << lane) - 1))] = r;
        before += sum;
        __syncthreads();
    }
    if (threadIdx.x == 0) *L.count = before;
}

// Row j of `to` (stride `width`, a multiple of 8): row index[j] of `from` (row j without an index), zeros behind its `cols` elements and in rows from count on.
template <bool WIDE>
__global__ __launch_bounds__(256) void k_head_pack(const uint16_t *from, int64_t stride, int64_t cols, const Live L, int64_t rows, uint16_t *to, int64_t width)
{
    const int64_t j = blockIdx.x;
    const bool there = L.count ? j < *L.count : j < rows;
    const uint16_t *f = from + (there ? (L.index ? (int64_t)L.index[j] : j) : 0) * stride;
    u32x4 *t = reinterpret_cast<u32x4 *>(to + j * width);
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

// What the tiles of z leave, or take.  Columns of a tile (n) are rows of the batch, its rows (m) are words.
struct Logit {
    const uint16_t *bias;
    const int64_t *targets;
    Live live;
    int64_t rows;             // of the packed batch
    int64_t word0, words;     // this piece of the vocabulary; tiles' words are counted from word0
    int64_t vocab;
    float k;                  // log2(e) / temperature
    float it;                 // 1 / temperature
    float2 *partials;         // [tile of words][rows]: maximum, sum
    float *target_logit;      // [rows]
    const float4 *row;        // [rows]: M, 1 / S, the gradient's factor over `unit`, unit
    uint16_t *dz;             // [rows][dz_stride]
    int64_t dz_stride;
};

// Words of a lane's elements, counted from its wave's first one on; `before` are of the first element of a block.
__device__ __forceinline__ int words_before(int lane) { return 4 * (lane >> 4); }
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

// Maximum and sum of exponentials of each row of the batch over a tile of words.
template <typename T>
__global__ __launch_bounds__(T::BLOCK, T::BLOCK / 256) void k_head_stats(Operand W, Operand X, int steps, Logit G)
{
    __shared__ __attribute__((aligned(128))) char lds[STAGES * T::STAGE];
    int64_t tw, tr;
    if (!my_tile((G.words + T::BM - 1) / T::BM, G.rows / T::BN, tw, tr)) return;
    const int count = *G.live.count;
    if (tr * T::BN >= count) return;
    f32x4 acc[T::MI][T::NI];
    product<T, true, true, false>(W, X, tw * T::BM, tr * T::BN, 0, steps, lds, acc);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / T::WN, wn = wave % T::WN;
    const int64_t w0 = G.word0 + tw * T::BM + wm * T::MI * 16;
    add_bias<T>(G, w0, lane, acc);
    const int left = words_left(G, w0, lane);
    float2 *joint = reinterpret_cast<float2 *>(lds);        // [WM][BN]
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
        const int n = (wn * T::NI + j) * 16 + column_of(lane);
        const int64_t row = tr * T::BN + n;
        const int target = row < count ? place_of(G.targets[G.live.index[row]], w0, lane) : -1;
        float m = -INFINITY, z = 0.0f;
        bool here = false;
#pragma unroll
        for (int i = 0; i < T::MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (word_of(i, r) >= left) acc[i][j][r] = -INFINITY;
                if (word_of(i, r) == target) z = acc[i][j][r], here = true;
                m = fmaxf(m, acc[i][j][r]);
            }
        if (here) G.target_logit[row] = z;
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float base = m == -INFINITY ? 0.0f : m;       // of nothing but -inf: a sum of 0
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < T::MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s += __builtin_amdgcn_exp2f(G.k * (acc[i][j][r] - base));
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (lane < 16) joint[wm * T::BN + n] = float2{m, s};
    }
    __syncthreads();
    for (int n = threadIdx.x; n < T::BN; n += T::BLOCK) {
        float m = -INFINITY, s = 0.0f;
        for (int q = 0; q < T::WM; ++q) m = fmaxf(m, joint[q * T::BN + n].x);
        const float base = m == -INFINITY ? 0.0f : m;
        for (int q = 0; q < T::WM; ++q) s += joint[q * T::BN + n].y * __builtin_amdgcn_exp2f(G.k * (joint[q * T::BN + n].x - base));
        G.partials[(G.word0 / T::BM + tw) * G.rows + tr * T::BN + n] = float2{m, s};
    }
}

// dz of a tile of words, rounded to bf16; zeros in rows from count on and for words behind the vocabulary, which products that follow may meet
template <typename T>
__global__ __launch_bounds__(T::BLOCK, T::BLOCK / 256) void k_head_dz(Operand W, Operand X, int steps, Logit G)
{
    __shared__ __attribute__((aligned(128))) char lds[STAGES * T::STAGE];
    int64_t tw, tr;
    if (!my_tile((G.words + T::BM - 1) / T::BM, G.rows / T::BN, tw, tr)) return;
    const int count = *G.live.count;
    if (tr * T::BN >= count) return;
    f32x4 acc[T::MI][T::NI];
    product<T, true, true, false>(W, X, tw * T::BM, tr * T::BN, 0, steps, lds, acc);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / T::WN, wn = wave % T::WN;
    const int64_t w0 = G.word0 + tw * T::BM + wm * T::MI * 16;
    add_bias<T>(G, w0, lane, acc);
    const int left = words_left(G, w0, lane);
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
        const int64_t row = tr * T::BN + (wn * T::NI + j) * 16 + column_of(lane);
        const bool live = row < count;
        const int target = live ? place_of(G.targets[G.live.index[row]], w0, lane) : -1;
        const int words = live ? left : 0;
        const float4 R = live ? G.row[row] : float4{};
        uint16_t *out = G.dz + row * G.dz_stride + (w0 - G.word0) + words_before(lane);
#pragma unroll
        for (int i = 0; i < T::MI; ++i) {
            float d[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int w = word_of(i, r);
                const float p = __builtin_amdgcn_exp2f(G.k * (acc[i][j][r] - R.x)) * R.y;
                d[r] = w < words ? R.z * ((w == target ? 1.0f : 0.0f) - p) : 0.0f;
            }
            *reinterpret_cast<u32x2 *>(out + word_of(i, 0)) = u32x2{two_bf16(d[0], d[1]), two_bf16(d[2], d[3])};
        }
    }
}

// sum[split][row][h] (+)= dz W over a piece of the vocabulary
struct ToRows {
    Live live;
    int64_t rows, hidden;
    float *sum;
    int first;                // of the pieces
    int splits, steps;        // steps: of the piece
};
template <typename T>
__global__ __launch_bounds__(T::BLOCK, T::BLOCK / 256) void k_head_dx(Operand DZ, Operand W, ToRows G)
{
    __shared__ __attribute__((aligned(128))) char lds[STAGES * T::STAGE];
    int64_t tr, th;
    if (!my_tile(G.rows / T::BM, (G.hidden + T::BN - 1) / T::BN, tr, th)) return;
    if (tr * T::BM >= *G.live.count) return;
    const int per = (G.steps + G.splits - 1) / G.splits, from = blockIdx.y * per, mine = G.steps - from < per ? G.steps - from : per;
    f32x4 acc[T::MI][T::NI];
    product<T, true, false, true>(DZ, W, tr * T::BM, th * T::BN, (int64_t)from * BK, mine, lds, acc);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / T::WN, wn = wave % T::WN;
#pragma unroll
    for (int i = 0; i < T::MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t row = tr * T::BM + (wm * T::MI + i) * 16 + row_of(r, lane);
            float *out = G.sum + ((int64_t)blockIdx.y * G.rows + row) * G.hidden;
#pragma unroll
            for (int j = 0; j < T::NI; ++j) {
                const int64_t h = th * T::BN + (wn * T::NI + j) * 16 + column_of(lane);
                if (h < G.hidden) out[h] = G.first ? acc[i][j][r] : out[h] + acc[i][j][r];
            }
        }
}

// dW[word][h] = dz^T x of a piece of the vocabulary
struct ToWeights {
    Live live;
    int64_t word0, words, hidden;
    uint16_t *dw;
    int64_t stride;
    const float4 *row;
};
template <typename T>
__global__ __launch_bounds__(T::BLOCK, T::BLOCK / 256) void k_head_dw(Operand DZ, Operand X, ToWeights G)
{
    __shared__ __attribute__((aligned(128))) char lds[STAGES * T::STAGE];
    int64_t tw, th;
    if (!my_tile((G.words + T::BM - 1) / T::BM, (G.hidden + T::BN - 1) / T::BN, tw, th)) return;
    f32x4 acc[T::MI][T::NI];
    const int count = *G.live.count;
    product<T, false, false, false>(DZ, X, tw * T::BM, th * T::BN, 0, (count + BK - 1) / BK, lds, acc);
    const float unit = count ? G.row[0].w : 1.0f;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / T::WN, wn = wave % T::WN;
#pragma unroll
    for (int i = 0; i < T::MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t w = tw * T::BM + (wm * T::MI + i) * 16 + row_of(r, lane);
            if (w >= G.words) continue;
            uint16_t *out = G.dw + (G.word0 + w) * G.stride;
#pragma unroll
            for (int j = 0; j < T::NI; ++j) {
                const int64_t h = th * T::BN + (wn * T::NI + j) * 16 + column_of(lane);
                if (h < G.hidden) out[h] = (uint16_t)f32_to_bf16_bits(acc[i][j][r] * unit);
            }
        }
}

// db[word] = sum over rows of dz: a lane two words, a wave a share of the rows
__global__ __launch_bounds__(1024) void k_head_db(const uint16_t *dz, int64_t dz_stride, Live live, int64_t words, const float4 *row, uint16_t *db)
{
    __shared__ float part[16][128];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 128 + lane * 2;           // a piece's rows have whole tiles of words
    const int count = *live.count;
    float a = 0.0f, b = 0.0f;
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
// Rows' maxima and sums, joined over the tiles of words: 32 rows a workgroup, 8 lanes a row.
struct Join {
    const float2 *partials;
    const float *target_logit;
    int64_t tiles, rows;       // rows: of the packed batch
    float k, it;
    float *logp, *row_stats;   // of the batch
    const float *weights;      // of the rows, or null for ones: factors of a loss's gradient are -weights / temperature
    float4 *row;               // null: no gradient follows
    Live live;
};
__global__ __launch_bounds__(256) void k_head_join(Join J)
{
    __shared__ float2 part[8][32];
    const int n = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int64_t j = (int64_t)blockIdx.x * 32 + n;
    const int count = *J.live.count;
    if ((int64_t)blockIdx.x * 32 >= count) return;
    float m = -INFINITY, s = 0.0f;
    for (int64_t t = slice; t < J.tiles; t += 8) {
        const float2 q = J.partials[t * J.rows + j];
        const float top = fmaxf(m, q.x), base = top == -INFINITY ? 0.0f : top;
        s = s * __builtin_amdgcn_exp2f(J.k * (m - base)) + q.y * __builtin_amdgcn_exp2f(J.k * (q.x - base));
        m = top;
    }
    part[slice][n] = float2{m, s};
    __syncthreads();
    if (slice != 0 || j >= count) return;
    for (int i = 0; i < 8; ++i) m = fmaxf(m, part[i][n].x);
    const float base = m == -INFINITY ? 0.0f : m;
    s = 0.0f;
    for (int i = 0; i < 8; ++i) s += part[i][n].y * __builtin_amdgcn_exp2f(J.k * (part[i][n].x - base));
    const int64_t r = J.live.index[j];
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

// Rows that do not count: logp 0, statistics (0, 1).  (Before k_head_join, which writes the others.)
__global__ __launch_bounds__(256) void k_head_none(int64_t rows, float *logp, float *row_stats)
{
    const int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (r >= rows) return;
    logp[r] = 0.0f;
    if (row_stats) row_stats[2 * r] = 0.0f, row_stats[2 * r + 1] = 1.0f;
}

// loss (+)= sum of weights times -logp over the rows that count
__global__ __launch_bounds__(1024) void k_head_loss(Live live, const float *logp, const float *weights, float *loss, int accumulate)
{
    __shared__ double lds[16];
    const int count = *live.count;
    double s = 0.0;
    for (int j = threadIdx.x; j < count; j += 1024) {
        const int r = live.index[j];
        s -= (double)(weights ? weights[r] : 1.0f) * (double)logp[r];
    }
    s = block_sum<1024>(s, lds);
    if (threadIdx.x == 0) *loss = (float)(s + (accumulate ? (double)*loss : 0.0));
}

// dx of the rows that count from their sums, and zeros
__global__ __launch_bounds__(256) void k_head_rows_out(Live live, const float *sum, int splits, int64_t rows, int64_t hidden, const float4 *row, uint16_t *dx, int64_t stride)
{
    const int64_t j = blockIdx.x;
    if (j >= *live.count) return;
    uint16_t *out = dx + (int64_t)live.index[j] * stride;
    const float unit = row[j].w;
    for (int64_t h = threadIdx.x; h < hidden; h += 256) {
        float s = sum[j * hidden + h];
        for (int i = 1; i < splits; ++i) s += sum[((int64_t)i * rows + j) * hidden + h];
        out[h] = (uint16_t)f32_to_bf16_bits(s * unit);
    }
}
__global__ __launch_bounds__(256) void k_head_zero(uint16_t *p, int64_t stride, int64_t cols)
{
    for (int64_t c = threadIdx.x; c < cols; c += 256) p[blockIdx.x * stride + c] = 0;
}

// ---- the plan of a call ------------------------------------------------------------------------
typedef Tile<256, 256, 2, 4> Big;

constexpr int64_t kMaxRows = 1 << 20, kMaxHidden = 1 << 17, kMaxVocab = 1 << 30;
constexpr int64_t kPieceBytes = 256 << 20;          // of dz

struct Plan {
    int64_t rows;            // of the packed batch
    int64_t width;           // of its rows, and of packed weights
    int64_t piece;           // words
    int64_t tiles;           // of words, 256 each
    int splits;              // of the sums to the rows
    size_t index, x, partials, target, row, dz, sum, w, all;      // places in the workspace, and its size
};
static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
// Packed weights are reckoned with in any case where they may be needed: alignment is not known when the size is asked for.
static Plan plan_of(int64_t rows, int64_t hidden, int64_t vocab, bool gradient)
{
    Plan P = {};
    P.rows = up(std::max<int64_t>(rows, 1), 256);
    P.width = up(hidden, 64);
    P.tiles = up(vocab, 256) / 256;
    const int64_t most = std::max<int64_t>(1, kPieceBytes / (2 * P.rows * 256));
    P.piece = std::min(P.tiles, most) * 256;
    const int64_t out = P.rows / 256 * (up(hidden, 256) / 256);                // tiles of the sums to the rows
    P.splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(P.piece / 1024, 32), 512 / out));
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += (size_t)up(bytes, 256);
        return here;
    };
    P.index = take(P.rows * 4 + 256);
    P.x = take(P.rows * P.width * 2);
    P.partials = take(P.tiles * P.rows * 8);
    P.target = take(P.rows * 4);
    P.row = take(P.rows * 16);
    P.dz = gradient ? take(P.rows * P.piece * 2) : at;
    P.sum = gradient ? take(P.splits * P.rows * hidden * 4) : at;
    P.w = take(P.piece * P.width * 2);
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
    int32_t *index() const { return reinterpret_cast<int32_t *>(ws + P.index); }
    uint16_t *x() const { return reinterpret_cast<uint16_t *>(ws + P.x); }
    uint16_t *w() const { return reinterpret_cast<uint16_t *>(ws + P.w); }
    uint16_t *dz() const { return reinterpret_cast<uint16_t *>(ws + P.dz); }
    float *sum() const { return reinterpret_cast<float *>(ws + P.sum); }
    float2 *partials() const { return reinterpret_cast<float2 *>(ws + P.partials); }
    float *target() const { return reinterpret_cast<float *>(ws + P.target); }
    float4 *row() const { return reinterpret_cast<float4 *>(ws + P.row); }
};

static bool multiple16(const void *p, int64_t stride) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(stride * 2)) & 15) == 0; }

static Call call_of(const gs_head &h, const int64_t *targets, float temperature, bool gradient, void *ws, void *stream)
{
    Call C = {};
    C.h = h;
    if (h.rows <= 1) C.h.x_stride = h.hidden;
    if (h.vocab <= 1) C.h.w_stride = h.hidden;
    C.P = plan_of(h.rows, h.hidden, h.vocab, gradient);
    C.ws = static_cast<char *>(ws);
    C.targets = targets;
    C.it = 1.0f / temperature;
    C.live = {C.index() + 64, C.index()};
    C.stream = static_cast<hipStream_t>(stream);
    C.packed = h.hidden % 64 != 0 || !multiple16(h.w, C.h.w_stride) || C.h.w_stride >= 1 << 23;
    return C;
}

// the rows that count, packed
static hipError_t pack_rows(const Call &C, const float *factor)
{
    k_head_live<<<1, LIVE_BLOCK, 0, C.stream>>>(C.targets, factor, (int)C.h.rows, (int)C.h.vocab, C.live);
    if (multiple16(C.h.x, C.h.x_stride)) k_head_pack<true><<<(uint32_t)C.P.rows, 256, 0, C.stream>>>(C.h.x, C.h.x_stride, C.h.hidden, C.live, C.P.rows, C.x(), C.P.width);
    else k_head_pack<false><<<(uint32_t)C.P.rows, 256, 0, C.stream>>>(C.h.x, C.h.x_stride, C.h.hidden, C.live, C.P.rows, C.x(), C.P.width);
    return hipGetLastError();
}
// the weights of a piece of the vocabulary, from word0 on
static Operand weights(const Call &C, int64_t word0, int64_t words)
{
    if (!C.packed) return {C.h.w + word0 * C.h.w_stride, C.h.w_stride, words, C.h.hidden};
    if (multiple16(C.h.w, C.h.w_stride))
        k_head_pack<true><<<(uint32_t)words, 256, 0, C.stream>>>(C.h.w + word0 * C.h.w_stride, C.h.w_stride, C.h.hidden, Live{}, words, C.w(), C.P.width);
    else k_head_pack<false><<<(uint32_t)words, 256, 0, C.stream>>>(C.h.w + word0 * C.h.w_stride, C.h.w_stride, C.h.hidden, Live{}, words, C.w(), C.P.width);
    return {C.w(), C.P.width, words, C.P.width};
}
static Logit logit_of(const Call &C, int64_t word0, int64_t words)
{
    Logit G = {};
    G.bias = C.h.bias;
    G.targets = C.targets;
    G.live = C.live;
    G.rows = C.P.rows;
    G.word0 = word0;
    G.words = words;
    G.vocab = C.h.vocab;
    G.k = kLog2e * C.it;
    G.it = C.it;
    G.partials = C.partials();
    G.target_logit = C.target();
    G.row = C.row();
    G.dz = C.dz();
    G.dz_stride = C.P.piece;
    return G;
}
static uint32_t grid_of(int64_t tiles) { return (uint32_t)(up(tiles, 8)); }

template <typename F> static hipError_t pieces(const Call &C, F each)
{
    for (int64_t w = 0; w < C.h.vocab; w += C.P.piece) {
        const int64_t words = std::min(C.P.piece, C.h.vocab - w);
        if (hipError_t e = each(w, words, weights(C, w, words)); e != hipSuccess) return e;
    }
    return hipSuccess;
}

static hipError_t forward(const Call &C, float *logp, float *row_stats, const float *row_weights, bool gradient)
{
    const Operand X = {C.x(), C.P.width, C.P.rows, C.P.width};
    hipError_t e = pieces(C, [&](int64_t w, int64_t words, const Operand &W) {
        Logit G = logit_of(C, w, words);
        k_head_stats<Big><<<grid_of(up(words, 256) / 256 * (C.P.rows / 256)), Big::BLOCK, 0, C.stream>>>(W, X, (int)(C.P.width / BK), G);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    if (C.h.rows) k_head_none<<<(uint32_t)((C.h.rows + 255) / 256), 256, 0, C.stream>>>(C.h.rows, logp, row_stats);
    const Join J = {C.partials(), C.target(), C.P.tiles, C.P.rows, kLog2e * C.it, C.it, logp, row_stats, row_weights, gradient ? C.row() : nullptr, C.live};
    k_head_join<<<(uint32_t)(C.P.rows / 32), 256, 0, C.stream>>>(J);
    return hipGetLastError();
}

static hipError_t backward(const Call &C, const gs_head_grads &D)
{
    const Operand X = {C.x(), C.P.width, C.P.rows, C.P.width};
    const int64_t H = C.h.hidden, htiles = up(H, 256) / 256, rtiles = C.P.rows / 256;
    hipError_t e = pieces(C, [&](int64_t w, int64_t words, const Operand &W) {
        Logit G = logit_of(C, w, words);
        const int64_t wtiles = up(words, 256) / 256;
        k_head_dz<Big><<<grid_of(wtiles * rtiles), Big::BLOCK, 0, C.stream>>>(W, X, (int)(C.P.width / BK), G);
        const Operand DZ = {C.dz(), C.P.piece, C.P.rows, C.P.piece};
        if (D.dx) {
            const ToRows R = {C.live, C.P.rows, H, C.sum(), w == 0, C.P.splits, (int)(up(words, BK) / BK)};
            k_head_dx<Big><<<dim3(grid_of(rtiles * htiles), (uint32_t)C.P.splits), Big::BLOCK, 0, C.stream>>>(DZ, W, R);
        }
        if (D.dw) {
            const ToWeights R = {C.live, w, words, H, D.dw, D.dw_stride, C.row()};
            k_head_dw<Big><<<grid_of(wtiles * htiles), Big::BLOCK, 0, C.stream>>>(DZ, X, R);
        }
        if (D.dbias) k_head_db<<<(uint32_t)((words + 127) / 128), 1024, 0, C.stream>>>(C.dz(), C.P.piece, C.live, words, C.row(), D.dbias + w);
        return hipGetLastError();
    });
    if (e != hipSuccess || !D.dx || !C.h.rows) return e;
    k_head_zero<<<(uint32_t)C.h.rows, 256, 0, C.stream>>>(D.dx, D.dx_stride, H);
    k_head_rows_out<<<(uint32_t)C.P.rows, 256, 0, C.stream>>>(C.live, C.sum(), C.P.splits, C.P.rows, H, C.row(), D.dx, D.dx_stride);
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
    return plan_of(rows, hidden, vocab, gradient != 0).all;
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
    const Call C = call_of(*head, targets, temperature, false, d_workspace, stream);
    hipError_t e = pack_rows(C, nullptr);
    if (e == hipSuccess) e = forward(C, logp, row_stats, nullptr, false);
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_head_logp launch");
}

gs_status gs_head_logp_grad(const gs_head *head, const int64_t *targets, float temperature, const float *row_stats, const float *dlogp,
                            const gs_head_grads *grads, void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!good_head(head) || !good_temperature(temperature) || !good_grads(*head, grads)) return GS_ERR_INVALID_ARG;
    const int64_t rows = head->rows;
    if (rows && (!good(targets, 8) || !good(row_stats, 4) || !good(dlogp, 4))) return GS_ERR_INVALID_ARG;
    if (!good(d_workspace, 256) || workspace_bytes < gs_head_workspace_bytes(rows, head->hidden, head->vocab, 1)) return GS_ERR_WORKSPACE;
    Ranges R;
    R.add(*head);
    R.add(*head, *grads);
    R.add(targets, rows * 8, false);
    R.add(row_stats, rows * 8, false);
    R.add(dlogp, rows * 4, false);
    R.add(d_workspace, (int64_t)workspace_bytes, true);
    if (!R.apart()) return GS_ERR_INVALID_ARG;
    const Call C = call_of(*head, targets, temperature, true, d_workspace, stream);
    hipError_t e = pack_rows(C, dlogp);
    if (e == hipSuccess) {
        k_head_rows<<<(uint32_t)(C.P.rows / 256), 256, 0, C.stream>>>(C.live, row_stats, dlogp, C.it, C.row());
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = backward(C, *grads);
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
    const Call C = call_of(*head, targets, temperature, grads != nullptr, d_workspace, stream);
    hipError_t e = pack_rows(C, weights);
    if (e == hipSuccess) e = forward(C, logp, nullptr, weights, grads != nullptr);
    if (e == hipSuccess) {
        k_head_loss<<<1, 1024, 0, C.stream>>>(C.live, logp, weights, d_loss, accumulate);
        e = hipGetLastError();
    }
    if (e == hipSuccess && grads) e = backward(C, *grads);
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_head_cross_entropy launch");
}

}  // extern "C"
