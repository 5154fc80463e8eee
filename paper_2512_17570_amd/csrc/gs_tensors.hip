// gs_tensors.hip -- norm and clip of gradients that are many tensors: a training program's list of parameters, where the
// other norms take one flat layer.
//
// One pass that reads every element (the norm) and one that reads and writes it (the clip): HBM-bound.  A launch takes a
// table of tensors in its arguments, so nothing is copied to the device first and nothing is kept from call to call; its workgroups
// are tiles of one tensor each, and find which by a look at the first tile of every tensor.
//   Measured: 805 M fp32 gradients in 12 tensors, norm 0.474 ms (6.8 TB/s), clip into other buffers 1.00 ms (6.4); 201 M in 48 tensors of
// both types 64 and 118 us (6.3, 6.8: the end of what the norm read is still in the memory-side cache, 184 us together against 189 in the
// norm's own order); 48 tensors of 2048 to 8192 bf16 elements 5.3 and 4.0 us on the GPU, 9 to 12 us a pass, as fast as the host calls.  A plain
// copy reaches 6.7 TB/s on the same card, reading 7.1.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdlib>
#include <cstring>
#include <type_traits>

#include "gs_device.h"
#include "gs_internal.h"

#pragma clang fp contract(off)

namespace gs {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int TENSOR_BLOCK = 256;
// Tensors of one launch, in the 4096 bytes that its arguments may have: a short list, which is quick to go through, a long one, and a long
// one of tensors that stay where they are.  With 128 at most, as addresses and lengths of 64 bits each would have it, norm and clip of 144 tensors
// of 100 to 40 000 elements take 21.5 us against 15, of 448 of 4096 elements 47 against 35; with 1.7 MB a tensor level, 1 to 3 % ahead.
constexpr int TABLE_SMALL = 16, TABLE = 160, TABLE_IN_PLACE = 240;
constexpr int64_t PIECE = (int64_t)1 << 31;     // longer tensors go as pieces of so many elements, whose number takes 32 bits

struct Entry {
    const void *in;
    void *out;
    int64_t numel;
    int32_t dtype;
    uint32_t first;                    // its first tile, of this launch's
};
__device__ __forceinline__ void *address(uint32_t lo, uint32_t hi)
{
    return (void *)(__attribute__((address_space(1))) void *)((uint64_t)hi << 32 | lo);       // device memory, not what may be LDS
}
// An address of either type is even: the type takes its lowest bit.
struct Whereabouts {
    uint32_t lo, hi, numel;
    static Whereabouts of(const gs_tensor &x)
    {
        const uint64_t a = reinterpret_cast<uintptr_t>(x.data) | (x.dtype == GS_BF16 ? 1 : 0);
        return {(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)x.numel};
    }
    __device__ __forceinline__ Entry entry(uint32_t first) const
    {
        void *p = address(lo & ~1u, hi);
        return {p, p, (int64_t)numel, lo & 1 ? GS_BF16 : GS_F32, first};
    }
};
struct WithOut {
    Whereabouts in;
    uint32_t lo, hi;
    static WithOut of(const gs_tensor &x)
    {
        const uint64_t a = reinterpret_cast<uintptr_t>(x.out ? x.out : x.data);
        return {Whereabouts::of(x), (uint32_t)a, (uint32_t)(a >> 32)};
    }
    __device__ __forceinline__ Entry entry(uint32_t first) const
    {
        Entry e = in.entry(first);
        e.out = address(lo, hi);
        return e;
    }
};
// First tiles beside each other, so that looking for a tile's tensor takes few lines of memory; ~0 behind the last tensor.
template <int N> struct Table {
    typedef std::conditional_t<N == TABLE_IN_PLACE, Whereabouts, WithOut> S;
    alignas(16) uint32_t first[N];
    uint32_t tiles, keep_tile;         // norm: tiles from this one on are left in the memory-side cache, for the clip
    int32_t count, runs;               // runs: of NV vectors a lane, one after another in a tile
    S e[N];
};

// The tensor that a tile belongs to: the last one whose first tile is not behind it.  A short list is gone through by the scalar unit, of
// a long one every lane looks at four, in one load: with a load each, clip of 144 tensors of 1.7 MB 207 us against 200.
template <int N>
__device__ __forceinline__ Entry entry_of(const Table<N> &t, uint32_t tile)
{
    int n = 0;
    if constexpr (N <= TABLE_SMALL) {
#pragma unroll
        for (int i = 1; i < N; ++i) n += t.first[i] <= tile ? 1 : 0;
    } else {
        static_assert(N % 4 == 0 && N <= 256);
        const int lane = threadIdx.x & 63;
        u32x4 f = {~0u, ~0u, ~0u, ~0u};
        if (lane < N / 4) f = reinterpret_cast<const u32x4 *>(t.first)[lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) n += __popcll(__ballot(f[i] <= tile));
        n = __builtin_amdgcn_readfirstlane(n - 1);
    }
    return t.e[n].entry(t.first[n]);
}

// A tile's part of a tensor: the vectors [at, end) behind `head` single elements, counted from the start of the first one's 128-byte line
// (`skip` of that line are not the tensor's), and whether it has the single ones of both ends (the tensor's first tile does).
struct Part {
    int64_t at, end, rest;             // rest: elements from the first of them behind the vectors
    int skip, head, singles;
};
template <int PER>
__device__ __forceinline__ Part part_of(const Entry &e, const void *p, uint32_t tile, uint32_t tile_vecs)
{
    Part c;
    const int64_t off = ((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (16 / PER);
    c.head = (int)(off < e.numel ? off : e.numel);
    const int64_t vecs = (e.numel - c.head) / PER;
    c.skip = (int)((reinterpret_cast<uintptr_t>(p) + 15) >> 4) & 7;
    c.at = (int64_t)(tile - e.first) * tile_vecs;
    c.end = c.skip + vecs;
    c.rest = c.head + vecs * PER;
    c.singles = tile == e.first ? c.head + (int)(e.numel - c.rest) : 0;          // at most 14
    return c;
}
__device__ __forceinline__ int64_t single(const Part &c, int i) { return i < c.head ? i : c.rest + (i - c.head); }

template <int PER>
__device__ __forceinline__ void square(u32x4 q, double &x, double &y)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (PER == 8) {
            const double lo = bf16_lo(q[i]), hi = bf16_hi(q[i]);
            x = fma(lo, lo, x);
            y = fma(hi, hi, y);
        } else {
            const double g = __uint_as_float(q[i]);
            if (i & 1) y = fma(g, g, y);
            else x = fma(g, g, x);
        }
    }
}
template <int PER> __device__ __forceinline__ float load_one(const void *p, int64_t i)
{
    if constexpr (PER == 8) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[i] << 16);
    else return static_cast<const float *>(p)[i];
}

template <int PER, int NV, bool KEEP>
__device__ __forceinline__ double tile_squares(const Entry &e, uint32_t tile, int runs)
{
    const Part c = part_of<PER>(e, e.in, tile, (uint32_t)(TENSOR_BLOCK * NV) * runs);
    const u32x4 *v = reinterpret_cast<const u32x4 *>(static_cast<const char *>(e.in) + c.head * (16 / PER)) - c.skip + c.at;
    int64_t from = c.skip - c.at, to = c.end - c.at;               // of the tile's vectors
    double x = 0.0, y = 0.0;
    if ((int)threadIdx.x < c.singles) {
        const double g = load_one<PER>(e.in, single(c, threadIdx.x));
        x = g * g;
    }
    for (int run = 0; run < runs && to > 0; ++run, v += TENSOR_BLOCK * NV, from -= TENSOR_BLOCK * NV, to -= TENSOR_BLOCK * NV) {
        u32x4 q[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = j * TENSOR_BLOCK + (int)threadIdx.x;
            q[j] = u32x4{0, 0, 0, 0};
            if (i >= from && i < to) q[j] = KEEP ? v[i] : __builtin_nontemporal_load(v + i);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) square<PER>(q[j], x, y);
    }
    return x + y;
}

// before: tiles of the launches in front of this one, which meet with its own.
template <int N, int NV>
__global__ __launch_bounds__(TENSOR_BLOCK) void k_tensors_sqnorm(Table<N> t, double *partials, Meeting meet, int before, double *out, int accumulate)
{
    __shared__ double lds[TENSOR_BLOCK / 64];
    const uint32_t tile = blockIdx.x;
    const Entry e = entry_of(t, tile);
    double x;
    if (e.dtype == GS_BF16) x = tile < t.keep_tile ? tile_squares<8, NV, false>(e, tile, t.runs) : tile_squares<8, NV, true>(e, tile, t.runs);
    else x = tile < t.keep_tile ? tile_squares<4, NV, false>(e, tile, t.runs) : tile_squares<4, NV, true>(e, tile, t.runs);
    const double s = block_sum<TENSOR_BLOCK>(x, lds);
    if (meet.n == 0) {
        if (threadIdx.x == 0) partials[tile] = s;
        return;
    }
    if (threadIdx.x >= 64) return;
    uint32_t w[2];
    halves(s, w[0], w[1]);
    if (threadIdx.x == 0) leave(meet, before + (int)tile, w);
    if (!last_of(meet, !accumulate, w)) return;
    double all[1];
    left_sums(meet, w, all);
    if (threadIdx.x == 63) *out = accumulate ? *out + all[0] : all[0];
    clear<2>(meet);
}

// The partials of many tiles, a run of FOLD_RUN of them a workgroup, or what that comes to with FOLD_MAX of them.
constexpr int FOLD_BLOCK = 1024, FOLD_RUN = 4096, FOLD_MAX = 64;
__global__ __launch_bounds__(FOLD_BLOCK) void k_tensors_fold(const double *partials, int count, Meeting meet, double *out, int accumulate)
{
    __shared__ double lds[FOLD_BLOCK / 64];
    double x = 0.0;
    for (int i = (int)blockIdx.x * FOLD_BLOCK + (int)threadIdx.x; i < count; i += meet.n * FOLD_BLOCK) x += partials[i];
    const double s = block_sum<FOLD_BLOCK>(x, lds);
    if (threadIdx.x >= 64) return;
    uint32_t w[2];
    halves(s, w[0], w[1]);
    if (threadIdx.x == 0) leave(meet, (int)blockIdx.x, w);
    if (!last_of(meet, !accumulate, w)) return;
    double all[1];
    left_sums(meet, w, all);
    if (threadIdx.x == 63) *out = accumulate ? *out + all[0] : all[0];
    clear<2>(meet);
}

template <int PER> __device__ __forceinline__ u32x4 scaled(u32x4 q, float c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (PER == 8) {                     // rounded to nearest even, NaN stays NaN
            const bf16x2 h = {(__bf16)(c * bf16_lo(q[i])), (__bf16)(c * bf16_hi(q[i]))};
            q[i] = __builtin_bit_cast(uint32_t, h);
        } else {
            q[i] = __float_as_uint(c * __uint_as_float(q[i]));
        }
    }
    return q;
}

template <int PER, int NV>
__device__ __forceinline__ void tile_scaled(const Entry &e, uint32_t tile, int runs, float c)
{
    const int64_t tile_vecs = (int64_t)(TENSOR_BLOCK * NV) * runs;
    auto one = [&](int64_t i) {
        const float g = c * load_one<PER>(e.in, i);
        if constexpr (PER == 8) static_cast<uint16_t *>(e.out)[i] = (uint16_t)f32_to_bf16_bits(g);
        else static_cast<float *>(e.out)[i] = g;
    };
    if (((reinterpret_cast<uintptr_t>(e.in) ^ reinterpret_cast<uintptr_t>(e.out)) & 15) != 0) {      // no vectors in common
        const int64_t a = (int64_t)(tile - e.first) * tile_vecs * PER, b = a + tile_vecs * PER;
        for (int64_t i = a + threadIdx.x; i < b && i < e.numel; i += TENSOR_BLOCK) one(i);
        return;
    }
    const Part p = part_of<PER>(e, e.in, tile, (uint32_t)tile_vecs);
    const int64_t shift = p.at - p.skip;
    int64_t from = p.skip - p.at, to = p.end - p.at;
    const u32x4 *vi = reinterpret_cast<const u32x4 *>(static_cast<const char *>(e.in) + p.head * (16 / PER)) + shift;
    u32x4 *vo = reinterpret_cast<u32x4 *>(static_cast<char *>(e.out) + p.head * (16 / PER)) + shift;
    for (int run = 0; run < runs && to > 0; ++run, vi += TENSOR_BLOCK * NV, vo += TENSOR_BLOCK * NV, from -= TENSOR_BLOCK * NV, to -= TENSOR_BLOCK * NV) {
        u32x4 q[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = j * TENSOR_BLOCK + (int)threadIdx.x;
            if (i >= from && i < to) q[j] = __builtin_nontemporal_load(vi + i);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = j * TENSOR_BLOCK + (int)threadIdx.x;
            if (i >= from && i < to) store_through(vo + i, scaled<PER>(q[j], c));
        }
    }
    if ((int)threadIdx.x < p.singles) one(single(p, threadIdx.x));
}

// From the last tile on: the end of what the norm read is still in the memory-side cache.  Where the coefficient is 1, tensors
// that stay where they are are left alone.
template <int N, int NV>
__global__ __launch_bounds__(TENSOR_BLOCK) void k_tensors_clip(Table<N> t, const double *d_sqnorm, float max_norm, float *d_norm)
{
    const double S = *d_sqnorm;
    if (d_norm && blockIdx.x == 0 && threadIdx.x == 0) *d_norm = (float)sqrt(S);
    if (t.count == 0) return;
    const uint32_t tile = t.tiles - 1 - blockIdx.x;
    const Entry e = entry_of(t, tile);
    const float c = clip_from(S, max_norm);
    if (c == 1.0f && e.out == e.in) return;
    if (e.dtype == GS_BF16) tile_scaled<8, NV>(e, tile, t.runs, c);
    else tile_scaled<4, NV>(e, tile, t.runs, c);
}

// ---- launchers --------------------------------------------------------------------------------
// Vectors of a lane.  Clip of 805 M fp32 with 1 / 2 / 4 / 8 of them 1.13/0.99/1.10/1.18 ms, with two of them not written through 1.05, with
// fewer workgroups on a CU more; norm of 201 M in 48 tensors 99/66/62/64 us.
constexpr int NORM_NV = 4, CLIP_NV = 2;
static int64_t size_of(const gs_tensor &t) { return t.dtype == GS_BF16 ? 2 : 4; }
// tiles of 2^shift vectors in a tensor: its vectors counted from the start of the first one's line
static uint64_t tiles_of(const gs_tensor &t, int shift) { return (uint64_t)(((t.numel >> (t.dtype == GS_BF16 ? 3 : 2)) + 7) >> shift) + 1; }
static uint64_t tiles_of(const gs_tensor *t, int64_t count, int shift)
{
    uint64_t n = 0;
    for (int64_t i = 0; i < count; ++i) n += t[i].numel ? tiles_of(t[i], shift) : 0;
    return n;
}

// Tiles of a list: 2^shift vectors each, in runs of NV a lane, so many that there are no more of them than `most`.
struct Tiles {
    uint64_t count;
    int shift, runs;
};
template <int NV>
static Tiles tiles_for(const gs_tensor *t, int64_t count, uint64_t most)
{
    static_assert((TENSOR_BLOCK * NV & (TENSOR_BLOCK * NV - 1)) == 0);
    Tiles r = {0, __builtin_ctz(TENSOR_BLOCK * NV), 1};
    while ((r.count = tiles_of(t, count, r.shift)) > most) ++r.shift, r.runs *= 2;
    return r;
}

// Calls launch(table) for tables of up to N tensors that hold all of them between them; `back`: from the last one on.  Bytes of the list
// from keep_from on are marked to be kept.
template <int N, typename F>
static hipError_t for_tables(const gs_tensor *tensors, int64_t count, const Tiles &tiles, bool back, int64_t keep_from, F launch)
{
    Table<N> t;
    int64_t at = 0;                    // bytes before this tensor
    for (int64_t left = count; left > 0;) {
        // the next N tensors with elements, or the last N of those that are left
        int64_t a = back ? left : count - left, b = a;
        for (int n = 0; n < N && (back ? a > 0 : b < count); back ? --a : ++b) n += tensors[back ? a - 1 : b].numel != 0;
        left -= b - a;
        t.count = 0;
        t.runs = tiles.runs;
        t.tiles = 0;
        t.keep_tile = ~0u;
        for (int64_t i = a; i < b; ++i) {
            const gs_tensor &x = tensors[i];
            if (x.numel == 0) continue;
            const int64_t bytes = x.numel * size_of(x);
            if (t.keep_tile == ~0u && at + bytes > keep_from) t.keep_tile = t.tiles + (uint32_t)(keep_from > at ? (keep_from - at) >> (tiles.shift + 4) : 0);
            at += bytes;
            t.first[t.count] = t.tiles;
            t.e[t.count++] = Table<N>::S::of(x);
            t.tiles += (uint32_t)tiles_of(x, tiles.shift);
        }
        if (t.count == 0) continue;
        for (int i = t.count; i < N; ++i) t.first[i] = ~0u;
        if (hipError_t e = launch(t); e != hipSuccess) return e;
    }
    return hipSuccess;
}

static bool good_tensors(const gs_tensor *tensors, int64_t count, bool outs)
{
    if (count < 0 || count > GS_MAX_TENSORS || (count && !tensors)) return false;
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) {
        const gs_tensor &t = tensors[i];
        if ((t.dtype != GS_BF16 && t.dtype != GS_F32) || t.numel < 0) return false;
        if (t.numel == 0) continue;
        const uintptr_t to = (uintptr_t)size_of(t) - 1;
        if (!t.data || (reinterpret_cast<uintptr_t>(t.data) & to)) return false;
        if (outs && (reinterpret_cast<uintptr_t>(t.out) & to)) return false;
        if (t.numel > (int64_t)1 << 44 || (total += t.numel) > (int64_t)1 << 44) return false;
    }
    return true;
}

// Every output against every other array but its own input: sorted by address, an overlap shows against the furthest end so far, of
// the outputs and of all.
static gs_status outputs_apart(const gs_tensor *tensors, int64_t count, const double *d_sqnorm, const float *d_norm)
{
    Range few[66], *r = few;
    if (count > 32 && !(r = static_cast<Range *>(malloc(sizeof(Range) * (2 * (size_t)count + 2))))) return GS_ERR_NOMEM;
    size_t n = 0;
    for (int64_t i = 0; i < count; ++i) {
        const gs_tensor &t = tensors[i];
        if (t.numel == 0) continue;
        const int64_t bytes = t.numel * size_of(t);
        if (t.out && t.out != t.data) r[n++] = range_of(t.data, bytes, false);
        r[n++] = range_of(t.out ? t.out : t.data, bytes, true);
    }
    r[n++] = range_of(d_sqnorm, 8, false);
    if (d_norm) r[n++] = range_of(d_norm, 4, true);
    auto less = [](const Range &a, const Range &b) { return a.lo < b.lo; };
    if (!std::is_sorted(r, r + n, less)) std::sort(r, r + n, less);
    uintptr_t any_end = 0, out_end = 0;
    bool good = true;
    for (size_t i = 0; i < n && good; ++i) {
        good = !(r[i].lo < out_end || (r[i].out && r[i].lo < any_end));
        any_end = std::max(any_end, r[i].hi);
        if (r[i].out) out_end = std::max(out_end, r[i].hi);
    }
    if (r != few) free(r);
    return good ? GS_OK : GS_ERR_INVALID_ARG;
}
static bool touches(const gs_tensor *tensors, int64_t count, const Range &o)
{
    for (int64_t i = 0; i < count; ++i)
        if (overlap(range_of(tensors[i].data, tensors[i].numel * size_of(tensors[i]), false), o)) return true;
    return false;
}

// Long tensors in pieces: another list, in memory of the caller's to free.
static bool cut_long(const gs_tensor *&tensors, int64_t &count, void *&memory)
{
    int64_t n = 0, longest = 0;
    for (int64_t i = 0; i < count; ++i) {
        n += tensors[i].numel > PIECE ? (tensors[i].numel + PIECE - 1) / PIECE : 1;
        longest = std::max(longest, tensors[i].numel);
    }
    memory = nullptr;
    if (longest <= PIECE) return true;
    gs_tensor *to = static_cast<gs_tensor *>(memory = malloc(sizeof(gs_tensor) * (size_t)n));
    if (!to) return false;
    n = 0;
    for (int64_t i = 0; i < count; ++i) {
        gs_tensor x = tensors[i];
        for (int64_t left = x.numel; left > 0; left -= PIECE) {
            x.numel = std::min(left, PIECE);
            to[n++] = x;
            x.data = static_cast<char *>(const_cast<void *>(x.data)) + PIECE * size_of(x);
            if (x.out) x.out = static_cast<char *>(x.out) + PIECE * size_of(x);
        }
    }
    tensors = to;
    count = n;
    return true;
}

template <int N>
static hipError_t norm(const gs_tensor *tensors, int64_t count, double *d_sqnorm, int accumulate, void *ws, hipStream_t stream)
{
    const Tiles tiles = tiles_for<NORM_NV>(tensors, count, GS_SQNORM_MAX_BLOCKS);
    Meeting meet = {};
    if (tiles.count > 0 && tiles.count <= MEET_MAX) meet = {static_cast<uint64_t *>(ws), next_tag(), (int)tiles.count};
    int64_t bytes = 0, done = 0;
    for (int64_t i = 0; i < count; ++i) bytes += tensors[i].numel * size_of(tensors[i]);
    double *partials = static_cast<double *>(ws);
    hipError_t e = for_tables<N>(tensors, count, tiles, false, bytes - GS_KEEP_BYTES, [&](const Table<N> &t) {
        k_tensors_sqnorm<N, NORM_NV><<<t.tiles, TENSOR_BLOCK, 0, stream>>>(t, partials + done, meet, (int)done, d_sqnorm, accumulate);
        done += t.tiles;
        return hipGetLastError();
    });
    if (e != hipSuccess || meet.n || (done == 0 && accumulate)) return e;
    const int64_t blocks = (done + FOLD_RUN - 1) / FOLD_RUN;
    // its slots lie behind the partials
    meet = {static_cast<uint64_t *>(ws) + GS_SQNORM_MAX_BLOCKS, next_tag(), (int)(blocks < 1 ? 1 : blocks > FOLD_MAX ? FOLD_MAX : blocks)};
    static_assert(2 * FOLD_MAX <= GS_FINAL_SLICES);
    k_tensors_fold<<<meet.n, FOLD_BLOCK, 0, stream>>>(partials, (int)done, meet, d_sqnorm, accumulate);
    return hipGetLastError();
}

template <int N>
static hipError_t clip(const gs_tensor *tensors, int64_t count, const double *d_sqnorm, float max_norm, float *d_norm, hipStream_t stream)
{
    const Tiles tiles = tiles_for<CLIP_NV>(tensors, count, 1u << 23);
    hipError_t e = for_tables<N>(tensors, count, tiles, true, INT64_MAX, [&](const Table<N> &t) {
        k_tensors_clip<N, CLIP_NV><<<t.tiles, TENSOR_BLOCK, 0, stream>>>(t, d_sqnorm, max_norm, d_norm);
        d_norm = nullptr;              // written by the first launch
        return hipGetLastError();
    });
    if (e == hipSuccess && d_norm) {   // nothing to scale, but a norm is asked for
        Table<TABLE_SMALL> none;
        memset(&none, 0, sizeof none);
        k_tensors_clip<TABLE_SMALL, CLIP_NV><<<1, TENSOR_BLOCK, 0, stream>>>(none, d_sqnorm, max_norm, d_norm);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace gs

using namespace gs;

extern "C" {

gs_status gs_grads_sqnorm(const gs_tensor *tensors, int64_t count, double *d_sqnorm, int accumulate, void *d_workspace,
                          size_t workspace_bytes, void *stream)
{
    if (!good_tensors(tensors, count, false)) return GS_ERR_INVALID_ARG;
    if (!d_sqnorm || (reinterpret_cast<uintptr_t>(d_sqnorm) & 7u)) return GS_ERR_INVALID_ARG;
    if (!d_workspace || workspace_bytes < gs_sqnorm_workspace_bytes() || (reinterpret_cast<uintptr_t>(d_workspace) & 7u)) return GS_ERR_WORKSPACE;
    const Range sq = range_of(d_sqnorm, 8, true), ws = range_of(d_workspace, (int64_t)workspace_bytes, true);
    if (touches(tensors, count, sq) || touches(tensors, count, ws) || overlap(sq, ws)) return GS_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    void *memory;
    if (!cut_long(tensors, count, memory)) return GS_ERR_NOMEM;
    const hipError_t e = (count <= TABLE_SMALL ? norm<TABLE_SMALL> : norm<TABLE_IN_PLACE>)(tensors, count, d_sqnorm, accumulate, d_workspace, st);
    free(memory);
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_grads_sqnorm launch");
}

gs_status gs_grads_clip(const gs_tensor *tensors, int64_t count, const double *d_sqnorm, float max_norm, float *d_norm, void *stream)
{
    if (!good_tensors(tensors, count, true)) return GS_ERR_INVALID_ARG;
    if (!d_sqnorm || (reinterpret_cast<uintptr_t>(d_sqnorm) & 7u) || (reinterpret_cast<uintptr_t>(d_norm) & 3u)) return GS_ERR_INVALID_ARG;
    if (!(max_norm > 0.0f)) return GS_ERR_INVALID_ARG;
    if (gs_status s = outputs_apart(tensors, count, d_sqnorm, d_norm); s != GS_OK) return s;
    hipStream_t st = static_cast<hipStream_t>(stream);
    void *memory;
    if (!cut_long(tensors, count, memory)) return GS_ERR_NOMEM;
    bool in_place = true;
    for (int64_t i = 0; i < count; ++i) in_place = in_place && (!tensors[i].out || tensors[i].out == tensors[i].data);
    const hipError_t e = (count <= TABLE_SMALL ? clip<TABLE_SMALL> : in_place ? clip<TABLE_IN_PLACE> : clip<TABLE>)(tensors, count, d_sqnorm, max_norm, d_norm, st);
    free(memory);
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_grads_clip launch");
}

}  // extern "C"
