// gs_tensors.hip -- norm and clip of gradients that are many tensors: a training program's list of parameters, where the
// other norms take one flat layer.
//
// One pass that reads every element (the norm) and one that reads and writes it (the clip): HBM-bound.  A launch takes a
// table of tensors in its arguments, so nothing is copied to the device first and nothing is kept from call to call; its workgroups
// are tiles of one tensor each, and find which by a look at the first tile of every tensor.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdlib>
#include <cstring>

#include "gs_device.h"
#include "gs_internal.h"

#pragma clang fp contract(off)

namespace gs {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int TENSOR_BLOCK = 256;
constexpr int TABLE = 120;             // tensors of one launch: 3848 of the 4096 bytes that a launch's arguments may have

struct Entry {
    const void *in;
    void *out;
    int64_t numel;
    uint32_t first;                    // its first tile, of this launch's
    int32_t dtype;
};
struct Table {
    int32_t count;
    uint32_t tile_vecs;                // 16-byte vectors of a tile
    Entry e[TABLE];
};

// The tensor that a tile belongs to: the last one whose first tile is not behind it.  Every lane looks at two of them.
__device__ __forceinline__ int tensor_of(const Table &t, uint32_t tile)
{
    const int lane = threadIdx.x & 63;
    const int a = __popcll(__ballot(lane < t.count && t.e[lane].first <= tile));
    const int b = __popcll(__ballot(lane + 64 < t.count && t.e[lane + 64 < TABLE ? lane + 64 : 0].first <= tile));
    return __builtin_amdgcn_readfirstlane(a + b - 1);
}

__device__ __forceinline__ void square(u32x4 q, bool bf16, double &x, double &y)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (bf16) {
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

// A tile's part of a tensor: whole aligned vectors [v0, v1) behind `head` single elements, and whether it has the single ones
// of both ends (the tensor's first tile does).
struct Part {
    int64_t v0, v1;
    int head, singles;
};
__device__ __forceinline__ Part part_of(const Table &t, const Entry &e, const void *aligned_for, bool vectors, uint32_t tile)
{
    const int size = e.dtype == GS_BF16 ? 2 : 4, per = 16 / size;
    Part p;
    const int64_t off = ((16 - (reinterpret_cast<uintptr_t>(aligned_for) & 15)) & 15) / size;
    const int64_t head = vectors ? (off < e.numel ? off : e.numel) : 0;
    const int64_t vecs = vectors ? (e.numel - head) / per : 0;
    p.head = (int)head;
    p.v0 = (int64_t)(tile - e.first) * t.tile_vecs;
    p.v1 = p.v0 + t.tile_vecs < vecs ? p.v0 + t.tile_vecs : vecs;
    p.singles = tile == e.first ? (int)(e.numel - vecs * per) : 0;
    return p;
}

__global__ __launch_bounds__(TENSOR_BLOCK) void k_tensors_sqnorm(Table t, double *partials)
{
    __shared__ double lds[TENSOR_BLOCK / 64];
    const Entry &e = t.e[tensor_of(t, blockIdx.x)];
    const Part p = part_of(t, e, e.in, true, blockIdx.x);
    const bool bf16 = e.dtype == GS_BF16;
    const int size = bf16 ? 2 : 4, per = 16 / size;
    const char *base = static_cast<const char *>(e.in);
    const u32x4 *v = reinterpret_cast<const u32x4 *>(base + p.head * size);
    double x = 0.0, y = 0.0;
    for (int64_t i = p.v0 + threadIdx.x; i < p.v1; i += TENSOR_BLOCK) square(v[i], bf16, x, y);
    if ((int)threadIdx.x < p.singles) {                // at most 14
        const int64_t vecs = (e.numel - p.head) / per, i = (int)threadIdx.x < p.head ? (int64_t)threadIdx.x : threadIdx.x + vecs * per;
        const double g = bf16 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(base)[i] << 16) : reinterpret_cast<const float *>(base)[i];
        x = fma(g, g, x);
    }
    const double s = block_sum<TENSOR_BLOCK>(x + y, lds);
    if (threadIdx.x == 0) partials[blockIdx.x] = s;
}

// Where the coefficient is 1, tensors that stay where they are are left alone.
__global__ __launch_bounds__(TENSOR_BLOCK) void k_tensors_clip(Table t, const double *d_sqnorm, float max_norm, float *d_norm)
{
    const double S = *d_sqnorm;
    if (d_norm && blockIdx.x == 0 && threadIdx.x == 0) *d_norm = (float)sqrt(S);
    if (t.count == 0) return;
    const float c = clip_from(S, max_norm);
    const Entry &e = t.e[tensor_of(t, blockIdx.x)];
    if (c == 1.0f && e.out == e.in) return;
    const bool bf16 = e.dtype == GS_BF16;
    const int size = bf16 ? 2 : 4, per = 16 / size;
    // without a common alignment, element by element
    const bool same = ((reinterpret_cast<uintptr_t>(e.in) ^ reinterpret_cast<uintptr_t>(e.out)) & 15) == 0;
    const char *in = static_cast<const char *>(e.in);
    char *out = static_cast<char *>(e.out);
    auto one = [&](int64_t i) {
        if (bf16) reinterpret_cast<uint16_t *>(out)[i] = (uint16_t)f32_to_bf16_bits(c * __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(in)[i] << 16));
        else reinterpret_cast<float *>(out)[i] = c * reinterpret_cast<const float *>(in)[i];
    };
    if (!same) {
        const int64_t a = (int64_t)(blockIdx.x - e.first) * t.tile_vecs * per, b = a + (int64_t)t.tile_vecs * per;
        for (int64_t i = a + threadIdx.x; i < b && i < e.numel; i += TENSOR_BLOCK) one(i);
        return;
    }
    const Part p = part_of(t, e, e.in, true, blockIdx.x);
    const u32x4 *vi = reinterpret_cast<const u32x4 *>(in + p.head * size);
    u32x4 *vo = reinterpret_cast<u32x4 *>(out + p.head * size);
    for (int64_t i = p.v0 + threadIdx.x; i < p.v1; i += TENSOR_BLOCK) {
        u32x4 q = vi[i];
#pragma unroll
        for (int w = 0; w < 4; ++w)
            q[w] = bf16 ? f32_to_bf16_bits(c * bf16_lo(q[w])) | f32_to_bf16_bits(c * bf16_hi(q[w])) << 16 : __float_as_uint(c * __uint_as_float(q[w]));
        vo[i] = q;
    }
    if ((int)threadIdx.x < p.singles) {
        const int64_t vecs = (e.numel - p.head) / per;
        one((int)threadIdx.x < p.head ? (int64_t)threadIdx.x : threadIdx.x + vecs * per);
    }
}

// ---- launchers --------------------------------------------------------------------------------
static int64_t size_of(const gs_tensor &t) { return t.dtype == GS_BF16 ? 2 : 4; }

// Vectors of a tile so that all tiles together leave no more partials than the workspace holds: every tensor may have one that
// is not full.
static uint32_t tile_vecs_for(const gs_tensor *tensors, int64_t count)
{
    int64_t vecs = 0;
    for (int64_t i = 0; i < count; ++i) vecs += tensors[i].numel / (16 / size_of(tensors[i])) + 1;
    uint32_t tile = TENSOR_BLOCK * 8;
    while (vecs / tile + count > GS_SQNORM_MAX_BLOCKS) tile *= 2;
    return tile;
}

// Calls launch(table, tiles) for tables that hold all tensors between them.
template <typename F>
static hipError_t for_tables(const gs_tensor *tensors, int64_t count, uint32_t tile_vecs, F launch)
{
    Table t;
    t.count = 0;
    t.tile_vecs = tile_vecs;
    uint32_t tiles = 0;
    for (int64_t i = 0; i < count; ++i) {
        const gs_tensor &x = tensors[i];
        if (x.numel == 0) continue;
        const int64_t per_tile = (int64_t)tile_vecs * (16 / size_of(x));
        t.e[t.count++] = {x.data, x.out ? x.out : const_cast<void *>(x.data), x.numel, tiles, x.dtype};
        tiles += (uint32_t)((x.numel + per_tile - 1) / per_tile);
        if (t.count == TABLE) {
            if (hipError_t e = launch(t, tiles); e != hipSuccess) return e;
            t.count = 0;
            tiles = 0;
        }
    }
    return t.count ? launch(t, tiles) : hipSuccess;
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

// Every output against every other array but its own input.  Sorted by address, an overlap shows between neighbours: each
// range is held against the furthest end so far, of the outputs and of all.
struct Range {
    uintptr_t lo, hi;
    bool out;
};
static gs_status outputs_apart(const gs_tensor *tensors, int64_t count)
{
    Range few[64], *r = few;
    if (count > 32 && !(r = static_cast<Range *>(malloc(sizeof(Range) * 2 * (size_t)count)))) return GS_ERR_NOMEM;
    size_t n = 0;
    for (int64_t i = 0; i < count; ++i) {
        const gs_tensor &t = tensors[i];
        if (t.numel == 0) continue;
        const uintptr_t bytes = (uintptr_t)(t.numel * size_of(t)), in = reinterpret_cast<uintptr_t>(t.data), out = reinterpret_cast<uintptr_t>(t.out);
        if (out && out != in) r[n++] = {in, in + bytes, false};
        r[n++] = {out ? out : in, (out ? out : in) + bytes, true};
    }
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

}  // namespace gs

using namespace gs;

extern "C" {

gs_status gs_grads_sqnorm(const gs_tensor *tensors, int64_t count, double *d_sqnorm, int accumulate, void *d_workspace,
                          size_t workspace_bytes, void *stream)
{
    if (!good_tensors(tensors, count, false)) return GS_ERR_INVALID_ARG;
    if (!d_sqnorm || (reinterpret_cast<uintptr_t>(d_sqnorm) & 7u)) return GS_ERR_INVALID_ARG;
    if (!d_workspace || workspace_bytes < gs_sqnorm_workspace_bytes() || (reinterpret_cast<uintptr_t>(d_workspace) & 7u)) return GS_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    double *partials = static_cast<double *>(d_workspace);
    int64_t done = 0;
    hipError_t e = for_tables(tensors, count, tile_vecs_for(tensors, count), [&](const Table &t, uint32_t tiles) {
        k_tensors_sqnorm<<<tiles, TENSOR_BLOCK, 0, st>>>(t, partials + done);
        done += tiles;
        return hipGetLastError();
    });
    if (e == hipSuccess && (done || !accumulate)) e = launch_fold(partials, GS_SQNORM_MAX_BLOCKS, (int)done, d_sqnorm, accumulate, st);
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_grads_sqnorm launch");
}

gs_status gs_grads_clip(const gs_tensor *tensors, int64_t count, const double *d_sqnorm, float max_norm, float *d_norm, void *stream)
{
    if (!good_tensors(tensors, count, true)) return GS_ERR_INVALID_ARG;
    if (!d_sqnorm || (reinterpret_cast<uintptr_t>(d_sqnorm) & 7u) || (reinterpret_cast<uintptr_t>(d_norm) & 3u)) return GS_ERR_INVALID_ARG;
    if (!(max_norm > 0.0f)) return GS_ERR_INVALID_ARG;
    if (gs_status s = outputs_apart(tensors, count); s != GS_OK) return s;
    hipStream_t st = static_cast<hipStream_t>(stream);
    float *norm = d_norm;
    hipError_t e = for_tables(tensors, count, tile_vecs_for(tensors, count), [&](const Table &t, uint32_t tiles) {
        k_tensors_clip<<<tiles, TENSOR_BLOCK, 0, st>>>(t, d_sqnorm, max_norm, norm);
        norm = nullptr;                // written by the first launch
        return hipGetLastError();
    });
    if (e == hipSuccess && norm) {     // nothing to scale, but a norm is asked for
        Table none;
        memset(&none, 0, sizeof none);
        k_tensors_clip<<<1, TENSOR_BLOCK, 0, st>>>(none, d_sqnorm, max_norm, norm);
        e = hipGetLastError();
    }
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_grads_clip launch");
}

}  // extern "C"
