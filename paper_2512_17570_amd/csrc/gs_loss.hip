// gs_loss.hip -- the losses that post-training takes its gradients from: token log-probabilities over rows of logits and
// their gradient, the clipped policy loss with a KL term, and the preference loss over pairs of sequences.
//
// All the work is one or two passes over rows of logits (2 or 4 bytes an element, one row a token, up to a few hundred
// thousand elements a row): read, and for a gradient written once, with one or two exponentials an element and no product of
// matrices, so HBM is the bound and there is no MFMA here.
//   * a row of up to 196608 bf16 (98304 fp32) elements is read once: it stays in its workgroup's registers (k_held)
//   * longer rows, and rows of which there are too few to fill the chip, go in parts (k_part), and a gradient reads them again (k_grad)
//   * the preference loss knows a token's gradient only when both sequences of its pair have been scored, so it reads twice
// Against what the same card copies (one 16-byte vector a lane, 6.7 TB/s) and only reads (7.1 TB/s): 16384 x 32000 bf16 scored at 7.0
// TB/s; policy loss with its gradient over 8192 x 131072 at 5.6 and 4095 x 50001 at 5.6 (a copy in the shape of k_held, a row held
// from its first load to its first store, 6.0 and 6.1); 2048 x 32003 fp32 at 5.5; gradients of known rows 6.2 to 6.5.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "gs_device.h"
#include "gs_internal.h"

#pragma clang fp contract(off)

namespace gs {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896340736f;

// ---- an element type: 16-byte vectors of it, to fp32 and back -------------------------------
struct Bf16 {
    typedef uint16_t T;
    static constexpr int PER = 8;
    static constexpr uint32_t LOWEST = 0xff80ff80u;   // -inf, twice
    // Maximum so far, two elements at a time as whole numbers.  Positive values are ordered as signed numbers, and lie above
    // negative ones; negative ones are ordered the other way round, which as unsigned numbers makes the largest the least.  One
    // operation an element where unpacked floats take one and a half.  NaN: either sign may be lost, the sum is NaN all the same.
    struct Max {
        i16x2 up = {-32768, -32768};
        u16x2 down = {65535, 65535};
        __device__ __forceinline__ void add(u32x4 q)
        {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                up = __builtin_elementwise_max(up, __builtin_bit_cast(i16x2, (uint32_t)q[i]));
                down = __builtin_elementwise_min(down, __builtin_bit_cast(u16x2, (uint32_t)q[i]));
            }
        }
        __device__ __forceinline__ float get() const
        {
            const int u = up[0] > up[1] ? up[0] : up[1];
            const uint32_t d = down[0] < down[1] ? down[0] : down[1];
            return __uint_as_float((u >= 0 ? (uint32_t)u : d) << 16);
        }
    };
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
    static constexpr uint32_t LOWEST = 0xff800000u;
    struct Max {
        float m = -INFINITY;
        __device__ __forceinline__ void add(u32x4 q)
        {
            // fmaxf would first make each element a quiet number
            asm("v_max3_f32 %0, %1, %2, %0" : "+v"(m) : "v"(q[0]), "v"(q[1]));
            asm("v_max3_f32 %0, %1, %2, %0" : "+v"(m) : "v"(q[2]), "v"(q[3]));
        }
        __device__ __forceinline__ float get() const { return m; }
    };
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

// Elements [0, n) of a row from an address of any alignment: `head` single ones, `vecs` whole aligned vectors, the rest
// single again.  Only what lies in the row is touched.
struct Cut {
    int head, vecs, singles;      // singles: those in front and behind together
    template <int PER> static __device__ __forceinline__ Cut of(const void *p, int n)
    {
        constexpr int SIZE = 16 / PER;
        Cut c;
        c.head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / SIZE);
        c.vecs = (n - c.head) / PER;
        c.singles = n - c.vecs * PER;
        return c;
    }
    // the element that single i is
    template <int PER> __device__ __forceinline__ int single(int i) const { return i < head ? i : i + vecs * PER; }
};
// whether two rows are cut in the same places
__device__ __forceinline__ bool common(const void *a, const void *b)
{
    return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15) == 0;
}
// vectors that a 128-byte line holds before this one
__device__ __forceinline__ int in_line(const void *v) { return (int)(reinterpret_cast<uintptr_t>(v) >> 4) & 7; }

// ---- what one token adds to the policy loss ---------------------------------------------------
struct Policy {
    float k;                      // log2(e) / temperature
    float it;                     // 1 / temperature
    float low, high, kl;          // bounds of the ratio, factor of the KL term
    const float *old_logp, *ref_logp, *advantages, *weights;
    Meeting meet;                 // of a launch with few rows
    float *stats;
    int accumulate;
};
struct Terms {
    float pg, kl, slope;          // slope: of pg + factor kl in logp
    bool clipped;
};
// what it takes besides the log-probability
struct Token {
    float old_logp, ref_logp, advantage;
};
__device__ __forceinline__ Token token_of(const Policy &P, int64_t r)
{
    return {P.old_logp[r], P.ref_logp ? P.ref_logp[r] : 0.0f, P.advantages[r]};
}
__device__ __forceinline__ Terms policy_terms(float logp, const Token &k, const Policy &P)
{
    Terms t;
    const float a = k.advantage, x = logp - k.old_logp, ratio = expf(x), held = fminf(fmaxf(ratio, P.low), P.high) * a;
    float plain = ratio * a;
    // too large for 32 bits, which its product with no advantage or a tiny one is not
    const bool beyond = ratio == INFINITY && x < INFINITY;
    if (__builtin_expect(__ballot(beyond) != 0, 0)) {
        const float root = expf(0.25f * fminf(x, 300.0f));
        plain = beyond ? a * root * root * root * root : plain;
    }
    t.clipped = held < plain;     // NaN: the plain product, which then is one
    t.pg = -(t.clipped ? held : plain);
    t.slope = t.clipped ? 0.0f : -plain;
    t.kl = 0.0f;
    if (P.ref_logp) {
        const float d = k.ref_logp - logp, em1 = expm1f(d);      // exp(d) - 1 without cancellation: d is small in earnest
        t.kl = em1 - d;
        if (P.kl != 0.0f) t.slope += P.kl * -em1;
    }
    return t;
}
__device__ __forceinline__ float weight_of(const float *weights, int64_t r) { return weights ? weights[r] : 1.0f; }

struct Logits {
    const void *x;
    int64_t stride;
    const int64_t *targets;
    int vocab;
};
__device__ __forceinline__ int target_of(const Logits &L, int64_t r)
{
    const int64_t t = L.targets[r];
    return t >= 0 && t < L.vocab ? (int)t : -1;
}

// What a row adds to the four sums of the policy loss.
struct Sums {
    double x[4];
};
__device__ __forceinline__ Sums sums_of(const Terms &e, float w, float kl_coef)
{
    const double pg = (double)w * e.pg, kl = (double)w * e.kl;
    return {{kl_coef != 0.0f ? pg + kl_coef * kl : pg, pg, kl, e.clipped ? (double)w : 0.0}};
}
// One row's, by a wave: the policy and the KL term in 64 bits each, as the sums of many rows are held, and a weight as it is.  Their sum with
// the KL term's factor is made of the sums: every workgroup looks at all words that are there, of which these are five.
__device__ __forceinline__ void leave_sums(const Meeting &M, int64_t r, const Sums &s, uint32_t (&w)[5])
{
    halves(s.x[1], w[0], w[1]);
    halves(s.x[2], w[2], w[3]);
    w[4] = __float_as_uint((float)s.x[3]);
    if ((threadIdx.x & 63) == 0) leave(M, (int)r, w);
}
__device__ __forceinline__ void finish_policy(const Meeting &M, uint32_t (&w)[5], const Policy &P)
{
    if (!last_of(M, !P.accumulate, w)) return;
    double pg = 0.0, kl = 0.0, clipped = 0.0;
    auto add = [&] {                                       // 0 without a slot
        pg += __hiloint2double((int)w[1], (int)w[0]);
        kl += __hiloint2double((int)w[3], (int)w[2]);
        clipped += __uint_as_float(w[4]);
    };
    add();
#pragma unroll 1
    for (int i = (threadIdx.x & 63) + 64; i < M.n; i += 64) {
        left_words(M, i, w);
        add();
    }
    pg = wave_sum(pg), kl = wave_sum(kl), clipped = wave_sum(clipped);
    if ((threadIdx.x & 63) == 63) {
        const double x[4] = {P.kl != 0.0f ? pg + P.kl * kl : pg, pg, kl, clipped};
#pragma unroll
        for (int q = 0; q < 4; ++q) P.stats[q] = (float)((P.accumulate ? (double)P.stats[q] : 0.0) + x[q]);
    }
    clear<5>(M);
}

// +0 over a row
template <typename E, int BLOCK>
__device__ __forceinline__ void zero_row(typename E::T *out, int n)
{
    const Cut c = Cut::of<E::PER>(out, n);
    u32x4 *v = reinterpret_cast<u32x4 *>(out + c.head);
    for (int i = threadIdx.x; i < c.vecs; i += BLOCK) __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, v + i);
    for (int i = threadIdx.x; i < c.singles; i += BLOCK) out[c.single<E::PER>(i)] = 0;
}

// Gradient over elements [from, to) of a row one by one, for an output that has no vectors in common with the row:
// d ([i = t] - exp2(k (z - m)) / s)
template <typename E, int BLOCK>
__device__ __forceinline__ void grad_singly(const typename E::T *row, typename E::T *out, int from, int to, int t, float m, float s, float k, float d)
{
    for (int i = from + threadIdx.x; i < to; i += BLOCK) {
        const float p = __builtin_amdgcn_exp2f((E::load(row + i) - m) * k) / s;
        E::store(out + i, i == t ? d * (1.0f - p) : -d * p);
    }
}

// ---- rows held in registers -------------------------------------------------------------------
// One workgroup a row, which is read once: its lanes keep NV vectors each, from the first maximum to the gradient.  The first LO vectors of a lane lie in the row whatever its length; the rest may not, and are -inf.
//
// A wave takes its exponentials from a maximum of its own, as soon as its vectors are there, and waits for the others once, for the
// row's maximum and sum; its gradient is then f exp2((m_wave - m) k) times those exponentials.  Of the first KEEP vectors the
// exponentials stay (four bytes an element), of the others the logits (two in bf16), and the exponential is taken again: 8192 x 131072,
// of 16 vectors none / 5 / 8 kept 0.80/0.78/0.77 ms (with a maximum of the whole row first, and all taken again, 0.89).
// A longer row leaves room for one workgroup on a CU, whose reading and writing then take turns; other CUs' fill the gaps.  Loads and
// stores carry the non-temporal hint: written through as well, or without the hint, they lose 1-3 and 2-8 %, loads without it 12 % where
// nothing is written.  Vectors are counted from a line's start: with rows that start anywhere (50001) 0.143 ms against 0.151.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float from_dpp(float x, float none)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
template <bool MAX>
__device__ __forceinline__ float join(float x, float y)
{
    if constexpr (MAX) return fmaxf(x, y);
    else return x + y;
}
// over 16 lanes, in all of them
template <bool MAX>
__device__ __forceinline__ float row_join(float x)
{
    x = join<MAX>(x, from_dpp<0xb1>(x, x));
    x = join<MAX>(x, from_dpp<0x4e>(x, x));
    x = join<MAX>(x, from_dpp<0x141>(x, x));
    return join<MAX>(x, from_dpp<0x140>(x, x));
}
__device__ __forceinline__ float of_lane(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }
template <bool MAX>
__device__ __forceinline__ float wave_join(float x)
{
    constexpr float none = MAX ? -INFINITY : 0.0f;
    x = row_join<MAX>(x);
    x = join<MAX>(x, from_dpp<0x142, 0xa>(x, none));
    x = join<MAX>(x, from_dpp<0x143, 0xc>(x, none));
    return of_lane(x, 63);
}

// exp2(k z - c) in place of exp2(k (z - m)): one rounding and one operation.  c is k m rounded, and `off` what the rounding took
// (k m - c, exact), by which all exponentials are too large together.  Where it could be more than 64, so that |k m| is over 2^31, logits
// that are not m itself lie so far below it that they count nothing: any k that keeps them there will do, and a power of two has no rounding.
struct Shift {
    float k, c, off;
    __device__ __forceinline__ static Shift from(float m, float k)
    {
        const float base = m == -INFINITY ? 0.0f : m, a = fabsf(base);          // nothing but -inf: all exponentials 0
        Shift s;
        s.k = a * k < 0x1p31f ? k : a < 0x1p80f ? 0x1p40f : 0x1p-20f;
        s.c = base * s.k;
        s.off = fmaf(base, s.k, -s.c);
        return s;
    }
    __device__ __forceinline__ float power(float z) const { return __builtin_amdgcn_exp2f(fmaf(z, k, -c)); }
};

template <typename E, int BLOCK, int NV, int LO, int KEEP, bool POLICY>
__global__ __launch_bounds__(BLOCK) void k_held(Logits L, int64_t row0, int64_t keep_row, Policy P, float *logp, float *row_stats, void *dlogits, int64_t dstride)
{
    typedef typename E::T T;
    constexpr int PER = E::PER, NW = BLOCK / 64;
    __shared__ float lds_m[NW], lds_s[NW];
    const int64_t r = row0 + blockIdx.x;
    const int t = target_of(L, r);
    const float w = POLICY ? weight_of(P.weights, r) : 1.0f;
    T *out = POLICY && dlogits ? static_cast<T *>(dlogits) + r * dstride : nullptr;
    const bool meets = POLICY && P.meet.n > 0;
    auto no_token = [&] {
        if (threadIdx.x == 0) {
            logp[r] = 0.0f;
            if (row_stats) row_stats[2 * r] = 0.0f, row_stats[2 * r + 1] = 1.0f;
        }
        if (meets && threadIdx.x >= BLOCK - 64) {
            uint32_t words[5];
            leave_sums(P.meet, r, Sums{}, words);
            finish_policy(P.meet, words, P);
        }
        if (out) zero_row<E, BLOCK>(out, L.vocab);
    };
    if (t < 0 || w == 0.0f) return no_token();
    Token token = {};
    if constexpr (POLICY) token = token_of(P, r);
    const T *row = static_cast<const T *>(L.x) + r * L.stride;
    const Cut c = Cut::of<PER>(row, L.vocab);
    // vectors counted from the start of the first one's 128-byte line, so that a wave's accesses are whole lines
    const int skip = in_line(row + c.head), end = skip + c.vecs;
    const u32x4 *v = reinterpret_cast<const u32x4 *>(row + c.head) - skip;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    auto inside = [&](int j) {         // whether the lane's vector j is the row's
        const int i = j * BLOCK + (int)threadIdx.x;
        return (j > 0 || i >= skip) && (j < LO || i < end);
    };
    u32x4 q[NV];
    auto load = [&](auto keep) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (j == 0 || j >= LO) q[j] = u32x4{E::LOWEST, E::LOWEST, E::LOWEST, E::LOWEST};
            if (inside(j)) q[j] = decltype(keep)::value ? v[j * BLOCK + threadIdx.x] : __builtin_nontemporal_load(v + j * BLOCK + threadIdx.x);
        }
    };
    if (!POLICY && r >= keep_row) load(std::true_type{});
    else load(std::false_type{});
    const int single = (int)threadIdx.x < c.singles ? c.single<PER>(threadIdx.x) : -1;
    const float zs = single >= 0 ? E::load(row + single) : -INFINITY;
    const float zt = E::load(row + t);
    auto used = [&](int j) { return j < LO || j * BLOCK + wave * 64 < end; };      // by any lane of the wave

    typename E::Max most;
#pragma unroll
    for (int j = 0; j < NV; ++j) most.add(q[j]);
    const float mw = wave_join<true>(fmaxf(most.get(), zs));
    const Shift shift = Shift::from(mw, P.k);
    const float es = shift.power(zs);
    float e[KEEP > 0 ? KEEP : 1][PER], sum[4] = {es, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (used(j)) {
            float z[PER];
            E::widen(q[j], z);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float x = shift.power(z[i]);
                sum[i & 3] += x;
                if (POLICY && j < KEEP) e[j < KEEP ? j : 0][i] = x;
            }
        }
    float m = mw, s = wave_join<false>((sum[0] + sum[1]) + (sum[2] + sum[3])) * __builtin_amdgcn_exp2f(-shift.off);
    if constexpr (NW > 1) {
        const int lane = threadIdx.x & 63;
        if (lane == 0) lds_m[wave] = m, lds_s[wave] = s;
        asm volatile("" ::"v"(zt));        // is there before another wave may store in its place
        __syncthreads();
        const float ml = lane < NW ? lds_m[lane] : -INFINITY, sl = lane < NW ? lds_s[lane] : 0.0f;
        m = of_lane(row_join<true>(ml), 0);
        s = of_lane(row_join<false>(lane < NW ? sl * __builtin_amdgcn_exp2f((ml - m) * P.k) : 0.0f), 0);
    }
    const float lp = (zt - m) * P.it - logf(s);
    if (threadIdx.x == 0) {
        logp[r] = lp;
        if (row_stats) row_stats[2 * r] = m, row_stats[2 * r + 1] = s;
    }
    if constexpr (POLICY) {
        const Terms terms = policy_terms(lp, token, P);
        // by the last wave, which has the fewest vectors
        uint32_t words[5] = {};
        if (meets && wave == NW - 1) leave_sums(P.meet, r, sums_of(terms, w, P.kl), words);
        const float d = w * terms.slope * P.it;
        if (!out) {
        } else if (d == 0.0f) {
            zero_row<E, BLOCK>(out, L.vocab);
        } else if (!common(row, out)) {
            grad_singly<E, BLOCK>(row, out, 0, L.vocab, t, m, s, P.k, d);       // reads the row again
        } else {
            const float f = -d / s * __builtin_amdgcn_exp2f((mw - m) * P.k - shift.off);
            u32x4 *vo = reinterpret_cast<u32x4 *>(out + c.head) - skip;
#pragma unroll
            for (int j = KEEP; j < NV; ++j) asm volatile("" : "+v"(q[j]));       // what was made of them is not kept
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (used(j)) {
                    float z[PER];
                    E::widen(q[j], z);
#pragma unroll
                    for (int i = 0; i < PER; ++i) z[i] = f * (j < KEEP ? e[j < KEEP ? j : 0][i] : shift.power(z[i]));
                    if (inside(j)) __builtin_nontemporal_store(E::narrow(z), vo + j * BLOCK + threadIdx.x);
                }
            if (single >= 0) E::store(out + single, f * es);
            // the token's own element a second time, by the lane that has just stored it
            const int at = t - c.head;
            if (at >= 0 && at < c.vecs * PER ? (at / PER + skip) % BLOCK == (int)threadIdx.x : single == t)
                E::store(out + t, d * (1.0f - __builtin_amdgcn_exp2f((zt - m) * P.k) / s));
        }
        if (meets && wave == NW - 1) finish_policy(P.meet, words, P);
    }
}

// ---- rows in parts ----------------------------------------------------------------------------
// Rows too long to be held, and rows of which there are too few to fill the chip: parts of PART_MIN elements or more, a
// workgroup each, leave a maximum and a sum, and what comes after joins those of a row, one to a lane.
constexpr int PART_BLOCK = 256;
constexpr int PART_MIN = 8192;
constexpr int PARTS = 64;
constexpr int HELD_MAX = 24 * 1024;          // vectors of the longest row that is held

struct MaxSum {
    float m, s;
};
// The row's maximum and sum from those of its parts, one in each lane.  A row of nothing but -inf has a sum of 0 here, from which all
// is NaN as well.
__device__ __forceinline__ MaxSum join_parts(MaxSum a, float k)
{
    const float m = wave_join<true>(a.m), base = m == -INFINITY ? 0.0f : m;
    return {m, wave_join<false>(a.s * __builtin_amdgcn_exp2f((a.m - base) * k))};
}

// The part's maximum and its sum of exp2(k (z - maximum)).  Lines may stay in the caches for the gradient, which reads them again: they do
// while a launch's rows are fewer than the memory-side cache holds, of more none is left by then (4096 x 128256 fp32 0.99 ms, 6.3 GB at 6.4 TB/s).
// A row has one entry more than parts: the token's own logit, which a gradient written in place would not leave for the others to read.
//   FINISH: the last of a row's workgroups also joins them, for a log-probability with no gradient after it
struct Finish {
    Meeting meet;
    float it;
    float *logp, *row_stats;
    bool once;                    // more than the caches hold, and not read again
};
template <typename E, bool FINISH>
__global__ __launch_bounds__(PART_BLOCK) void k_part(Logits L, int64_t row0, int parts, int len, float k, const float *weights, MaxSum *partials, Finish F)
{
    constexpr int NV = PART_MIN / PART_BLOCK / E::PER, NW = PART_BLOCK / 64;
    __shared__ float lds_m[NW], lds_s[NW];
    const uint32_t which = blockIdx.x / (uint32_t)parts, part = blockIdx.x - which * (uint32_t)parts;
    const int64_t r = row0 + which;
    const int t = target_of(L, r);
    if (t < 0 || weight_of(weights, r) == 0.0f) {
        if (FINISH && part == 0 && threadIdx.x == 0) {
            F.logp[r] = 0.0f;
            if (F.row_stats) F.row_stats[2 * r] = 0.0f, F.row_stats[2 * r + 1] = 1.0f;
        }
        return;
    }
    const int from = (int)part * len, n = min(len, L.vocab - from);
    const typename E::T *row = static_cast<const typename E::T *>(L.x) + r * L.stride + from;
    const Cut c = Cut::of<E::PER>(row, n);
    const u32x4 *v = reinterpret_cast<const u32x4 *>(row + c.head);
    const float zs = (int)threadIdx.x < c.singles ? E::load(row + c.single<E::PER>(threadIdx.x)) : -INFINITY;
    float m = -INFINITY, s = 0.0f;
    for (int i0 = 0; i0 == 0 || i0 < c.vecs; i0 += NV * PART_BLOCK) {
        u32x4 q[NV];
        auto load = [&](auto keep) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int i = i0 + j * PART_BLOCK + (int)threadIdx.x;
                q[j] = u32x4{E::LOWEST, E::LOWEST, E::LOWEST, E::LOWEST};
                if (i < c.vecs) q[j] = decltype(keep)::value ? v[i] : __builtin_nontemporal_load(v + i);
            }
        };
        if (FINISH && F.once) load(std::false_type{});
        else load(std::true_type{});
        typename E::Max most;
#pragma unroll
        for (int j = 0; j < NV; ++j) most.add(q[j]);
        const float extra = i0 == 0 ? zs : -INFINITY, mi = wave_join<true>(fmaxf(most.get(), extra));
        const Shift shift = Shift::from(mi, k);
        float sum[4] = {shift.power(extra), 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float z[E::PER];
            E::widen(q[j], z);
#pragma unroll
            for (int e = 0; e < E::PER; ++e) sum[e & 3] += shift.power(z[e]);
        }
        const float si = wave_join<false>((sum[0] + sum[1]) + (sum[2] + sum[3])) * __builtin_amdgcn_exp2f(-shift.off);
        const float both = fmaxf(m, mi), base = both == -INFINITY ? 0.0f : both;
        s = s * __builtin_amdgcn_exp2f((m - base) * k) + si * __builtin_amdgcn_exp2f((mi - base) * k);
        m = both;
    }
    if ((threadIdx.x & 63) == 0) lds_m[threadIdx.x >> 6] = m, lds_s[threadIdx.x >> 6] = s;
    __syncthreads();
    const int lane = threadIdx.x & 63;
    const float ml = lane < NW ? lds_m[lane] : -INFINITY, sl = lane < NW ? lds_s[lane] : 0.0f;
    m = of_lane(row_join<true>(ml), 0);
    const float base = m == -INFINITY ? 0.0f : m;
    s = of_lane(row_join<false>(lane < NW ? sl * __builtin_amdgcn_exp2f((ml - base) * k) : 0.0f), 0);
    if constexpr (FINISH) {
        if (threadIdx.x >= 64) return;
        F.meet.slots += (int64_t)which * parts * 2;
        uint32_t w[2] = {__float_as_uint(m), __float_as_uint(s)};
        if (threadIdx.x == 0) leave(F.meet, (int)part, w);
        const float zt = E::load(row + t - from);
        if (!last_of(F.meet, true, w)) return;
        const MaxSum a = join_parts({lane < parts ? __uint_as_float(w[0]) : -INFINITY, __uint_as_float(w[1])}, k);
        if (lane == 0) {
            F.logp[r] = (zt - a.m) * F.it - logf(a.s);
            if (F.row_stats) F.row_stats[2 * r] = a.m, F.row_stats[2 * r + 1] = a.s;
        }
        clear<2>(F.meet);
    } else if (threadIdx.x == 0) {
        partials += (int64_t)which * (parts + 1);
        partials[part] = {m, s == s ? s : NAN};              // a NaN of a logit's bits could be taken for a tag
        if (t >= from && t < from + n) partials[parts].m = E::load(row + t - from);
    }
}

__device__ __forceinline__ MaxSum joined(const MaxSum *partials, int parts, float k)
{
    const int lane = threadIdx.x & 63;
    return join_parts(lane < parts ? partials[lane] : MaxSum{-INFINITY, 0.0f}, k);
}

// Log-probabilities of rows in parts whose gradient is not asked for, a wave each.
__global__ __launch_bounds__(PART_BLOCK) void k_join(Logits L, int64_t row0, int rows, int parts, float k, float it, const float *weights,
                                                     const MaxSum *partials, float *logp)
{
    const int which = (int)blockIdx.x * (PART_BLOCK / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (which >= rows) return;
    const int64_t r = row0 + which;
    const int t = target_of(L, r);
    float lp = 0.0f;
    if (t >= 0 && weight_of(weights, r) != 0.0f) {
        partials += (int64_t)which * (parts + 1);
        const MaxSum a = joined(partials, parts, k);
        lp = (partials[parts].m - a.m) * it - logf(a.s);
    }
    if ((threadIdx.x & 63) == 0) logp[r] = lp;
}

// ---- gradient of rows whose maximum and sum are known -------------------------------------------
// A workgroup takes a run of GRAD_VECS vectors of a row, counted from the start of the row's first line; the first one has the single elements
// too.  Two vectors a lane, written through: 8192 x 131072 bf16 0.683 ms (6.3 TB/s) against 0.718 without, 0.718 with one and 0.740 with
// four; rows of 2000 0.59 against 1.09 with one.
// FROM_PARTS: maximum and sum come from a row's parts, and its policy loss is worked out here; else they and the loss's gradient in logp
// are given, and the rows are taken from the last one on: the end of what was read before is still in the memory-side cache.
constexpr int GRAD_BLOCK = 256;
constexpr int GRAD_NV = 2;
constexpr int GRAD_VECS = GRAD_BLOCK * GRAD_NV;
struct GradArgs {
    Logits L;
    int64_t row0, rows, dstride;
    Policy P;
    const float *row_stats, *dlogp;
    const MaxSum *partials;
    float *logp;
    void *dlogits;
    uint32_t runs;
    int parts;
};
template <typename E, bool FROM_PARTS>
__global__ __launch_bounds__(GRAD_BLOCK) void k_grad(GradArgs A)
{
    typedef typename E::T T;
    constexpr int PER = E::PER;
    const uint32_t which = blockIdx.x / A.runs, run = blockIdx.x - which * A.runs;
    const int64_t r = A.row0 + (FROM_PARTS ? (int64_t)which : A.rows - 1 - which);
    const Logits &L = A.L;
    const int t = target_of(L, r);
    const T *row = static_cast<const T *>(L.x) + r * L.stride;
    T *out = static_cast<T *>(A.dlogits) + r * A.dstride;
    float d = 0.0f;
    MaxSum a = {0.0f, 1.0f};
    if constexpr (FROM_PARTS) {
        const float w = weight_of(A.P.weights, r);
        float lp = 0.0f;
        Sums sums = {};
        if (t >= 0 && w != 0.0f) {
            const Token token = token_of(A.P, r);
            const MaxSum *partials = A.partials + (int64_t)which * (A.parts + 1);
            a = joined(partials, A.parts, A.P.k);
            lp = (partials[A.parts].m - a.m) * A.P.it - logf(a.s);
            const Terms terms = policy_terms(lp, token, A.P);
            sums = sums_of(terms, w, A.P.kl);
            d = w * terms.slope * A.P.it;
        }
        if (run == 0 && threadIdx.x < 64) {
            if (threadIdx.x == 0) A.logp[r] = lp;
            if (A.P.meet.n > 0) {
                uint32_t words[5];
                leave_sums(A.P.meet, r, sums, words);
                finish_policy(A.P.meet, words, A.P);
            }
        }
    } else if (t >= 0) {
        d = A.dlogp[r] * A.P.it;
        a = {A.row_stats[2 * r], A.row_stats[2 * r + 1]};
    }
    const bool vectors = d == 0.0f || common(row, out);
    const Cut c = Cut::of<PER>(d == 0.0f ? out : row, L.vocab);
    const int skip = in_line((d == 0.0f ? out : row) + c.head), end = skip + c.vecs;
    const int i0 = (int)run * GRAD_VECS + (int)threadIdx.x;
    u32x4 *vo = reinterpret_cast<u32x4 *>(out + c.head) - skip;
    const int single = run == 0 && (int)threadIdx.x < c.singles ? c.single<PER>(threadIdx.x) : -1;
    if (d == 0.0f) {
#pragma unroll
        for (int j = 0; j < GRAD_NV; ++j)
            if (i0 + j * GRAD_BLOCK >= skip && i0 + j * GRAD_BLOCK < end) __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, vo + i0 + j * GRAD_BLOCK);
        if (single >= 0) out[single] = 0;
        return;
    }
    if (!vectors) {
        const int from = (int)run * GRAD_VECS * PER;
        return grad_singly<E, GRAD_BLOCK>(row, out, from, min(from + GRAD_VECS * PER, L.vocab), t, a.m, a.s, A.P.k, d);
    }
    const u32x4 *v = reinterpret_cast<const u32x4 *>(row + c.head) - skip;
    u32x4 q[GRAD_NV];
#pragma unroll
    for (int j = 0; j < GRAD_NV; ++j)
        if (i0 + j * GRAD_BLOCK >= skip && i0 + j * GRAD_BLOCK < end) q[j] = __builtin_nontemporal_load(v + i0 + j * GRAD_BLOCK);
    const Shift shift = Shift::from(a.m, A.P.k);
    const float f = -d / a.s * __builtin_amdgcn_exp2f(-shift.off);
    const int at = t - c.head + skip * PER;                  // as an element of the vectors
#pragma unroll
    for (int j = 0; j < GRAD_NV; ++j) {
        const int i = i0 + j * GRAD_BLOCK;
        if (i < skip || i >= end) continue;
        float z[PER];
        E::widen(q[j], z);
        const int rel = at - i * PER;
        if (rel >= 0 && rel < PER) {                         // the lane with the token's own element
            const float zt = E::load(row + t);
#pragma unroll
            for (int e = 0; e < PER; ++e) z[e] = f * shift.power(z[e]);
#pragma unroll
            for (int e = 0; e < PER; ++e) z[e] = e == rel ? d * (1.0f - __builtin_amdgcn_exp2f((zt - a.m) * A.P.k) / a.s) : z[e];
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e) z[e] = f * shift.power(z[e]);
        }
        store_through(vo + i, E::narrow(z));
    }
    if (single >= 0) {
        const float p = __builtin_amdgcn_exp2f((E::load(row + single) - a.m) * A.P.k) / a.s;
        E::store(out + single, single == t ? d * (1.0f - p) : -d * p);
    }
}

// ---- sums over tokens -------------------------------------------------------------------------
constexpr int SUM_BLOCK = 512;
// N sums of every workgroup, added up by the last of them
template <int N, typename T>
__device__ __forceinline__ void finish_sums(double (&x)[N], const Meeting &M, T *out, int accumulate)
{
    constexpr int NW = SUM_BLOCK / 64;
    __shared__ double lds[N][NW];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int q = 0; q < N; ++q) {
        x[q] = wave_sum(x[q]);
        if (lane == 63) lds[q][wave] = x[q];
    }
    __syncthreads();
    if (wave > 0) return;
    uint32_t w[2 * N];
#pragma unroll
    for (int q = 0; q < N; ++q) halves(row_sum(lane < NW ? lds[q][lane] : 0.0), w[2 * q], w[2 * q + 1]);
    if (threadIdx.x == 0) leave(M, (int)blockIdx.x, w);
    if (!last_of(M, !accumulate, w)) return;
    left_sums(M, w, x);
    if (threadIdx.x == 63)
#pragma unroll
        for (int q = 0; q < N; ++q) out[q] = (T)((accumulate ? (double)out[q] : 0.0) + x[q]);
    clear<2 * N>(M);
}

__global__ __launch_bounds__(SUM_BLOCK) void k_policy_sums(const int64_t *targets, int vocab, int64_t rows, Policy P, const float *logp)
{
    double x[4] = {};
    for (int64_t r = (int64_t)blockIdx.x * SUM_BLOCK + threadIdx.x; r < rows; r += (int64_t)P.meet.n * SUM_BLOCK) {
        // all loads together; what a token without weight holds is not added
        const float w = weight_of(P.weights, r), lp = logp[r];
        const int64_t t = targets[r];
        const Token token = token_of(P, r);
        const bool counts = t >= 0 && t < vocab && w != 0.0f;
        const Sums e = sums_of(policy_terms(lp, token, P), w, P.kl);
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] += counts ? e.x[q] : 0.0;
    }
    finish_sums(x, P.meet, P.stats, P.accumulate);
}

// ---- preference loss --------------------------------------------------------------------------
constexpr int PAIR_BLOCK = 512;
struct Pairs {
    const float *logp, *ref_logp, *weights;
    const int64_t *offsets;
    int64_t tokens, pairs;
    float beta, smoothing, scale;
    float *margins, *dlogp;
    Meeting meet;                 // of a launch with few pairs; of one with many its slots are where the margins go in 64 bits, for the loss
    float *loss;
    int accumulate, ends;         // ends: bit 0 in the launch that has the first pair, bit 1 in that of the last
};
__device__ __forceinline__ int64_t offset_of(const Pairs &A, int64_t s)
{
    const int64_t o = A.offsets[s];
    return o < 0 ? 0 : o > A.tokens ? A.tokens : o;
}
__device__ __forceinline__ double log_ratio_sum(const Pairs &A, int64_t from, int64_t to)
{
    double x = 0.0;
    for (int64_t i = from + threadIdx.x; i < to; i += PAIR_BLOCK) {
        const float w = weight_of(A.weights, i), lp = A.logp[i], ref = A.ref_logp ? A.ref_logp[i] : 0.0f;
        x += w != 0.0f ? (double)w * ((double)lp - (double)ref) : 0.0;
    }
    return x;
}
__device__ __forceinline__ void spread(const Pairs &A, int64_t from, int64_t to, float d)
{
    for (int64_t i = from + threadIdx.x; i < to; i += PAIR_BLOCK) {
        const float w = weight_of(A.weights, i);
        A.dlogp[i] = w != 0.0f ? d * w : 0.0f;
    }
}
// Of a margin h, in 64 bits: loss and slope from one exponential, which is never over 1.
struct PairLoss {
    double h, t;                  // exp(-|h|)
    __device__ __forceinline__ explicit PairLoss(double margin) : h(margin), t(exp(-fabs(margin))) {}
    // e sigmoid(h) - (1 - e) sigmoid(-h)
    __device__ __forceinline__ double slope(double e) const
    {
        const double inv = 1.0 / (1.0 + t), up = h > 0.0 ? inv : t * inv, down = h > 0.0 ? t * inv : inv;
        return e * up - (1.0 - e) * down;
    }
    // -(1 - e) ln sigmoid(h) - e ln sigmoid(-h)
    __device__ __forceinline__ double loss(double e) const
    {
        const double ln = log1p(t);
        return (1.0 - e) * (fmax(-h, 0.0) + ln) + (e != 0.0 ? e * (fmax(h, 0.0) + ln) : 0.0);
    }
};

// One workgroup a pair: 4 to 6 us up to some hundred pairs, a chain of loads, a reduction and two functions in 64 bits (10 000 pairs 30 us).  Both sums are held
// in 64 bits: a margin is a small difference of sums over thousands of tokens.
__global__ __launch_bounds__(PAIR_BLOCK) void k_pairs(Pairs A)
{
    constexpr int NW = PAIR_BLOCK / 64;
    __shared__ double lds[2][NW];
    const int64_t p = blockIdx.x, q = A.pairs + p;
    const int64_t a0 = offset_of(A, p), a1 = offset_of(A, p + 1), b0 = offset_of(A, q), b1 = offset_of(A, q + 1);
    const double mine[2] = {wave_sum(log_ratio_sum(A, a0, a1)), wave_sum(log_ratio_sum(A, b0, b1))};
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (lane == 63) lds[0][wave] = mine[0], lds[1][wave] = mine[1];
    __syncthreads();
    // every wave works out the pair's slope for itself
    const double chosen = row_sum(lane < NW ? lds[0][lane] : 0.0), rejected = row_sum(lane < NW ? lds[1][lane] : 0.0);
    const PairLoss pair((double)A.beta * (chosen - rejected));
    const float slope = of_lane((float)((double)A.scale * A.beta * pair.slope(A.smoothing)), 0);
    if (A.meet.n == 0) {
        if (threadIdx.x == 0) reinterpret_cast<double *>(A.meet.slots)[p] = pair.h;
    } else if (wave == 0) {
        if (threadIdx.x == 0) A.margins[p] = (float)pair.h;
        uint32_t w[2];
        halves((double)A.scale * pair.loss(A.smoothing), w[0], w[1]);
        if (threadIdx.x == 0) leave(A.meet, (int)p, w);
        if (last_of(A.meet, !A.accumulate, w)) {
            double x[1];
            left_sums(A.meet, w, x);
            if (threadIdx.x == 63) *A.loss = (float)((A.accumulate ? (double)*A.loss : 0.0) + x[0]);
            clear<2>(A.meet);
        }
    }
    spread(A, a0, a1, slope);
    spread(A, b0, b1, -slope);
    if (p == 0 && (A.ends & 1)) spread(A, 0, a0, 0.0f);
    if (p + 1 == gridDim.x && (A.ends & 2)) spread(A, b1, A.tokens, 0.0f);
}
// Many pairs: what is left of a launch's, from their margins in 64 bits.  The loss takes them as they are: rounded to 32 bits a margin is off by
// 2^-24 of itself, the loss of a well separated pair by h times that.  The margins go out here, whole lines at a time: 100 000 pairs 256 us
// against 281 with a second store of a few bytes in k_pairs.  `before`: the loss of the launches in front.
template <typename T>
__global__ __launch_bounds__(SUM_BLOCK) void k_pair_sums(const double *wide, float *margins, int count, float smoothing, float scale, Meeting meet,
                                                         const double *before, T *out, int accumulate)
{
    double x[1] = {before && blockIdx.x == 0 && threadIdx.x == 0 ? *before : 0.0};
    for (int i = (int)blockIdx.x * SUM_BLOCK + (int)threadIdx.x; i < count; i += meet.n * SUM_BLOCK) {
        const double h = wide[i];
        margins[i] = (float)h;
        x[0] += (double)scale * PairLoss(h).loss(smoothing);
    }
    finish_sums(x, meet, out, accumulate);
}
__global__ __launch_bounds__(SUM_BLOCK) void k_zero(float *p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * SUM_BLOCK + threadIdx.x; i < n; i += (int64_t)gridDim.x * SUM_BLOCK) p[i] = 0.0f;
}

// ---- launchers --------------------------------------------------------------------------------
// Workgroups that meet with more work behind them than a sum: each looks at the words of all.  Policy loss, 64 / 100 / 128 rows of 8000 bf16
// 5.8/6.1/6.3 us, with a launch of its own for the sums 6.7/6.9/7.1; of 32000 8.1/9.2/8.9 against 8.8/9.0/9.2, and 32003 fp32
// 8.2/9.4/10.3 against 9.7/9.9/10.2.  128 / 256 pairs 5.4/6.9 against 6.6.
constexpr int MEET_FEW = 128;
static Meeting meeting(void *ws, int n) { return {static_cast<uint64_t *>(ws), next_tag(), n}; }
// of the workgroups that go through n tokens or pairs
static Meeting sums_meeting(int64_t n, void *ws)
{
    const int64_t b = (n + SUM_BLOCK - 1) / SUM_BLOCK;
    return meeting(ws, (int)(b < 1 ? 1 : b > MEET_FEW ? MEET_FEW : b));
}

static constexpr int64_t kMaxItems = 0xffffffffLL;      // HIP launches fewer than 2^32 work items at a time

typedef void (*RowKernel)(Logits, int64_t, int64_t, Policy, float *, float *, void *, int64_t);
struct RowShape {
    RowKernel kernel;
    int block;
};
// The kernel for rows of up to `vecs` vectors: the least that holds one.
template <typename E, bool POLICY>
static RowShape row_shape(int64_t vecs)
{
    // Of a row that the shape before, of up to PREV vectors, does not hold, at least PREV - 7 are there, counted from its line: it may start late in it.
#define GS_HELD(PREV, BLOCK, NV, KEEP) \
    if (vecs <= (BLOCK) * (NV)) return {k_held<E, BLOCK, NV, ((PREV) > 7 ? ((PREV) - 7) / (BLOCK) : 0), POLICY ? KEEP : 0, POLICY>, BLOCK}
    GS_HELD(0, 64, 4, 4);
    GS_HELD(256, 128, 4, 4);
    GS_HELD(512, 256, 4, 4);
    if constexpr (POLICY) {
        // wide workgroups, whose waves have few vectors and keep all exponentials
        GS_HELD(1024, 512, 4, 4);
        GS_HELD(2048, 1024, 3, 3);
        GS_HELD(3072, 1024, 4, 4);
        GS_HELD(4096, 1024, 6, 6);
        GS_HELD(6144, 1024, 8, 8);
    } else {
        // few registers either way: narrow ones, of which a CU holds more
        GS_HELD(1024, 256, 8, 0);
        GS_HELD(2048, 512, 6, 0);
        GS_HELD(3072, 512, 8, 0);
        GS_HELD(4096, 512, 12, 0);
        GS_HELD(6144, 512, 16, 0);
    }
    // KEEP: as many as 128 registers a lane have room for; an fp32 vector takes as much as its exponentials
    constexpr bool ALL = E::PER == 4;
    GS_HELD(8192, 1024, 12, 12);
    GS_HELD(12288, 1024, 16, (ALL ? 16 : 8));
    GS_HELD(16384, 1024, 20, (ALL ? 20 : 4));
    static_assert(HELD_MAX == 1024 * 24);
    return {k_held<E, 1024, 24, (20480 - 7) / 1024, POLICY && ALL ? 24 : 0, POLICY>, 1024};
#undef GS_HELD
}

struct Grid {
    int64_t rows;          // of a launch
    int parts, len;
};
// Rows in parts: as many parts as a wave joins, and rows as the workspace holds partials for.
static Grid parts_of(const gs_logits &X)
{
    Grid g;
    const int64_t len = (X.vocab + PARTS - 1) / PARTS;
    g.len = (int)(len <= PART_MIN ? PART_MIN : (len + PART_MIN - 1) / PART_MIN * PART_MIN);
    g.parts = (int)((X.vocab + g.len - 1) / g.len);
    g.rows = GS_SQNORM_MAX_BLOCKS / (2 * g.parts);      // a slot has 16 bytes a part, a row of partials 8 and 8 more
    return g;
}
// Vectors of a row from the start of its first one's line on.  Rows that start on a line each have none missing there.
static int64_t vecs_of(const gs_logits &X)
{
    const bool on_lines = (reinterpret_cast<uintptr_t>(X.data) & 127) == 0 && (X.rows == 1 || X.row_stride % (X.dtype == GS_BF16 ? 64 : 32) == 0);
    return X.vocab / (X.dtype == GS_BF16 ? Bf16::PER : F32::PER) + (on_lines ? 0 : 7);
}
// Whether rows go in parts though they could be held: a long row takes one CU's share of the memory's rate, unless there are about as many
// rows as CUs.  One launch against one without a gradient, two with one.  By elements, of which both types take as long from some rows on: a
// row's exponentials are as many.  us, held against parts:
//   rows                       1           16           32           64           128          256
//   32768 fp32, scored         4.1/4.0     5.0/4.2      4.5/4.1      4.9/4.2      5.6/4.8      7.0/6.1
//   49152 bf16, scored         4.6/3.8     5.0/4.3      5.0/4.4      5.1/4.9      5.4/5.6      6.5/7.5
//   81920 fp32, scored         6.2/4.1     6.8/4.6      6.7/5.2      8.6/5.8      9.6/10.2     14.7/16.2
//   81920 bf16, scored         6.2/4.0     6.7/4.5      6.6/5.3      6.6/5.9      7.5/7.1      9.3/11.5
//   131072 bf16, scored        8.1/4.0     8.4/4.1      8.5/4.7      9.4/6.0      10.5/8.8     16.2/15.5
//   (the policy loss with its gradient; without one it takes the same lines)
//   32768 fp32, policy         5.6/6.5     7.4/7.8      7.8/8.8      8.0/10.7     11.2/16.1
//   49152 fp32, policy         7.4/6.7     9.3/8.3      9.4/9.7      10.7/12.3    13.8/20.5
//   49152 bf16, policy         6.5/6.7     8.3/8.3      8.6/8.5      8.8/10.8     10.0/13.9
//   81920 fp32, policy         10.4/6.8    10.7/9.1     12.4/10.5    14.1/15.9    18.2/27.2
//   81920 bf16, policy         8.7/6.8     10.1/8.5     10.3/10.4    11.3/12.6    13.5/19.8
//   131072 bf16, policy        12.9/7.0    13.7/8.4     14.4/10.7    15.5/15.4    17.6/25.2
// (20480 fp32: scored 3.2/3.6 with one row and 3.4/4.1 with 16, policy 5.0/6.7 and 6.1/7.8; 32000 bf16: scored 3.8/3.9 and 4.1/4.1.)
static bool in_parts(const gs_logits &X, bool gradient)
{
    if (vecs_of(X) > HELD_MAX) return true;
    const int64_t n = X.vocab;
    if (gradient) return X.rows <= (n > 100000 ? 64 : n > 60000 ? 32 : n > 45000 ? 16 : 0);
    return X.rows <= (n > 55000 ? 128 : n > 30000 ? 64 : 0);
}

template <typename E>
static uint32_t grad_runs(int64_t vocab) { return (uint32_t)((vocab / E::PER + 7) / GRAD_VECS + 1); }

template <typename E, bool FROM_PARTS>
static hipError_t launch_grad(GradArgs A, int64_t rows, hipStream_t stream)
{
    A.runs = grad_runs<E>(A.L.vocab);
    const int64_t most = kMaxItems / GRAD_BLOCK / A.runs;               // 31 rows of 2^30 fp32 elements
    const int64_t first = A.row0;
    for (int64_t done = 0; done < rows; done += A.rows) {
        A.rows = rows - done < most ? rows - done : most;
        A.row0 = FROM_PARTS ? first + done : first + rows - done - A.rows;
        k_grad<E, FROM_PARTS><<<(uint32_t)A.rows * A.runs, GRAD_BLOCK, 0, stream>>>(A);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename E, bool POLICY>
static hipError_t launch_in_parts(const gs_logits &X, const Logits &L, const Policy &P, float *logp, float *row_stats, void *dlogits, int64_t dstride,
                                  MaxSum *partials, hipStream_t stream)
{
    const Grid g = parts_of(X);
    for (int64_t r = 0; r < X.rows; r += g.rows) {
        const int rows = (int)(X.rows - r < g.rows ? X.rows - r : g.rows);
        if (!POLICY) {
            const bool once = !row_stats && X.rows * X.vocab * (int64_t)sizeof(typename E::T) > GS_KEEP_BYTES;
            const Finish F = {meeting(partials, g.parts), P.it, logp, row_stats, once};
            k_part<E, true><<<(uint32_t)rows * g.parts, PART_BLOCK, 0, stream>>>(L, r, g.parts, g.len, P.k, nullptr, nullptr, F);
            if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
            continue;
        }
        k_part<E, false><<<(uint32_t)rows * g.parts, PART_BLOCK, 0, stream>>>(L, r, g.parts, g.len, P.k, P.weights, partials, Finish{});
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        if (dlogits) {
            const GradArgs A = {L, r, rows, dstride, P, nullptr, nullptr, partials, logp, dlogits, 0, g.parts};
            // a launch takes as many rows as it can, and joins the partials of its own from the first on: no more than those
            const int64_t most = kMaxItems / GRAD_BLOCK / grad_runs<E>(X.vocab);
            for (int64_t q = 0; q < rows; q += most) {
                GradArgs B = A;
                B.row0 = r + q;
                B.partials = partials + q * (g.parts + 1);
                if (hipError_t e = launch_grad<E, true>(B, rows - q < most ? rows - q : most, stream); e != hipSuccess) return e;
            }
        } else {
            k_join<<<(rows + PART_BLOCK / 64 - 1) / (PART_BLOCK / 64), PART_BLOCK, 0, stream>>>(L, r, rows, g.parts, P.k, P.it, P.weights, partials, logp);
            if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

template <typename E, bool POLICY>
static hipError_t launch_rows_of(const gs_logits &X, const Logits &L, const Policy &P, float *logp, float *row_stats, void *dlogits, int64_t dstride, void *ws,
                                 hipStream_t stream)
{
    if (in_parts(X, POLICY)) return launch_in_parts<E, POLICY>(X, L, P, logp, row_stats, dlogits, dstride, static_cast<MaxSum *>(ws), stream);
    const RowShape s = row_shape<E, POLICY>(vecs_of(X));
    // with the row statistics asked for, the rows are read again for a gradient: what the memory-side cache holds is left there
    const int64_t kept = GS_KEEP_BYTES / (L.stride * (int64_t)sizeof(typename E::T)), keep_row = row_stats ? X.rows - kept : INT64_MAX;
    const int64_t most = kMaxItems / s.block;
    for (int64_t r = 0; r < X.rows; r += most) {
        const int grid = (int)(X.rows - r < most ? X.rows - r : most);
        s.kernel<<<grid, s.block, 0, stream>>>(L, r, keep_row, P, logp, row_stats, dlogits, dstride);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <bool POLICY>
static hipError_t launch_rows(const gs_logits &X, const Logits &L, const Policy &P, float *logp, float *row_stats, void *dlogits, int64_t dstride, void *ws,
                              hipStream_t stream)
{
    if (X.dtype == GS_BF16) return launch_rows_of<Bf16, POLICY>(X, L, P, logp, row_stats, dlogits, dstride, ws, stream);
    return launch_rows_of<F32, POLICY>(X, L, P, logp, row_stats, dlogits, dstride, ws, stream);
}

// ---- checks -----------------------------------------------------------------------------------
// no output overlaps another array; ranges `a` and `b` may, where `skip` says so
static bool apart(const Range *s, int n, bool skip = false, int a = -1, int b = -1)
{
    for (int i = 0; i < n; ++i)
        for (int j = i + 1; j < n; ++j)
            if ((s[i].out || s[j].out) && !(skip && i == a && j == b) && overlap(s[i], s[j])) return false;
    return true;
}
static bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static bool good(const void *p, uintptr_t to) { return p && aligned(p, to); }
static int64_t size_of(int32_t dtype) { return dtype == GS_BF16 ? 2 : 4; }

// bytes from a matrix's first element to behind its last one; -1 if they do not fit an address
static int64_t extent(int64_t rows, int64_t cols, int64_t stride, int64_t size)
{
    int64_t n;
    if (rows > 1 && (__builtin_mul_overflow(rows - 1, stride, &n) || __builtin_add_overflow(n, cols, &n) || __builtin_mul_overflow(n, size, &n))) return -1;
    return rows > 1 ? n : rows * cols * size;
}
static bool good_matrix(const gs_logits *x)
{
    if (!x || (x->dtype != GS_BF16 && x->dtype != GS_F32)) return false;
    if (x->rows < 0 || x->vocab < 1 || x->vocab > (int64_t)1 << 30) return false;
    if (x->rows > (int64_t)1 << 40 || (x->rows > 1 && x->row_stride < x->vocab)) return false;
    if (extent(x->rows, x->vocab, x->row_stride, size_of(x->dtype)) < 0) return false;
    return x->rows == 0 || good(x->data, size_of(x->dtype));
}
static bool good_output(const gs_logits &x, const void *out, int64_t stride)
{
    if (x.rows > 1 && stride < x.vocab) return false;
    return good(out, size_of(x.dtype)) && extent(x.rows, x.vocab, stride, size_of(x.dtype)) >= 0;
}
// Whether an output may lie where the logits do: it is their own memory, row for row, or its rows lie between theirs, at the same distance.
static bool fits_logits(const gs_logits &x, const void *out, int64_t stride)
{
    if (out == x.data && (x.rows == 1 || stride == x.row_stride)) return true;
    if (x.rows == 1 || stride != x.row_stride) return false;
    const int64_t size = size_of(x.dtype), step = stride * size, by = (int64_t)(reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(x.data)) % step;
    const int64_t gap = by < 0 ? by + step : by;           // from a row of logits to the next row of the output
    return gap >= x.vocab * size && step - gap >= x.vocab * size;
}
static bool good_temperature(float t) { return t >= 1e-4f && t <= 1e4f; }
static bool finite_from(float x, float lo) { return std::isfinite(x) && x >= lo; }
static bool good_workspace(const void *ws, size_t bytes) { return ws && bytes >= gs_sqnorm_workspace_bytes() && aligned(ws, 8); }

static Logits logits_of(const gs_logits &x, const int64_t *targets)
{
    return {x.data, x.rows > 1 ? x.row_stride : x.vocab, targets, (int)x.vocab};
}
static Policy scaled_by(float temperature)
{
    Policy P = {};
    P.it = 1.0f / temperature;
    P.k = kLog2e / temperature;
    return P;
}

}  // namespace gs

using namespace gs;

extern "C" {

gs_status gs_token_logp(const gs_logits *logits, const int64_t *targets, float temperature, float *logp, float *row_stats,
                        void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!good_matrix(logits) || !good_temperature(temperature)) return GS_ERR_INVALID_ARG;
    const int64_t rows = logits->rows;
    if (rows && (!good(targets, 8) || !good(logp, 4) || !aligned(row_stats, 4))) return GS_ERR_INVALID_ARG;
    if (!good_workspace(d_workspace, workspace_bytes)) return GS_ERR_WORKSPACE;
    if (rows == 0) return GS_OK;
    const Range s[] = {range_of(logits->data, extent(rows, logits->vocab, logits->row_stride, size_of(logits->dtype)), false),
                       range_of(targets, rows * 8, false), range_of(logp, rows * 4, true), range_of(row_stats, rows * 8, true),
                       range_of(d_workspace, (int64_t)workspace_bytes, true)};
    if (!apart(s, 5)) return GS_ERR_INVALID_ARG;
    hipError_t e = launch_rows<false>(*logits, logits_of(*logits, targets), scaled_by(temperature), logp, row_stats, nullptr, 0, d_workspace,
                                      static_cast<hipStream_t>(stream));
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_token_logp launch");
}

gs_status gs_token_logp_grad(const gs_logits *logits, const int64_t *targets, float temperature, const float *row_stats,
                             const float *dlogp, void *dlogits, int64_t dlogits_stride, void *stream)
{
    if (!good_matrix(logits) || !good_temperature(temperature)) return GS_ERR_INVALID_ARG;
    const int64_t rows = logits->rows, size = size_of(logits->dtype);
    if (rows == 0) return GS_OK;
    if (!good(targets, 8) || !good(row_stats, 4) || !good(dlogp, 4) || !good_output(*logits, dlogits, dlogits_stride)) return GS_ERR_INVALID_ARG;
    const Range s[] = {range_of(logits->data, extent(rows, logits->vocab, logits->row_stride, size), false),
                       range_of(dlogits, extent(rows, logits->vocab, dlogits_stride, size), true), range_of(targets, rows * 8, false),
                       range_of(row_stats, rows * 8, false), range_of(dlogp, rows * 4, false)};
    if (!apart(s, 5, fits_logits(*logits, dlogits, dlogits_stride), 0, 1)) return GS_ERR_INVALID_ARG;
    GradArgs A = {};
    A.L = logits_of(*logits, targets);
    A.P = scaled_by(temperature);
    A.dstride = rows > 1 ? dlogits_stride : logits->vocab;
    A.row_stats = row_stats;
    A.dlogp = dlogp;
    A.dlogits = dlogits;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e = logits->dtype == GS_BF16 ? launch_grad<Bf16, false>(A, rows, st) : launch_grad<F32, false>(A, rows, st);
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_token_logp_grad launch");
}

gs_status gs_policy_loss(const gs_logits *logits, const int64_t *targets, const gs_policy_hparams *hp, const float *old_logp,
                         const float *ref_logp, const float *advantages, const float *weights, float *logp, void *dlogits,
                         int64_t dlogits_stride, float *d_stats, int accumulate, void *d_workspace, size_t workspace_bytes,
                         void *stream)
{
    if (!good_matrix(logits) || !hp || !good_temperature(hp->temperature)) return GS_ERR_INVALID_ARG;
    if (!finite_from(hp->clip_low, 0.0f) || hp->clip_low > 1.0f || !finite_from(hp->clip_high, 0.0f) || !finite_from(hp->kl_coef, 0.0f))
        return GS_ERR_INVALID_ARG;
    const int64_t rows = logits->rows, size = size_of(logits->dtype);
    if (!good(d_stats, 4)) return GS_ERR_INVALID_ARG;
    if (rows) {
        if (!good(targets, 8) || !good(old_logp, 4) || !good(advantages, 4) || !aligned(ref_logp, 4) || !aligned(weights, 4) || !good(logp, 4))
            return GS_ERR_INVALID_ARG;
        if (dlogits && !good_output(*logits, dlogits, dlogits_stride)) return GS_ERR_INVALID_ARG;
    }
    if (!good_workspace(d_workspace, workspace_bytes)) return GS_ERR_WORKSPACE;
    if (rows == 0 && accumulate) return GS_OK;
    if (rows) {
        const Range s[] = {range_of(logits->data, extent(rows, logits->vocab, logits->row_stride, size), false),
                           range_of(dlogits, extent(rows, logits->vocab, dlogits_stride, size), true), range_of(targets, rows * 8, false),
                           range_of(old_logp, rows * 4, false), range_of(ref_logp, rows * 4, false), range_of(advantages, rows * 4, false),
                           range_of(weights, rows * 4, false), range_of(logp, rows * 4, true), range_of(d_stats, 16, true),
                           range_of(d_workspace, (int64_t)workspace_bytes, true)};
        if (!apart(s, 10, dlogits && fits_logits(*logits, dlogits, dlogits_stride), 0, 1)) return GS_ERR_INVALID_ARG;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    Policy P = scaled_by(hp->temperature);
    P.low = 1.0f - hp->clip_low;
    P.high = 1.0f + hp->clip_high;
    P.kl = hp->kl_coef;
    P.old_logp = old_logp;
    P.ref_logp = ref_logp;
    P.advantages = advantages;
    P.weights = weights;
    P.stats = d_stats;
    P.accumulate = accumulate;
    // with few rows the last of them adds up their sums; the workspace's end is theirs, its start holds parts
    const bool meets = rows > 0 && rows <= MEET_FEW && (dlogits || !in_parts(*logits, true));
    if (meets) P.meet = meeting(static_cast<char *>(d_workspace) + (size_t)GS_SQNORM_MAX_BLOCKS * 8 - MEET_FEW * 40, (int)rows);
    hipError_t e = launch_rows<true>(*logits, logits_of(*logits, targets), P, logp, nullptr, dlogits, rows > 1 ? dlogits_stride : logits->vocab, d_workspace, st);
    if (e != hipSuccess) return hip_fail(e, "gs_policy_loss launch");
    if (meets) return GS_OK;
    P.meet = sums_meeting(rows, d_workspace);
    k_policy_sums<<<P.meet.n, SUM_BLOCK, 0, st>>>(targets, (int)logits->vocab, rows, P, logp);
    e = hipGetLastError();
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_policy_loss launch");
}

gs_status gs_preference_loss(const float *logp, const float *ref_logp, const float *weights, int64_t tokens,
                             const int64_t *offsets, int64_t pairs, const gs_preference_hparams *hp, float *margins, float *dlogp,
                             float *d_loss, int accumulate, void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!hp || !std::isfinite(hp->beta) || !(hp->beta > 0.0f) || !finite_from(hp->label_smoothing, 0.0f) || hp->label_smoothing >= 1.0f ||
        !std::isfinite(hp->scale))
        return GS_ERR_INVALID_ARG;
    if (tokens < 0 || tokens > (int64_t)1 << 40 || pairs < 0 || pairs > kMaxItems / PAIR_BLOCK) return GS_ERR_INVALID_ARG;
    if (tokens && (!good(logp, 4) || !good(dlogp, 4) || !aligned(ref_logp, 4) || !aligned(weights, 4))) return GS_ERR_INVALID_ARG;
    if (pairs && (!good(offsets, 8) || !good(margins, 4))) return GS_ERR_INVALID_ARG;
    if (!good(d_loss, 4)) return GS_ERR_INVALID_ARG;
    if (!good_workspace(d_workspace, workspace_bytes)) return GS_ERR_WORKSPACE;
    const Range s[] = {range_of(logp, tokens * 4, false), range_of(ref_logp, tokens * 4, false), range_of(weights, tokens * 4, false),
                       range_of(offsets, pairs ? (2 * pairs + 1) * 8 : 0, false), range_of(margins, pairs * 4, true), range_of(dlogp, tokens * 4, true),
                       range_of(d_loss, 4, true), range_of(d_workspace, (int64_t)workspace_bytes, true)};
    if (!apart(s, 8)) return GS_ERR_INVALID_ARG;
    if (pairs == 0 && tokens == 0 && accumulate) return GS_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    // many pairs: as many margins a launch as the workspace holds, then the loss so far, and behind that the slots of its sum
    const int64_t most = GS_SQNORM_MAX_BLOCKS - 1;
    double *wide = static_cast<double *>(d_workspace), *so_far = wide + most;
    auto sum = [&](int64_t first, int64_t n, const double *before, auto *out, int onto) {
        Meeting meet = sums_meeting(n, so_far + 1);
        meet.n = std::min(meet.n, GS_FINAL_SLICES / 2);
        k_pair_sums<<<meet.n, SUM_BLOCK, 0, st>>>(wide, margins + first, (int)n, hp->label_smoothing, hp->scale, meet, before, out, onto);
    };
    hipError_t e = hipSuccess;
    if (pairs == 0) {
        if (tokens) k_zero<<<(int)(tokens > 256 * SUM_BLOCK ? 256 : (tokens + SUM_BLOCK - 1) / SUM_BLOCK), SUM_BLOCK, 0, st>>>(dlogp, tokens);
        if (!accumulate) sum(0, 0, nullptr, d_loss, 0);
        e = hipGetLastError();
    }
    const bool few = pairs <= MEET_FEW;
    for (int64_t first = 0; first < pairs && e == hipSuccess; first += most) {
        const int64_t n = std::min(most, pairs - first);
        const bool last = first + n == pairs;
        k_pairs<<<(int)n, PAIR_BLOCK, 0, st>>>(Pairs{logp, ref_logp, weights, offsets + first, tokens, pairs, hp->beta, hp->label_smoothing, hp->scale,
                                                     margins + first, dlogp, few ? meeting(d_workspace, (int)n) : Meeting{static_cast<uint64_t *>(d_workspace), 0, 0},
                                                     d_loss, accumulate, (first == 0 ? 1 : 0) | (last ? 2 : 0)});
        if (!few && last) sum(first, n, first > 0 ? so_far : nullptr, d_loss, accumulate);
        else if (!few) sum(first, n, nullptr, so_far, first > 0);
        e = hipGetLastError();
    }
    return e == hipSuccess ? GS_OK : hip_fail(e, "gs_preference_loss launch");
}

}  // extern "C"
