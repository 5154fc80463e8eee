// A HIP runtime that launches nothing and writes down what the launchers of a head without its logits ask it to launch: gs_head.hip is
// compiled here, for the host only, so its kernels' arguments are read as the types they have, and each launch is written down with the memory that
// it reads and writes by them.  Test infrastructure only.
//
// As the HIP runtime does, hipLaunchKernel refuses an empty launch and one of 2^32 work items or more.
#include "gs_head.hip"

#include <cxxabi.h>

#include <cstdio>
#include <cstring>
#include <map>
#include <string>
#include <vector>

struct Span {
    char role[24];
    uint64_t lo, bytes;
    int32_t write, launch;
};
struct Launch {
    char kernel[256];            // with its template arguments
    uint64_t grid, grid_y, block;
    int64_t word0, words;        // of the vocabulary that it takes
    int64_t steps, splits, first;
    int64_t rows, hidden;        // as its tiles are counted
    uint64_t rows_workgroups;    // of a launch that has two kinds, those of the first
    int32_t status, pad;
};

static std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> n;
    return n;
}
static std::vector<Launch> g_launches;
static std::vector<Span> g_spans;
static hipError_t g_last = hipSuccess;

static std::string kernel_name(const char *mangled)
{
    int st = 0;
    char *d = abi::__cxa_demangle(mangled, nullptr, nullptr, &st);
    std::string s = st == 0 && d ? d : mangled;
    free(d);
    const size_t at = s.find("gs::k_");
    return at == std::string::npos ? s : s.substr(at + 4);
}

struct Args {
    void **at;
    template <typename T>
    const T &next()
    {
        return *static_cast<const T *>(*at++);
    }
};

static void span(const char *role, const void *p, int64_t bytes, bool write)
{
    if (!p || bytes <= 0) return;
    Span s = {};
    strncpy(s.role, role, sizeof s.role - 1);
    s.lo = reinterpret_cast<uint64_t>(p);
    s.bytes = (uint64_t)bytes;
    s.write = write;
    s.launch = (int32_t)g_launches.size();
    g_spans.push_back(s);
}
// rows of `cols` elements of `size` bytes, `stride` elements apart
static void rows_span(const char *role, const void *p, int64_t rows, int64_t cols, int64_t stride, int64_t size, bool write)
{
    if (rows > 0) span(role, p, ((rows - 1) * stride + cols) * size, write);
}
static void live_span(const Live &L, int64_t rows, bool write)
{
    span("count", L.count, 4, write);
    span("index", L.index, rows * 4, write);
    span("place", L.place, rows * 4, write);
    span("token", L.token, rows * 4, write);
}
static void operand(const char *role, const Operand &X) { rows_span(role, X.p, X.rows, X.cols, X.stride, 2, false); }

extern "C" {

extern const char __hip_fatbin[16] = {0};
void **__hipRegisterFatBinary(const void *) { static void *handle; return &handle; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *)
{
    names()[host] = kernel_name(name);
}

static dim3 g_grid, g_block;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t)
{
    g_grid = grid;
    g_block = block;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, hipStream_t *stream)
{
    *grid = g_grid;
    *block = g_block;
    *shared = 0;
    *stream = nullptr;
    return hipSuccess;
}

hipError_t hipLaunchKernel(const void *fn, dim3 grid, dim3 block, void **args, size_t, hipStream_t)
{
    Launch l;
    memset(&l, 0, sizeof l);
    const std::string &name = names()[fn];
    strncpy(l.kernel, name.substr(0, name.find('(')).c_str(), sizeof l.kernel - 1);
    l.grid = grid.x;
    l.grid_y = grid.y;
    l.block = block.x;
    const bool good = grid.x && grid.y && grid.y < 65536 && grid.z == 1 && block.x && block.x <= 1024 && block.y == 1 && block.z == 1 &&
                      (uint64_t)grid.x * block.x < (1ull << 32) && (uint64_t)grid.x * grid.y * block.x < (1ull << 40);
    l.status = good ? hipSuccess : hipErrorInvalidConfiguration;
    auto is = [&](const char *p) { return name.compare(0, strlen(p), p) == 0; };
    auto takes = [&](const char *parameters) {
        if (name.find(parameters) != std::string::npos) return;
        fprintf(stderr, "the recorder does not know how to read %s\n", name.c_str());
        abort();
    };
    auto logit = [&](const Logit &G) {
        l.word0 = G.word0;
        l.words = G.words;
        l.rows = G.rows;
        span("bias", G.bias, G.vocab * 2, false);
        live_span(G.live, G.rows, false);
    };
    Args a{args};
    if (is("k_head_live")) {
        takes("(long const*, float const*, int, int, gs::Live, float*, float*)");
        a.next<const int64_t *>();
        a.next<const float *>();
        const int rows = a.next<int>();
        a.next<int>();
        live_span(a.next<Live>(), rows, true);
    } else if (is("k_head_pack<")) {
        takes("(unsigned short const*, long, long, gs::Live, long, unsigned short*, long)");
        const uint16_t *from = a.next<const uint16_t *>();
        const int64_t stride = a.next<int64_t>(), cols = a.next<int64_t>();
        const Live &L = a.next<Live>();
        const int64_t rows = a.next<int64_t>();
        uint16_t *to = a.next<uint16_t *>();
        const int64_t width = a.next<int64_t>();
        live_span(L, L.count ? rows : 0, false);
        if (!L.count) rows_span("w", from, rows, cols, stride, 2, false);
        rows_span(L.count ? "x packed" : "w packed", to, grid.x, width, width, 2, true);
    } else if (is("k_head_gather<")) {
        takes("(long const*, float const*, int, int, gs::Live, float*, float*, unsigned short const*, long, long, unsigned short*, long)");
        a.next<const int64_t *>();
        a.next<const float *>();
        const int rows = a.next<int>();
        a.next<int>();
        live_span(a.next<Live>(), rows, true);
        a.next<float *>();
        a.next<float *>();
        a.next<const uint16_t *>();
        a.next<int64_t>();
        a.next<int64_t>();
        uint16_t *to = a.next<uint16_t *>();
        const int64_t width = a.next<int64_t>();
        rows_span("x packed", to, grid.x, width, width, 2, true);
    } else if (is("k_head_stats<") || is("k_head_dz<")) {
        takes("(gs::Operand, gs::Operand, int, gs::Logit)");
        const Operand &W = a.next<Operand>(), &X = a.next<Operand>();
        l.steps = a.next<int>();
        const Logit &G = a.next<Logit>();
        logit(G);
        int bm = 0;
        sscanf(name.c_str() + name.find("Tile<"), "Tile<%d", &bm);
        const int64_t tiles = (G.words + bm - 1) / bm;
        if (W.rows != G.words || l.steps * BK > W.cols || l.steps * BK > X.cols) l.status = -1;
        operand("w read", W);
        operand("x packed", X);
        if (is("k_head_stats<")) {
            if (G.word0 % bm) l.status = -1;
            span("partials", G.partials + G.word0 / bm * G.rows, tiles * G.rows * 8, true);
            span("target", G.target_logit, G.rows * 4, true);
            if (G.z) rows_span("z", G.z, G.rows, tiles * bm, G.z_stride, 4, true);
        } else {
            span("row", G.row, G.rows * 16, false);
            rows_span("dz", G.dz, G.rows, tiles * bm, G.stride, 2, true);
        }
    } else if (is("k_head_dz_kept")) {
        takes("(gs::Logit, gs::Loss)");
        const Logit &G = a.next<Logit>();
        logit(G);
        const int64_t words = up(G.words, 256);
        if ((int64_t)grid.y * 1024 < words || grid.x != (uint64_t)G.rows + 1) l.status = -1;
        span("row", G.row, G.rows * 16, false);
        rows_span("z", G.z, G.rows, words, G.z_stride, 4, false);
        rows_span("dz", G.dz, G.rows, words, G.stride, 2, true);
    } else if (is("k_head_dx") || is("k_head_dw<")) {
        auto to_rows = [&](const Operand &W, const Operand &DZ, const ToRows &R) {
            l.rows = R.rows;
            l.steps = R.steps;
            l.splits = R.splits;
            l.first = R.first;
            l.hidden = R.hidden;
            l.words = W.rows;
            if ((int64_t)R.steps * BK > DZ.cols || R.hidden > W.cols) l.status = -1;
            operand("w read", W);
            rows_span("dz", DZ.p, R.rows, (int64_t)R.steps * BK, DZ.stride, 2, false);
            span("sum", R.sum, R.splits * R.rows * R.hidden * 4, true);
        };
        auto to_weights = [&](const Operand &X, const ToWeights &G) {
            l.word0 = G.word0;
            l.words = G.words;
            operand("x packed", X);
            span("row", G.row, 16, false);
            rows_span("dw", G.dw + G.word0 * G.stride, G.words, G.hidden, G.stride, 2, true);
        };
        if (is("k_head_dx_dw<")) {
            takes("(gs::Operand, gs::Operand, gs::Operand, gs::ToRows, gs::ToWeights, unsigned int)");
            const Operand &W = a.next<Operand>(), &X = a.next<Operand>(), &DZ = a.next<Operand>();
            const ToRows &R = a.next<ToRows>();
            to_rows(W, DZ, R);
            to_weights(X, a.next<ToWeights>());
            l.rows_workgroups = a.next<uint32_t>() / (uint64_t)R.splits;
        } else if (is("k_head_dx<")) {
            takes("(gs::Operand, gs::Operand, gs::ToRows)");
            const Operand &W = a.next<Operand>(), &DZ = a.next<Operand>();
            const ToRows &R = a.next<ToRows>();
            to_rows(W, DZ, R);
            l.rows_workgroups = grid.x;
            if (grid.y != (uint32_t)R.splits) l.status = -1;
        } else {
            takes("(gs::Operand, gs::Operand, gs::ToWeights)");
            const Operand &X = a.next<Operand>();
            a.next<Operand>();
            to_weights(X, a.next<ToWeights>());
        }
    } else if (is("k_head_db")) {
        takes("(unsigned short const*, long, gs::Live, long, HIP_vector_type<float, 4u> const*, unsigned short*)");
        const uint16_t *dz = a.next<const uint16_t *>();
        const int64_t stride = a.next<int64_t>();
        a.next<Live>();
        l.words = a.next<int64_t>();
        span("row", a.next<const float4 *>(), 16, false);
        span("db", a.next<uint16_t *>(), l.words * 2, true);
        rows_span("dz", dz, 1, grid.x * 128, stride, 2, false);
        if ((int64_t)grid.x * 128 < l.words || (int64_t)grid.x * 128 > stride) l.status = -1;
    } else if (is("k_head_rows_out")) {
        takes("(gs::Live, float const*, int, long, long, long, HIP_vector_type<float, 4u> const*, unsigned short*, long)");
        const Live &L = a.next<Live>();
        const float *sum = a.next<const float *>();
        const int splits = a.next<int>();
        const int64_t rows = a.next<int64_t>(), width = a.next<int64_t>(), hidden = a.next<int64_t>();
        span("place", L.place, (int64_t)grid.x * 4, false);
        span("sum", sum, splits * rows * width * 4, false);
        span("row", a.next<const float4 *>(), rows * 16, false);
        uint16_t *dx = a.next<uint16_t *>();
        rows_span("dx", dx, grid.x, hidden, a.next<int64_t>(), 2, true);
        l.rows = grid.x;
    } else if (is("k_head_join<")) {
        takes("(gs::Join)");
        const Join &J = a.next<Join>();
        l.rows = J.rows;
        span("partials", J.partials, J.tiles * J.rows * 8, false);
        span("target", J.target_logit, J.rows * 4, false);
        span("row", J.row, J.rows * 16, true);
        live_span(J.live, J.live.count ? J.rows : 0, false);
    } else if (is("k_head_rows(")) {
        takes("(gs::Live, float const*, float const*, float, HIP_vector_type<float, 4u>*)");
        const Live &L = a.next<Live>();
        a.next<const float *>();
        a.next<const float *>();
        a.next<float>();
        live_span(L, 1, false);
        span("row", a.next<float4 *>(), (int64_t)grid.x * 16, true);          // as many as count: no more than this at least
    } else if (is("k_head_loss")) {
        takes("(gs::Live, gs::Loss)");
        live_span(a.next<Live>(), 1, false);
    } else {
        if (!is("k_head_few<") && !is("k_head_dot<")) takes("no such kernel");
        takes("(gs::Few)");
        const Few &G = a.next<Few>();
        l.rows = G.rows;
        l.words = G.vocab;
        rows_span("w read", G.w, G.vocab, G.hidden, G.w_stride, 2, false);
        span("partials", G.partials, (int64_t)grid.x * G.rows * 8, true);
        span("target", G.target_logit, G.rows * 4, true);
        if ((int64_t)grid.x * FEW_WORDS < G.vocab) l.status = -1;
    }
    g_launches.push_back(l);
    if (l.status != hipSuccess) g_last = hipErrorInvalidConfiguration;
    return (hipError_t)l.status;
}

hipError_t hipGetLastError()
{
    const hipError_t e = g_last;
    g_last = hipSuccess;
    return e;
}

// ---- what the tests call -------------------------------------------------------------------------
void rec_reset()
{
    g_launches.clear();
    g_spans.clear();
    g_last = hipSuccess;
}
int rec_count() { return (int)g_launches.size(); }
void rec_get(int i, Launch *out) { *out = g_launches[i]; }
int rec_spans() { return (int)g_spans.size(); }
void rec_span(int i, Span *out) { *out = g_spans[i]; }
int rec_kernels(char *out, int cap)              // the names of all kernels, one a line
{
    std::string s;
    for (const auto &n : names()) s += n.second.substr(0, n.second.find('(')) + "\n";
    strncpy(out, s.c_str(), cap);
    return (int)s.size();
}
// The tile of a workgroup, as the kernels find it; bm: the larger side of the kernel's tile, bn: its side of rows.
int rec_tile(int bm, int bn, int of_rows, uint32_t id, int64_t across, int64_t rows, int count, uint32_t *a, uint32_t *b)
{
    auto with = [&](auto t) {
        typedef decltype(t) T;
        return of_rows ? tile_of_rows<T>(id, across, rows, count, *a, *b) : tile_of_z<T>(id, across, rows, count, *a, *b);
    };
    if (bm == Big::BM && bn == Big::BN) return with(Big{});
    if (bm == Mid::BM && bn == Mid::BN) return with(Mid{});
    if (bm == Slim::BM && bn == Slim::BN) return with(Slim{});
    if (bm == Tiny::BM && bn == Tiny::BN) return with(Tiny{});
    return -1;
}
}

namespace gs {
gs_status hip_fail(hipError_t, const char *) { return GS_ERR_HIP; }
}  // namespace gs
