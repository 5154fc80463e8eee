// A HIP runtime that launches nothing and writes down what the launchers of the losses and of norm and clip over many tensors
// ask it to launch: those two files are compiled here, for the host only, so their kernels' arguments are read as the types they have.
// Test infrastructure only.
//
// As the HIP runtime does, hipLaunchKernel refuses an empty launch and one of 2^32 work items or more.
#include "gs_loss.hip"
#include "gs_tensors.hip"

#include <cxxabi.h>

#include <cstdio>
#include <map>
#include <string>
#include <vector>

struct Launch {
    char kernel[512];            // with its template arguments
    uint64_t grid, block;
    int64_t row0, rows;          // rows of logits, or pairs, that it takes
    int64_t parts, len, runs;
    int64_t count;               // values that it sums, tensors of its table
    uint64_t partials, slots;    // where partials and slots start
    int64_t slot0, meet;         // of those slots the launch's first one, and all that meet (0: none do)
    uint64_t tag;
    int64_t words;               // a slot
    int64_t tiles, tile_runs, nv, keep_tile;
    uint64_t out;                // a sum's result
    int32_t accumulate, ends, status;
};
struct Tensor {
    int32_t launch;
    uint64_t in, out, numel;
    int32_t dtype;
    uint32_t first;
};

static std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> n;
    return n;
}
static std::vector<Launch> g_launches;
static std::vector<Tensor> g_tensors;
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
static uint64_t addr(const void *p) { return reinterpret_cast<uint64_t>(p); }

struct Args {
    void **at;
    template <typename T>
    const T &next()
    {
        return *static_cast<const T *>(*at++);
    }
};

static void meet_of(Launch &l, const Meeting &m, int64_t first, int words)
{
    l.slots = addr(m.slots);
    l.meet = m.n;
    l.tag = m.tag;
    l.slot0 = first;
    l.words = words;
}

// host side of an entry, as the kernel has it
template <typename S>
static Tensor entry(const S &e);
template <>
Tensor entry(const Whereabouts &e)
{
    const uint64_t a = (uint64_t)e.hi << 32 | e.lo;
    return {0, a & ~1ull, a & ~1ull, e.numel, a & 1 ? GS_BF16 : GS_F32, 0};
}
template <>
Tensor entry(const WithOut &e)
{
    Tensor t = entry(e.in);
    t.out = (uint64_t)e.hi << 32 | e.lo;
    return t;
}
template <int N>
static void table_of(Launch &l, const Table<N> &t)
{
    l.count = t.count;
    l.tiles = t.tiles;
    l.tile_runs = t.runs;
    l.keep_tile = t.keep_tile;
    for (int i = 0; i < t.count; ++i) {
        Tensor x = entry(t.e[i]);
        x.launch = (int)g_launches.size();
        x.first = t.first[i];
        g_tensors.push_back(x);
    }
    for (int i = t.count; i < N && t.count; ++i)
        if (t.first[i] != ~0u) l.status = -1;
}

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
    l.block = block.x;
    const uint64_t items = (uint64_t)grid.x * block.x;
    l.status = items == 0 || items >= (1ull << 32) || block.x > 1024 || grid.y != 1 || grid.z != 1 ? hipErrorInvalidConfiguration : hipSuccess;
    auto is = [&](const char *p) { return name.compare(0, strlen(p), p) == 0; };
    auto takes = [&](const char *parameters) {
        if (name.find(parameters) != std::string::npos) return;
        fprintf(stderr, "the recorder does not know how to read %s\n", name.c_str());
        abort();
    };
    Args a{args};
    if (is("k_held<")) {
        takes("(gs::Logits, long, long, gs::Policy, ");
        a.next<Logits>();
        l.row0 = a.next<int64_t>();
        l.rows = grid.x;
        a.next<int64_t>();
        const Policy &P = a.next<Policy>();
        meet_of(l, P.meet, l.row0, 5);
    } else if (is("k_part<")) {
        takes("(gs::Logits, long, int, int, float, float const*, gs::MaxSum*, gs::Finish)");
        const Logits &L = a.next<Logits>();
        l.row0 = a.next<int64_t>();
        l.parts = a.next<int>();
        l.len = a.next<int>();
        l.rows = grid.x / l.parts;
        if (grid.x % l.parts || (l.parts - 1) * l.len >= L.vocab || l.parts * l.len < L.vocab) l.status = -1;
        a.next<float>();
        a.next<const float *>();
        l.partials = addr(a.next<MaxSum *>());
        const Finish &F = a.next<Finish>();
        meet_of(l, F.meet, 0, 2);
    } else if (is("k_join")) {
        takes("(gs::Logits, long, int, int, float, float, float const*, gs::MaxSum const*, float*)");
        a.next<Logits>();
        l.row0 = a.next<int64_t>();
        l.rows = a.next<int>();
        l.parts = a.next<int>();
        a.next<float>();
        a.next<float>();
        a.next<const float *>();
        l.partials = addr(a.next<MaxSum *>());
        if (grid.x * (block.x / 64) < l.rows) l.status = -1;
    } else if (is("k_grad<")) {
        takes("(gs::GradArgs)");
        const GradArgs &A = a.next<GradArgs>();
        l.row0 = A.row0;
        l.rows = A.rows;
        l.runs = A.runs;
        l.parts = A.parts;
        l.partials = addr(A.partials);
        meet_of(l, A.P.meet, l.row0, 5);
    } else if (is("k_policy_sums")) {
        takes("(long const*, int, long, gs::Policy, float const*)");
        a.next<const int64_t *>();
        a.next<int>();
        l.count = a.next<int64_t>();
        const Policy &P = a.next<Policy>();
        meet_of(l, P.meet, 0, 8);
        l.out = addr(P.stats);
        l.accumulate = P.accumulate;
    } else if (is("k_pairs")) {
        takes("(gs::Pairs)");
        const Pairs &A = a.next<Pairs>();
        l.rows = grid.x;
        l.row0 = (int64_t)addr(A.offsets);
        l.ends = A.ends;
        l.partials = A.meet.n ? 0 : addr(A.meet.slots);
        l.out = addr(A.margins);
        if (A.meet.n) meet_of(l, A.meet, 0, 2);
    } else if (is("k_pair_sums<")) {
        takes("(double const*, float*, int, float, float, gs::Meeting, double const*, ");
        l.partials = addr(a.next<const double *>());
        l.row0 = (int64_t)addr(a.next<float *>());
        l.count = a.next<int>();
        a.next<float>();
        a.next<float>();
        meet_of(l, a.next<Meeting>(), 0, 2);
        l.len = (int64_t)addr(a.next<const double *>());       // the loss so far, or nothing
        l.out = addr(a.next<const void *>());
        l.accumulate = a.next<int>();
    } else if (is("k_zero")) {
        takes("(float*, long)");
        l.out = addr(a.next<float *>());
        l.count = a.next<int64_t>();
    } else if (is("k_tensors_sqnorm<") || is("k_tensors_clip<")) {
        int n = 0, nv = 0;
        sscanf(name.c_str() + name.find('<'), "<%d, %d>", &n, &nv);
        l.nv = nv;
        if (n == TABLE_SMALL) table_of(l, a.next<Table<TABLE_SMALL>>());
        else if (n == TABLE) table_of(l, a.next<Table<TABLE>>());
        else if (n == TABLE_IN_PLACE) table_of(l, a.next<Table<TABLE_IN_PLACE>>());
        else takes("no such table");
        if (is("k_tensors_sqnorm<")) {
            takes(">, double*, gs::Meeting, int, double*, int)");
            l.partials = addr(a.next<double *>());
            const Meeting &m = a.next<Meeting>();
            meet_of(l, m, a.next<int>(), 2);
            l.out = addr(a.next<double *>());
            l.accumulate = a.next<int>();
        } else {
            takes(">, double const*, float, float*)");
            a.next<const double *>();
            a.next<float>();
            l.out = addr(a.next<float *>());
        }
    } else {
        takes("k_tensors_fold(double const*, int, gs::Meeting, double*, int)");
        l.partials = addr(a.next<const double *>());
        l.count = a.next<int>();
        meet_of(l, a.next<Meeting>(), 0, 2);
        l.out = addr(a.next<double *>());
        l.accumulate = a.next<int>();
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

// ---- what the two files take from the library's others, and what the tests call ----------------
size_t gs_sqnorm_workspace_bytes(void) { return (size_t)(GS_SQNORM_MAX_BLOCKS + GS_FINAL_SLICES) * sizeof(double); }

void rec_reset()
{
    g_launches.clear();
    g_tensors.clear();
    g_last = hipSuccess;
}
int rec_count() { return (int)g_launches.size(); }
void rec_get(int i, Launch *out) { *out = g_launches[i]; }
int rec_tensors() { return (int)g_tensors.size(); }
void rec_tensor(int i, Tensor *out) { *out = g_tensors[i]; }
int rec_kernels(char *out, int cap)              // the names of all kernels, one a line
{
    std::string s;
    for (const auto &n : names()) s += n.second.substr(0, n.second.find('(')) + "\n";
    strncpy(out, s.c_str(), cap);
    return (int)s.size();
}
}

namespace gs {
gs_status hip_fail(hipError_t, const char *) { return GS_ERR_HIP; }
uint32_t next_tag()
{
    static uint32_t n = 0;
    return 0x7ff00001u + n++;
}
}  // namespace gs
