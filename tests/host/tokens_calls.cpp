// The host side of the calls for several tokens per user on a HIP runtime that is not there: this program defines the runtime's functions itself, so
// that the built library (loaded with dlopen) allocates from the heap.  A table's upload is carried out; of every other launch the arguments
// are kept, and what the kernels would do by them is gone through here, key by key or byte by byte.  Run without a GPU by tests/test_tokens_calls.py.
#include <dlfcn.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <string>
#include <utility>
#include <vector>

#include "../../paper_2409_19134_amd/csrc/rotary.hpp"
#include "../../paper_2409_19134_amd/csrc/tokens_schedule.hpp"

using namespace spd;
using namespace spd::host;

struct Launch {
    std::string kernel;
    dim3 grid, block;
    TokArgs attend;      // the attention's kernels and the join
    const TokJoin *joins;
    RotateArgs rotate;
    AppendArgs append;
    AppendItems given;
};
static std::vector<Launch> launches;
static int uploads = 0;
static hipError_t last_error = hipSuccess;
static hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;

static std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> m;
    return m;
}

extern "C" {
struct Config {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
};
static Config pushed;
static char static_array[SPD_STATIC_SCRATCH_BYTES] __attribute__((aligned(256)));
hipError_t hipGetDeviceCount(int *n) { return *n = 1, hipSuccess; }
hipError_t hipGetDevice(int *n) { return *n = 0, hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t, int) { return *v = 256, hipSuccess; }  // compute units
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n) { return *p = std::malloc(n), *p ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipFree(void *p) { return std::free(p), hipSuccess; }
hipError_t hipHostMalloc(void **p, size_t n, unsigned) { return *p = std::malloc(n), *p ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipHostFree(void *p) { return std::free(p), hipSuccess; }
hipError_t hipGetSymbolAddress(void **p, const void *) { return *p = static_array, hipSuccess; }
hipError_t hipEventCreate(hipEvent_t *e) { return *e = (hipEvent_t)e, hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) { return *e = (hipEvent_t)e, hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipGetLastError() { return std::exchange(last_error, hipSuccess); }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *status) { return *status = capture, hipSuccess; }
void **__hipRegisterFatBinary(const void *)
{
    static void *handle;
    return &handle;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *fn, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names()[fn] = name; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream)
{
    pushed = Config{grid, block, lds, stream};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    *grid = pushed.grid, *block = pushed.block, *lds = pushed.lds, *stream = pushed.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *fn, dim3 grid, dim3 block, void **args, size_t, hipStream_t)
{
    Launch l = {names()[fn], grid, block, {}, nullptr, {}, {}, {}};
    for (uint64_t threads : {(uint64_t)grid.x * block.x, (uint64_t)grid.y * block.y, (uint64_t)grid.z * block.z})
        if (threads == 0 || threads > 0xffffffffull)  // the runtime's limit for each dimension
            return last_error = hipErrorInvalidConfiguration;
    if (l.kernel.find("tokens_upload_kernel") != std::string::npos) {
        std::memcpy(*static_cast<char **>(args[1]), *static_cast<const char **>(args[0]), (size_t)*static_cast<unsigned *>(args[2]) * 16);
        ++uploads;
        return hipSuccess;
    }
    if (l.kernel.find("tokens_") != std::string::npos)
        std::memcpy(&l.attend, args[0], sizeof l.attend);
    if (l.kernel.find("rotate_kernel") != std::string::npos)
        std::memcpy(&l.rotate, args[0], sizeof l.rotate);
    if (l.kernel.find("append_kernel") != std::string::npos) {
        std::memcpy(&l.append, args[0], sizeof l.append);
        std::memcpy(&l.given, args[1], sizeof l.given);
    }
    if (l.kernel.find("tokens_join_kernel") != std::string::npos)
        l.joins = *static_cast<const TokJoin **>(args[1]);
    launches.push_back(l);
    return hipSuccess;
}
}

#define FAIL(...)                 \
    do {                          \
        std::printf(__VA_ARGS__); \
        std::printf("\n");        \
        std::exit(1);             \
    } while (0)

template <class F>
static F symbol(void *lib, F, const char *name)
{
    return reinterpret_cast<F>(dlsym(lib, name));
}
static void *lib;
#define SYM(f) static const auto f##_ = symbol(lib, &f, #f)

static void *const kNowhere = reinterpret_cast<void *>(0x700000000000ull);  // an address that is passed on, never read

// One call of the attention; users' lengths and positions may be changed from call to call.
struct Attend {
    spd_shape s;
    std::vector<int32_t> lens, n_new, q_pos, k_pos, prefix;
    std::vector<const void *> ptrs;
    spd_kv_view v = {};
    spd_score c = {};

    Attend(int dtype, int Hq, int Hkv, int d, std::vector<int32_t> lens_, std::vector<int32_t> n_new_, std::vector<int32_t> q_pos_)
        : s{dtype, Hq, Hkv, d, 0.1f}, lens(lens_), n_new(n_new_), q_pos(q_pos_), k_pos(lens.size(), 0), prefix(lens.size(), 0),
          ptrs(lens.size(), kNowhere)
    {
        v.n_users = (int32_t)lens.size();
        v.lens = lens.data();
        v.k_ptrs = v.v_ptrs = ptrs.data();
        v.token_stride = d;
        v.head_stride = (int64_t)100000 * d;
        c.causal = 1;
        c.q_pos = q_pos.data();
        c.k_pos = k_pos.data();
        c.prefix = prefix.data();
    }
    Attend(const Attend &) = delete;

    bool visible(int u, int64_t pos_q, int64_t pos_k) const
    {
        if (pos_k < prefix[(size_t)u])
            return true;
        return !(c.causal && pos_k > pos_q) && (c.window == 0 || std::llabs(pos_q - pos_k) < c.window);
    }

    int call(spd_ctx *ctx)
    {
        SYM(spd_partial_attn_tokens);
        launches.clear();
        return spd_partial_attn_tokens_(ctx, &s, kNowhere, (int64_t)s.n_q_heads * s.head_dim, &v, n_new.data(), &c, kNowhere, SPD_F32,
                                        static_cast<float *>(kNowhere), nullptr);
    }

    // Goes through the launched items as their kernels do: every key that a row sees in exactly one step of the row's items, no key twice.
    void check(const char *what) const
    {
        const int G = s.n_q_heads / s.n_kv_heads, row_bytes = s.head_dim * elt_size(s.dtype);
        std::map<std::pair<int, int>, std::vector<int>> taken;  // (user, row) of KV head 0 and the last: how often each key
        for (const Launch &l : launches) {
            const bool many = l.kernel.find("tokens_many_kernel") != std::string::npos;
            if (!many && l.kernel.find("tokens_few_kernel") == std::string::npos)
                continue;
            const int step = many ? many_keys(s.dtype) : row_bytes == 512 ? 16 : 32, waves = many ? 1 : 4;
            for (unsigned i = 0; i < l.grid.x; ++i) {
                const TokItem &it = l.attend.items[i];
                if (it.n_rows == 0 || it.kv_head != s.n_kv_heads - 1)
                    continue;
                const TokUser &u = l.attend.users[it.user];
                const int len = u.len + l.attend.grow_len, q0 = u.q_pos + l.attend.grow_q, end = it.k_end + (it.to_len ? l.attend.grow_len : 0);
                if (len != lens[(size_t)it.user] || q0 != q_pos[(size_t)it.user] - k_pos[(size_t)it.user])
                    FAIL("%s: user %d: %d keys, queries from %d; the table says %d, %d", what, it.user, lens[(size_t)it.user], q_pos[(size_t)it.user], len, q0);
                const Limits lim = tile_limits(l.attend.score, u, len, q0 + it.row0 / G, q0 + (it.row0 + it.n_rows - 1) / G);
                const KeyWalk walk(lim, it.k_begin, end, step, waves);
                std::vector<char> here((size_t)len, 0);
                for (int w = 0; w < waves; ++w)
                    for (int t = walk.first(w); t < walk.hi; t = walk.next(t))
                        for (int key = t; key < std::min(t + step, walk.hi); ++key)
                            ++here[(size_t)key];
                for (int r = it.row0; r < it.row0 + it.n_rows; ++r) {
                    std::vector<int> &row = taken[{it.user, r}];
                    row.resize((size_t)len, 0);
                    for (int key = 0; key < len; ++key)
                        row[(size_t)key] += here[(size_t)key];
                }
            }
        }
        for (int u = 0; u < v.n_users; ++u)
            for (int r = 0; r < n_new[(size_t)u] * G; ++r) {
                const auto found = taken.find({u, r});
                if (found == taken.end())
                    FAIL("%s: user %d row %d is in no tile", what, u, r);
                for (int key = 0; key < lens[(size_t)u]; ++key) {
                    const int n = found->second[(size_t)key];
                    const bool want = visible(u, (int64_t)q_pos[(size_t)u] + r / G, (int64_t)k_pos[(size_t)u] + key);
                    if (n > 1 || (want && n != 1))
                        FAIL("%s: user %d of %d keys, queries from %d, window %d, prefix %d: row %d sees key %d, which is taken %d times", what, u,
                             lens[(size_t)u], q_pos[(size_t)u] - k_pos[(size_t)u], c.window, prefix[(size_t)u] - k_pos[(size_t)u], r, key, n);
                }
            }
    }
};

static spd_ctx *make()
{
    SYM(spd_create);
    spd_ctx *ctx = nullptr;
    if (spd_create_(&ctx, 0) != SPD_OK)
        FAIL("spd_create");
    return ctx;
}
static void drop(spd_ctx *ctx)
{
    SYM(spd_destroy);
    spd_destroy_(ctx);
}

// Tables that are used again after lengths and positions have moved on, each by itself.
static void growth()
{
    struct Moved {
        int window, prefix, n_new, len[2], q_pos[2];
    };
    const Moved moved[] = {
        {32, 0, 1, {64, 104}, {104, 104}},      // the window lay behind the last key, then keys came into it
        {50, 0, 3, {100, 160}, {159, 160}},     // ... with a query that moved on too
        {2, 0, 1, {10, 13}, {12, 12}},
        {8, 5, 2, {40, 60}, {60, 60}},          // ... behind a prefix
        {20, 200, 1, {100, 150}, {180, 180}},   // ... inside the prefix, which the keys grow into
        {20, 120, 1, {100, 150}, {180, 181}},
        {64, 0, 1, {100, 164}, {163, 164}},     // the window began at the last key already
        {64, 0, 1, {100, 101}, {164, 164}},
    };
    for (const Moved &m : moved) {
        spd_ctx *ctx = make();
        Attend a(SPD_BF16, 8, 2, 64, {m.len[0]}, {m.n_new}, {m.q_pos[0]});
        a.c.window = m.window;
        a.prefix[0] = m.prefix;
        for (int i = 0; i < 2; ++i) {
            a.lens[0] = m.len[i];
            a.q_pos[0] = m.q_pos[i];
            if (a.call(ctx) != SPD_OK)
                FAIL("growth: the call fails");
            a.check("growth");
        }
        drop(ctx);
    }
    // a walk: lengths and positions of all users move on (or back) by steps of their own
    std::mt19937 rng(5);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    for (int round = 0; round < 300; ++round) {
        spd_ctx *ctx = make();
        const int U = pick(1, 3), window = pick(0, 4) ? pick(1, 150) : 0;
        std::vector<int32_t> lens, n_new, q_pos;
        for (int u = 0; u < U; ++u) {
            lens.push_back(pick(1, 300));
            n_new.push_back(pick(1, 4));
            q_pos.push_back(std::max(0, lens.back() + window + pick(-70, 70)));
        }
        Attend a(pick(0, 2), 4, 2, pick(0, 1) ? 64 : 128, lens, n_new, q_pos);
        a.c.window = window;
        a.c.causal = pick(0, 5) != 0;
        for (int u = 0; u < U; ++u) {
            a.k_pos[(size_t)u] = pick(0, 2) ? 0 : pick(0, 30);
            a.q_pos[(size_t)u] += a.k_pos[(size_t)u];
            a.prefix[(size_t)u] = pick(0, 2) ? 0 : pick(0, 400);
        }
        for (int step = 0; step < 40; ++step) {
            if (a.call(ctx) != SPD_OK)
                FAIL("growth: the call fails");
            a.check("walk");
            const int dl = pick(0, 2) ? pick(0, 40) : 0, dq = pick(0, 2) ? pick(0, 40) : 0;
            for (int u = 0; u < U; ++u) {
                a.lens[(size_t)u] += dl;
                a.q_pos[(size_t)u] += dq;
            }
            if (pick(0, 3) == 0) {
                const size_t u = (size_t)pick(0, U - 1);
                a.lens[u] = std::max(1, a.lens[u] + pick(-200, 0));
                a.q_pos[u] = std::max(0, a.lens[u] + a.k_pos[u] + window + pick(-70, 70));
            }
        }
        drop(ctx);
    }
    // a decode loop builds nothing: queries that move on past a prompt that stays, windows before, across and behind its end
    for (int from : {0, 40, 200}) {
        spd_ctx *ctx = make();
        Attend a(SPD_F16, 8, 2, 128, {300, 300}, {1, 2}, {300 + from, 300 + from});
        a.c.window = 60;
        for (int step = 0; step <= 64; ++step) {
            const int before = uploads;
            if (a.call(ctx) != SPD_OK)
                FAIL("loop: the call fails");
            a.check("loop");
            if (step > 0 && uploads != before)
                FAIL("loop from %d: step %d builds its tables again", from, step);
            ++a.q_pos[0], ++a.q_pos[1];
        }
        drop(ctx);
    }
}

// As many views are remembered as the context was told to (argument; 0: not told), by each of the calls that remember any.
static void entries(int told)
{
    SYM(spd_append_tokens);
    spd_ctx *ctx = make();
    const int n = told ? told : 128, users = 20;  // (an append for few users has no table)
    for (int which = 0; which < 2; ++which) {
        auto call = [&](int view) {
            Attend a(SPD_BF16, 4, 2, 64, std::vector<int32_t>(users, 200), std::vector<int32_t>(users, 1), std::vector<int32_t>(users, 199));
            a.ptrs[0] = static_cast<const char *>(kNowhere) + 1024 * view;
            const int before = uploads;
            if (which == 0 ? a.call(ctx) != SPD_OK
                           : spd_append_tokens_(ctx, &a.s, &a.v, a.n_new.data(), nullptr, nullptr, nullptr, 0, nullptr, kNowhere, 128, kNowhere, 128, nullptr) != SPD_OK)
                FAIL("entries: the call fails");
            return uploads - before;
        };
        for (int round = 0; round < 3; ++round)
            for (int i = 0; i < n; ++i)
                if (call(i) != (round == 0))
                    FAIL("call %d, %d views: view %d of round %d", which, n, i, round);
        if (call(n) != 1 || call(n) != 0 || call(0) != 1)  // one more: the one not used for longest goes
            FAIL("call %d: more than %d views", which, n);
    }
    drop(ctx);
}

// Append tables that are used again after the lengths have moved on: every new token goes to its place, and a loop in which all users move on alike
// builds its table once.
static void append()
{
    SYM(spd_append_tokens);
    std::mt19937 rng(9);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    for (int round = 0; round < 60; ++round) {
        spd_ctx *ctx = make();
        const int users = pick(1, 60), mode = round % 4;  // contiguous, a head stride for each user, device pointer tables, pages
        std::vector<int32_t> lens, n_new;
        std::vector<int64_t> head_strides;
        for (int u = 0; u < users; ++u) {
            n_new.push_back(pick(0, 3) ? pick(0, 9) : 0);
            lens.push_back(n_new.back() + pick(0, 200));
            head_strides.push_back(64 * pick(300, 2000));
        }
        Attend a(SPD_F16, 4, 2, 64, lens, n_new, std::vector<int32_t>((size_t)users, 0));
        for (int u = 0; u < users; ++u)
            a.ptrs[(size_t)u] = static_cast<const char *>(kNowhere) + ((int64_t)u << 30);
        if (mode == 1)
            a.v.head_strides = head_strides.data();
        if (mode == 2)
            a.v.k_ptrs_dev = a.v.v_ptrs_dev = a.ptrs.data();
        if (mode == 3) {
            a.v.block_size = 16;
            a.v.k_pool = a.v.v_pool = kNowhere;
            a.v.block_table = static_cast<const int32_t *>(kNowhere);
            a.v.max_blocks = 100;
            a.v.block_stride = 2 * 16 * 64;
        }
        bool alike = false;
        for (int step = 0; step < 20; ++step) {
            const int before = uploads;
            launches.clear();
            if (spd_append_tokens_(ctx, &a.s, &a.v, a.n_new.data(), nullptr, nullptr, nullptr, 0, nullptr, kNowhere, 128, kNowhere, 128, nullptr) != SPD_OK)
                FAIL("append: the call fails");
            if (alike && uploads != before)
                FAIL("append: step %d builds its table again", step);
            int32_t token = 0, user = 0, taken = 0;
            for (const Launch &l : launches)
                for (unsigned i = 0; i < l.grid.x; ++i) {
                    const AppendItem &it = l.append.by_value ? l.given.it[i] : l.append.items[i];
                    while (taken == a.n_new[(size_t)user])
                        ++user, taken = 0;
                    const void *base = l.append.k_pool ? nullptr : l.append.k_ptrs ? l.append.k_ptrs[user] : it.k_base;
                    if (it.user != user || it.token != token || it.count < 1 || it.count > a.n_new[(size_t)user] - taken ||
                        it.place + l.append.grow != a.lens[(size_t)user] - a.n_new[(size_t)user] + taken || (!l.append.k_pool && base != a.ptrs[(size_t)user]) ||
                        it.head_stride != 2 * (mode == 1 ? head_strides[(size_t)user] : a.v.head_stride))
                        FAIL("append: step %d: user %d token %d goes to user %d, %d tokens at %d", step, user, token, it.user, it.count, it.place + l.append.grow);
                    taken += it.count;
                    token += it.count;
                }
            for (int n : a.n_new)
                token -= n;
            if (token != 0)
                FAIL("append: step %d: not every token is taken", step);
            alike = pick(0, 2) != 0;
            const int all = pick(0, 40);
            for (int32_t &l : a.lens)
                l += all;
            if (!alike)
                a.lens[(size_t)pick(0, users - 1)] += pick(1, 20);
        }
        drop(ctx);
    }
}

// Calls of so many workgroups that one launch would pass the runtime's limit of 2^32 threads to a dimension: they go through, and take everything once.
static void limits()
{
    SYM(spd_rotate);
    SYM(spd_append_tokens);
    spd_ctx *ctx = make();
    spd_rope rope = {1, 32, 0, nullptr, static_cast<const float *>(kNowhere), 1.f};
    struct Case {
        int32_t tokens, heads;
    };
    for (const Case &c : {Case{(1 << 26) + 5, 1}, Case{0x7fffffff, 2}, Case{(1 << 24) + 3, 64}, Case{1 << 23, 100}, Case{1000, 3}}) {
        launches.clear();
        const int rc = spd_rotate_(ctx, SPD_BF16, 64, &rope, c.tokens, static_cast<const int32_t *>(kNowhere), c.heads, kNowhere, 64 * c.heads, kNowhere, 64 * c.heads, 0, nullptr);
        if (rc != SPD_OK)
            FAIL("rotation of %d tokens of %d heads: %d", c.tokens, c.heads, rc);
        int64_t next = 0;
        for (const Launch &l : launches) {
            const RotateArgs &a = l.rotate;
            if (a.first != next || a.turn.n_tokens != c.tokens || a.per_group < 1 || a.per_group > kTurnTokens)
                FAIL("rotation of %d tokens: a launch from %d, %lld were taken", c.tokens, a.first, (long long)next);
            next += (int64_t)l.grid.x * a.per_group;
        }
        if (next < c.tokens || next - c.tokens >= launches.back().rotate.per_group)
            FAIL("rotation of %d tokens: %lld are taken", c.tokens, (long long)next);
    }
    {
        const int32_t tokens = (1 << 26) + 9;
        Attend a(SPD_BF16, 1, 1, 64, {tokens + 7}, {tokens}, {0});
        launches.clear();
        const int rc = spd_append_tokens_(ctx, &a.s, &a.v, a.n_new.data(), nullptr, nullptr, nullptr, 0, nullptr, kNowhere, 64, kNowhere, 64, nullptr);
        if (rc != SPD_OK)
            FAIL("append of %d tokens: %d", tokens, rc);
        int64_t next = 0;
        for (const Launch &l : launches)
            for (unsigned i = 0; i < l.grid.x; ++i) {
                const AppendItem &it = l.append.items[i];
                if (it.token != next || it.place + l.append.grow != next + 7 || it.count < 1 || it.count > kTurnTokens)
                    FAIL("append of %d tokens: %d tokens from %d at %d, %lld were taken", tokens, it.count, it.token, it.place + l.append.grow, (long long)next);
                next += it.count;
            }
        if (next != tokens)
            FAIL("append of %d tokens: %lld are taken", tokens, (long long)next);
    }
    {
        const int users = (1 << 18) + 1, heads = 64;
        Attend a(SPD_BF16, heads, heads, 64, std::vector<int32_t>(users, 1), std::vector<int32_t>(users, 1), std::vector<int32_t>(users, 0));
        if (const int rc = a.call(ctx); rc != SPD_OK)
            FAIL("attention of %d users: %d", users, rc);
        std::vector<char> seen((size_t)users * heads, 0);
        for (const Launch &l : launches)
            for (unsigned i = 0; i < l.grid.x; ++i) {
                const TokItem &it = l.attend.items[i];
                if (it.n_rows != 1 || seen[(size_t)it.user * heads + (size_t)it.kv_head]++)
                    FAIL("attention of %d users: user %d head %d is taken twice", users, it.user, it.kv_head);
            }
        for (char x : seen)
            if (!x)
                FAIL("attention of %d users: a row is not taken", users);
    }
    drop(ctx);
}

int main(int argc, char **argv)
{
    const std::string what = argc > 2 ? argv[2] : "";
    lib = argc > 2 ? dlopen(argv[1], RTLD_NOW) : nullptr;
    if (!lib)
        FAIL("tokens_calls <library> growth | append | limits | entries <number>");
    if (what == "growth")
        growth();
    else if (what == "limits")
        limits();
    else if (what == "append")
        append();
    else if (what == "entries" && argc == 4)
        entries(std::atoi(argv[3]));
    else
        FAIL("no such part");
    std::printf("ok\n");
    return 0;
}
