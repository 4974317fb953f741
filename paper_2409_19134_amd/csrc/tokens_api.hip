// Host side of the calls for several tokens per user: tables and scratch memory of a context, launches, the C entry points; and the kernels
// that turn, append and join.
#include <hip/hip_runtime.h>

#include <new>

#include "context.hpp"
#include "rotary.hpp"
#include "schedule_key.hpp"
#include "tokens_schedule.hpp"

namespace spd {

// Joins the partials of a tile's rows (Theorem 1, n-way) in the order of the keys.  GROUPS groups of D / 4 lanes share a row's partials
// (and are added up through LDS): eight where there are many, else a group takes a row of its own.  A launch of its own, 4-5 us: joined by a tile's last
// workgroup instead, whose partials must then pass through memory that all XCDs see, the attention of 16 users' tokens took 35.5 us (33.3 with this),
// of 24 users' six tokens 90.5 (85.2).
template <int DT, int D, int GROUPS>
__global__ __launch_bounds__(256) void tokens_join_kernel(const TokArgs a, const TokJoin *joins, int tile_rows)
{
    constexpr int kLanes = D / 4, kAll = 256 / kLanes, kRowsPerBlock = kAll / GROUPS;
    __shared__ __attribute__((aligned(16))) float part[GROUPS > 1 ? kAll : 1][D];
    __shared__ float part_w[GROUPS > 1 ? kAll : 1];
    const TokJoin j = scalar_load(joins, blockIdx.x);
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    const int row = blockIdx.y * kRowsPerBlock + group / GROUPS, mine = group % GROUPS;
    const bool live = row < j.n_rows;
    const int64_t first = (int64_t)j.slot * tile_rows + min(row, j.n_rows - 1);
    float m = -INFINITY;
    for (int c = lane; c < j.n_chunks; c += kLanes)
        m = fmaxf(m, a.part_lse[first + (int64_t)c * tile_rows].x);
#pragma unroll
    for (int x = 1; x < kLanes; x *= 2)
        m = fmaxf(m, __shfl_xor(m, x));
    const float m_use = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int c = mine; c < j.n_chunks; c += GROUPS) {
        const float lse2 = a.part_lse[first + (int64_t)c * tile_rows].x;
        const f32x4 v = *reinterpret_cast<const f32x4 *>(a.part_o + (first + (int64_t)c * tile_rows) * D + lane * 4);
        const float w = fast_exp2(lse2 - m_use);  // (a stretch without keys of this row holds zeros; a vanishing weight keeps what is not finite)
        sum += w;
        o += w * v;
    }
    if constexpr (GROUPS > 1) {
        *reinterpret_cast<f32x4 *>(&part[group][lane * 4]) = o;
        if (lane == 0)
            part_w[group] = sum;
        __syncthreads();
        if (mine != 0)
            return;
        for (int g = 1; g < GROUPS; ++g) {
            o += *reinterpret_cast<const f32x4 *>(&part[group + g][lane * 4]);
            sum += part_w[group + g];
        }
    }
    if (!live)
        return;
    const TokUser u = scalar_load(a.users, j.user);
    const int r = j.row0 + row, token = r / a.G, head = j.kv_head * a.G + (r - token * a.G);
    const int64_t at = (int64_t)(u.tok0 + token) * a.Hq + head;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    store4<DT>(a, at * D + lane * 4, sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * inv);
    if (lane == 0)
        a.lse[at] = sum == 0.f ? -INFINITY : (m_use + fast_log2(sum)) * kLn2 + a.part_lse[first].y;
}

__global__ __launch_bounds__(256) void tokens_upload_kernel(const u32x4 *__restrict__ src, u32x4 *__restrict__ dst, unsigned n16)
{
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    if (i < n16)
        dst[i] = src[i];
}

// A table on the device, remembered by the bytes that determine it.
struct TokEntry {
    bool valid = false, kept = false;  // kept: a recorded graph reads it
    uint64_t hash = 0, last_use = 0;
    std::vector<uint8_t> key;
    std::vector<int32_t> lens, q_pos;  // attention: what may have grown since
    char *dev = nullptr, *pinned = nullptr;
    size_t capacity = 0;
    bool in_slab = false;
    hipEvent_t uploaded = nullptr;
    hipStream_t last_stream = nullptr;
    // attention
    size_t off_items[host::kTokKernels] = {}, off_joins[host::kTokKernels] = {};
    int64_t n_items[host::kTokKernels] = {}, n_joins[host::kTokKernels] = {}, slots[host::kTokKernels] = {};
    int join_rows[host::kTokKernels] = {}, join_chunks[host::kTokKernels] = {};
    bool growable = false, following = false;  // as in TokTables
    // append
    int64_t n_append = 0;
};

struct TokensState {
    std::vector<TokEntry> entries[2];  // attention, append
    char *slab_dev[2] = {nullptr, nullptr}, *slab_pinned[2] = {nullptr, nullptr};
    uint64_t tick = 0;
    size_t latest = 0;          // the attention's entry that the latest call used
    float *part = nullptr;      // scratch memory of the attention: [slots][rows][D], then float2 [slots][rows]
    size_t part_bytes = 0;
    bool part_kept = false;     // a recorded graph uses it: it is not freed when it is outgrown
    std::vector<float *> retired;
    std::vector<uint8_t> key;   // reused from call to call
    std::vector<int32_t> lens, q_pos;
    std::vector<host::TokUserPlan> plan;
};

namespace {

using namespace spd::host;

// A launch takes fewer than 2^32 threads to a dimension: calls of more workgroups (tens of millions of tokens, or of users' heads) go in parts, each
// launch(first, count).  (A multiple of eight: the XCD that a workgroup runs on stays its number's.)
constexpr int64_t kMostGroups = (int64_t)1 << 23;
template <class F>
void in_parts(int64_t groups, F &&launch)
{
    for (int64_t first = 0; first < groups; first += kMostGroups)
        launch(first, (unsigned)std::min(groups - first, kMostGroups));
}

constexpr size_t kSlot = 32 * 1024;

#define SPD_TRY(ctx, call)                                  \
    do {                                                    \
        hipError_t e_ = (call);                             \
        if (e_ != hipSuccess) {                             \
            (ctx)->last_hip = (int)e_;                      \
            return SPD_ERR_HIP;                             \
        }                                                   \
    } while (0)

// The context's device for the length of a call; the thread's own is put back.
struct OnDevice {
    int before = -1;
    hipError_t error;
    explicit OnDevice(int device)
    {
        error = hipGetDevice(&before);
        if (error == hipSuccess && before != device)
            error = hipSetDevice(device);
        else
            before = -1;
    }
    ~OnDevice()
    {
        if (before >= 0)
            (void)hipSetDevice(before);
    }
};

void free_storage(TokEntry &e)
{
    if (e.dev && !e.in_slab)
        (void)hipFree(e.dev);
    if (e.pinned && !e.in_slab)
        (void)hipHostFree(e.pinned);
    e.dev = e.pinned = nullptr;
    e.capacity = 0;
    e.in_slab = false;
}

void free_state(TokensState *t)
{
    for (auto &list : t->entries)
        for (TokEntry &e : list) {
            free_storage(e);
            if (e.uploaded)
                (void)hipEventDestroy(e.uploaded);
        }
    for (int i = 0; i < 2; ++i) {
        if (t->slab_dev[i])
            (void)hipFree(t->slab_dev[i]);
        if (t->slab_pinned[i])
            (void)hipHostFree(t->slab_pinned[i]);
    }
    if (t->part)
        (void)hipFree(t->part);
    for (float *p : t->retired)
        (void)hipFree(p);
    delete t;
}

TokensState *state_of(ContextBase *ctx)
{
    if (!ctx->tokens) {
        TokensState *t = new TokensState();
        try {
            for (auto &list : t->entries)
                list.resize((size_t)ctx->cache_entries);
        } catch (...) {
            delete t;
            throw;
        }
        ctx->tokens = t;
        ctx->tokens_free = free_state;
    }
    return ctx->tokens;
}

// Whether calls on the stream are being recorded.  (An error - the null stream is asked about while another one is being recorded - means that
// this one is not.)
bool recording(hipStream_t stream)
{
    hipStreamCaptureStatus s = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(stream, &s) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    return s != hipStreamCaptureStatusNone;
}

// An entry that a call on `stream` reads.  (Its upload came before an earlier call of the same entry point: calls do not overlap in time, so nothing
// has to be waited for, and nothing is asked of the runtime that a recording would not allow.)
void use_entry(TokensState *t, TokEntry &e, hipStream_t stream, bool in_graph)
{
    e.kept = e.kept || in_graph;
    e.last_use = ++t->tick;
    e.last_stream = stream;
}

// Room for a new table of `bytes` (a multiple of 16): an unused entry, or the one that has not been used for longest and that no graph keeps.
int new_entry(ContextBase *ctx, TokensState *t, int which, size_t bytes, hipStream_t stream, TokEntry **out)
{
    std::vector<TokEntry> &list = t->entries[which];
    size_t idx = list.size();
    for (size_t i = 0; i < list.size(); ++i) {
        const TokEntry &e = list[i];
        if (e.kept)
            continue;
        if (idx == list.size() || (!e.valid && list[idx].valid) || (e.valid == list[idx].valid && e.last_use < list[idx].last_use))
            idx = i;
        if (!e.valid)
            break;
    }
    if (idx == list.size())
        list.emplace_back();
    TokEntry &e = list[idx];
    if (e.valid) {
        // Its last call may still be running: on this stream the upload comes behind it; on another one (which may be gone by now) the device
        // is waited for.  The staging copy is rewritten once its upload has left it.
        if (e.last_stream != stream)
            SPD_TRY(ctx, hipDeviceSynchronize());
        SPD_TRY(ctx, hipEventSynchronize(e.uploaded));
        e.valid = false;
    }
    if (e.capacity < bytes) {
        size_t cap = kSlot;
        while (cap < bytes)
            cap *= 2;
        free_storage(e);
        const size_t slots = (size_t)ctx->cache_entries;
        if (cap == kSlot && idx < slots) {
            if (!t->slab_dev[which])
                SPD_TRY(ctx, hipMalloc(reinterpret_cast<void **>(&t->slab_dev[which]), kSlot * slots));
            if (!t->slab_pinned[which])
                SPD_TRY(ctx, hipHostMalloc(reinterpret_cast<void **>(&t->slab_pinned[which]), kSlot * slots, hipHostMallocDefault));
            e.dev = t->slab_dev[which] + idx * kSlot;
            e.pinned = t->slab_pinned[which] + idx * kSlot;
            e.in_slab = true;
        } else {
            SPD_TRY(ctx, hipMalloc(reinterpret_cast<void **>(&e.dev), cap));
            SPD_TRY(ctx, hipHostMalloc(reinterpret_cast<void **>(&e.pinned), cap, hipHostMallocDefault));
        }
        e.capacity = cap;
    }
    if (!e.uploaded)
        SPD_TRY(ctx, hipEventCreateWithFlags(&e.uploaded, hipEventDisableTiming));
    *out = &e;
    return SPD_OK;
}

// Sends the staged table (by a kernel that reads it over the bus: a copy command would leave the compute queue and come back).
int upload(ContextBase *ctx, TokensState *t, TokEntry &e, size_t bytes, hipStream_t stream)
{
    const unsigned n16 = (unsigned)(bytes / 16);
    hipLaunchKernelGGL(tokens_upload_kernel, dim3((n16 + 255) / 256), dim3(256), 0, stream, reinterpret_cast<const u32x4 *>(e.pinned),
                       reinterpret_cast<u32x4 *>(e.dev), n16);
    SPD_TRY(ctx, hipGetLastError());
    SPD_TRY(ctx, hipEventRecord(e.uploaded, stream));
    e.last_stream = stream;
    e.valid = true;
    e.last_use = ++t->tick;
    return SPD_OK;
}

// A call that would have to build or allocate something while its stream is recorded.
int cannot_record(ContextBase *ctx)
{
    ctx->last_hip = (int)hipErrorStreamCaptureUnsupported;
    return SPD_ERR_HIP;
}

// Writes a key in place: `most` bytes of room, cut to what was written at the end.
struct KeyWriter {
    std::vector<uint8_t> &key;
    uint8_t *at;
    KeyWriter(std::vector<uint8_t> &k, size_t most) : key(k)
    {
        key.resize(most);
        at = key.data();
    }
    template <class T>
    void put(const T &v)
    {
        std::memcpy(at, &v, sizeof v);
        at += sizeof v;
    }
    void done() { key.resize((size_t)(at - key.data())); }
};

// What the tables hold of a user's storage.
constexpr size_t kStorageBytes = 24;
void put_storage(KeyWriter &w, const spd_kv_view *v, int u, bool used)
{
    if (v->block_size != 0)
        return;
    if (v->head_strides)
        w.put(used ? v->head_strides[u] : (int64_t)0);
    if (!v->k_ptrs_dev) {
        w.put(used ? v->k_ptrs[u] : nullptr);
        w.put(used ? v->v_ptrs[u] : nullptr);
    }
}

TokEntry *find(std::vector<TokEntry> &list, const std::vector<uint8_t> &key, uint64_t hash)
{
    for (TokEntry &e : list)
        if (e.valid && e.hash == hash && e.key == key)
            return &e;
    return nullptr;
}

// How far the lengths or positions of the users with tokens have grown since, the same for all: 0 .. kMaxGrow, or -1.
int32_t growth(const std::vector<int32_t> &was, const std::vector<int32_t> &now)
{
    if (was.size() != now.size() || was.empty())
        return -1;
    const int64_t g = (int64_t)now[0] - was[0];
    if (g < 0 || g > kMaxGrow)
        return -1;
    for (size_t i = 1; i < was.size(); ++i)
        if ((int64_t)now[i] - was[i] != g)
            return -1;
    return (int32_t)g;
}

size_t padded(size_t n) { return (n + 255) / 256 * 256; }

int find_or_build(ContextBase *ctx, TokensState *t, const spd_shape *s, const spd_kv_view *v, const spd_score *c, hipStream_t stream, bool in_graph,
                  TokEntry **out, int32_t *grow_len, int32_t *grow_q)
{
    const int causal = c ? c->causal : 0, window = c ? c->window : 0;
    t->lens.clear();
    t->q_pos.clear();
    KeyWriter w(t->key, 64 + (size_t)v->n_users * (12 + kStorageBytes));
    const int32_t head[9] = {s->dtype, s->n_q_heads, s->n_kv_heads, s->head_dim, v->n_users, v->block_size, causal, window,
                             (v->block_size == 0 && v->k_ptrs_dev) ? 1 : 0};
    w.put(head);
    w.put(v->head_stride);
    for (int u = 0; u < v->n_users; ++u) {
        const TokUserPlan &p = t->plan[(size_t)u];
        const bool used = p.n_tok > 0;
        w.put(p.n_tok);
        w.put(used ? p.prefix : 0);
        w.put(used ? p.k_pos : 0);
        put_storage(w, v, u, used && p.len > 0);
        if (used) {
            t->lens.push_back(p.len);
            t->q_pos.push_back(p.q_pos);
        }
    }
    w.done();
    const uint64_t hash = hash_key(t->key.data(), t->key.size());
    TokEntry *grown = nullptr;
    TokEntry &latest = t->entries[0][t->latest];  // (a decode loop asks for the same one every time)
    if (latest.valid && latest.hash == hash && latest.key == t->key && latest.lens == t->lens && latest.q_pos == t->q_pos) {
        *grow_len = *grow_q = 0;
        *out = &latest;
        use_entry(t, latest, stream, in_graph);
        return SPD_OK;
    }
    for (TokEntry &e : t->entries[0]) {
        if (!e.valid || e.hash != hash || e.key != t->key)
            continue;
        const int32_t gl = growth(e.lens, t->lens), gq = growth(e.q_pos, t->q_pos);
        if (gl < 0 || gq < 0 || ((gl || gq) && !(gl > gq ? e.growable : e.following)))
            continue;
        if (grown && gl + gq >= *grow_len + *grow_q)
            continue;
        grown = &e;
        *grow_len = gl;
        *grow_q = gq;
    }
    if (grown) {
        *out = grown;
        t->latest = (size_t)(grown - t->entries[0].data());
        use_entry(t, *grown, stream, in_graph);
        return SPD_OK;
    }
    if (in_graph)
        return cannot_record(ctx);
    TokTables T;
    build_tok_tables(s, v, t->plan, causal, window, ctx->n_cus, T);
    size_t bytes = padded(T.users.size() * sizeof(TokUser)), off_items[kTokKernels], off_joins[kTokKernels];
    for (int k = 0; k < kTokKernels; ++k) {
        off_items[k] = bytes;
        bytes += padded(T.items[k].size() * sizeof(TokItem));
        off_joins[k] = bytes;
        bytes += padded(T.joins[k].size() * sizeof(TokJoin));
    }
    TokEntry *e = nullptr;
    const int rc = new_entry(ctx, t, 0, bytes, stream, &e);
    if (rc != SPD_OK)
        return rc;
    auto copy = [e](size_t at, const auto &list) {
        if (!list.empty())
            std::memcpy(e->pinned + at, list.data(), list.size() * sizeof list[0]);
    };
    copy(0, T.users);
    for (int k = 0; k < kTokKernels; ++k) {
        copy(off_items[k], T.items[k]);
        copy(off_joins[k], T.joins[k]);
        e->off_items[k] = off_items[k];
        e->off_joins[k] = off_joins[k];
        e->n_items[k] = (int64_t)T.items[k].size();
        e->n_joins[k] = (int64_t)T.joins[k].size();
        e->slots[k] = T.slots[k];
        e->join_rows[k] = e->join_chunks[k] = 0;
        for (const TokJoin &j : T.joins[k]) {
            e->join_rows[k] = std::max(e->join_rows[k], (int)j.n_rows);
            e->join_chunks[k] = std::max(e->join_chunks[k], (int)j.n_chunks);
        }
    }
    e->growable = T.growable;
    e->following = T.following;
    e->key = t->key;
    e->hash = hash;
    e->lens = t->lens;
    e->q_pos = t->q_pos;
    *grow_len = *grow_q = 0;
    *out = e;
    t->latest = (size_t)(e - t->entries[0].data());
    return upload(ctx, t, *e, bytes, stream);
}

int ensure_parts(ContextBase *ctx, TokensState *t, size_t bytes, bool in_graph)
{
    if (t->part_bytes < bytes) {
        if (in_graph)
            return cannot_record(ctx);
        float *old = t->part;
        t->part = nullptr;
        t->part_bytes = 0;
        if (old && t->part_kept)
            t->retired.push_back(old);
        else if (old)
            SPD_TRY(ctx, hipFree(old));  // waits for work that may still use it
        t->part_kept = false;
        const size_t cap = bytes + bytes / 4;
        if (hipMalloc(reinterpret_cast<void **>(&t->part), cap) != hipSuccess) {
            (void)hipGetLastError();
            t->part = nullptr;
            return SPD_ERR_WORKSPACE;
        }
        t->part_bytes = cap;
    }
    t->part_kept = t->part_kept || (in_graph && bytes > 0);
    return SPD_OK;
}

template <int DT, int D>
void launch_join(int64_t n, int max_rows, int max_chunks, const TokArgs &a, const TokJoin *joins, int tile_rows, hipStream_t stream)
{
    constexpr int kAll = 256 / (D / 4);
    if (max_chunks > 8)
        hipLaunchKernelGGL((tokens_join_kernel<DT, D, kAll>), dim3((unsigned)n, (unsigned)max_rows), dim3(256), 0, stream, a, joins, tile_rows);
    else
        hipLaunchKernelGGL((tokens_join_kernel<DT, D, 1>), dim3((unsigned)n, (unsigned)((max_rows + kAll - 1) / kAll)), dim3(256), 0, stream, a, joins,
                           tile_rows);
}
template <int DT>
void launch_join(int head_dim, int64_t n, int max_rows, int max_chunks, const TokArgs &a, const TokJoin *joins, int tile_rows, hipStream_t stream)
{
    if (head_dim == 64)
        launch_join<DT, 64>(n, max_rows, max_chunks, a, joins, tile_rows, stream);
    else
        launch_join<DT, 128>(n, max_rows, max_chunks, a, joins, tile_rows, stream);
}

int attend(ContextBase *ctx, const spd_shape *s, const void *q, int64_t q_stride, const spd_kv_view *v, const int32_t *n_new, const spd_score *c,
           void *out, int32_t out_dtype, float *lse, hipStream_t stream)
{
    int rc = validate_tokens(s, q, q_stride, v, n_new, c, out, out_dtype, lse);
    if (rc != SPD_OK)
        return rc;
    int64_t total = 0;
    for (int u = 0; u < v->n_users; ++u)
        total += n_new[u];
    if (total == 0)
        return SPD_OK;
    const OnDevice on(ctx->device);
    SPD_TRY(ctx, on.error);
    TokensState *t = state_of(ctx);
    plan_users(v, n_new, c, t->plan);
    const bool in_graph = recording(stream);
    TokEntry *e = nullptr;
    int32_t grow_len = 0, grow_q = 0;
    rc = find_or_build(ctx, t, s, v, c, stream, in_graph, &e, &grow_len, &grow_q);
    if (rc != SPD_OK)
        return rc;
    size_t rows[kTokKernels], part_rows = 0;
    for (int k = 0; k < kTokKernels; ++k) {
        rows[k] = part_rows;
        part_rows += (size_t)e->slots[k] * (size_t)tile_rows((TokKernel)k);
    }
    rc = ensure_parts(ctx, t, part_rows * ((size_t)s->head_dim * sizeof(float) + sizeof(float2)), in_graph);
    if (rc != SPD_OK)
        return rc;

    const int es = elt_size(s->dtype);
    const bool paged = v->block_size != 0;
    TokArgs a = {};
    a.users = reinterpret_cast<const TokUser *>(e->dev);
    a.q = static_cast<const char *>(q);
    a.q_stride = q_stride * es;
    if (paged) {
        a.k_pool = static_cast<const char *>(v->k_pool);
        a.v_pool = static_cast<const char *>(v->v_pool);
        a.block_table = v->block_table;
        a.max_blocks = v->max_blocks;
        a.page_shift = page_shift(v->block_size);
        a.block_stride = v->block_stride * es;
    } else {
        a.k_ptrs = reinterpret_cast<const char *const *>(v->k_ptrs_dev);
        a.v_ptrs = reinterpret_cast<const char *const *>(v->v_ptrs_dev);
    }
    a.token_stride = v->token_stride * es;
    a.Hq = s->n_q_heads;
    a.G = s->n_q_heads / s->n_kv_heads;
    a.grow_len = grow_len;
    a.grow_q = grow_q;
    a.out = static_cast<char *>(out);
    a.out_f32 = out_dtype == SPD_F32;
    a.lse = lse;
    ScoreArgs &sc = a.score;
    const float scale = std::fabs(s->scale);
    sc.c = scale == 0.f ? 1.f : scale * kLog2e;
    sc.q_and = scale == 0.f ? 0u : 0xffffffffu;
    sc.q_xor = s->scale < 0.f ? (s->dtype == SPD_F32 ? 0x80000000u : 0x80008000u) : 0u;
    if (c) {
        sc.cap_in = c->cap > 0.f ? scale / c->cap : 0.f;
        sc.cap_out = c->cap > 0.f ? c->cap * kLog2e : 0.f;
        sc.slopes = c->slopes;
        sc.ranges = c->ranges;
        sc.causal = c->causal;
        sc.window = c->window;
    }
    const bool modified = sc.cap_out != 0.f || sc.slopes;
    float2 *const part_lse = reinterpret_cast<float2 *>(t->part + part_rows * (size_t)s->head_dim);
    for (int k = 0; k < kTokKernels; ++k) {
        if (e->n_items[k] == 0)
            continue;
        const int cap = tile_rows((TokKernel)k);
        const TokItem *const items = reinterpret_cast<const TokItem *>(e->dev + e->off_items[k]);
        a.part_o = t->part + rows[k] * (size_t)s->head_dim;
        a.part_lse = part_lse + rows[k];
        in_parts(e->n_items[k], [&](int64_t first, unsigned n) {
            a.items = items + first;
            if (k == (int)TokKernel::kMany)
                launch_tokens_many(s->dtype, s->head_dim, modified, n, a, stream);
            else
                launch_tokens_few(s->dtype, s->head_dim, paged, cap, modified, n, a, stream);
        });
        SPD_TRY(ctx, hipGetLastError());
        if (e->n_joins[k] == 0)
            continue;
        const TokJoin *joins = reinterpret_cast<const TokJoin *>(e->dev + e->off_joins[k]);
        in_parts(e->n_joins[k], [&](int64_t first, unsigned n) {
            if (s->dtype == SPD_F32)
                launch_join<SPD_F32>(s->head_dim, n, e->join_rows[k], e->join_chunks[k], a, joins + first, cap, stream);
            else if (s->dtype == SPD_BF16)
                launch_join<SPD_BF16>(s->head_dim, n, e->join_rows[k], e->join_chunks[k], a, joins + first, cap, stream);
            else
                launch_join<SPD_F16>(s->head_dim, n, e->join_rows[k], e->join_chunks[k], a, joins + first, cap, stream);
        });
        SPD_TRY(ctx, hipGetLastError());
    }
    return SPD_OK;
}

TurnArgs turn_args(const spd_rope *r, const int32_t *positions, int64_t n_tokens, bool transposed)
{
    TurnArgs a = {};
    if (!r)
        return a;
    a.positions = positions;
    a.inv_freq = r->inv_freq;
    a.n_tokens = (int32_t)n_tokens;
    a.n_pairs = r->n_pairs;
    a.amplitude = r->amplitude;
    a.sign = transposed ? -1.f : 1.f;
    if (r->pair_axis)
        for (int j = 0; j < r->n_pairs; ++j)
            a.axis[j / 32] |= (uint64_t)r->pair_axis[j] << (2 * (j % 32));
    return a;
}

// Kernel template arguments from run-time values: f gets integral constants of the type's code, the head's size, whether pairs are adjacent and whether
// the data passes by once.
template <class F>
void with_turn_kernel(int dtype, int head_dim, bool adjacent, bool once, F &&f)
{
    auto by_once = [&](auto dt, auto d, auto adj) {
        if (once)
            f(dt, d, adj, std::true_type());
        else
            f(dt, d, adj, std::false_type());
    };
    auto by_pairs = [&](auto dt, auto d) {
        if (adjacent)
            by_once(dt, d, std::true_type());
        else
            by_once(dt, d, std::false_type());
    };
    auto by_dim = [&](auto dt) {
        if (head_dim == 64)
            by_pairs(dt, std::integral_constant<int, 64>());
        else
            by_pairs(dt, std::integral_constant<int, 128>());
    };
    if (dtype == SPD_F32)
        by_dim(std::integral_constant<int, SPD_F32>());
    else if (dtype == SPD_BF16)
        by_dim(std::integral_constant<int, SPD_BF16>());
    else
        by_dim(std::integral_constant<int, SPD_F16>());
}

// Bytes written by a call from which on they, and what is read, pass the caches by: there is no room for them until they are read (us without / with: the
// video 75.3 / 69.1, the prompts' 125 MB 56.8 / 51.2; the 31 MB of fp32, still in the last cache when they come up again, 10.9 / 13.7).
constexpr int64_t kOnceBytes = (int64_t)64 << 20;

// Tokens of a workgroup: one each until every unit has several workgroups, then about 12 KB of them (us with one / two / four: a video's 20240 tokens
// of 10 KB 68.4 / 72.2 / 77.3, 5003 tokens of 6 KB in fp32 11.9 / 11.1 / 10.7, prompts of 6 KB a token appended 56.0 / 47.3 / 47.1).
int tokens_per_group(int64_t tokens, int64_t token_bytes, int n_cus)
{
    return tokens <= 8 * (int64_t)n_cus ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(kTurnTokens, 12288 / token_bytes));
}

int append(ContextBase *ctx, const spd_shape *s, const spd_kv_view *v, const int32_t *n_new, const spd_rope *rope, const int32_t *positions,
           const void *q, int64_t q_stride, void *q_out, const void *k, int64_t k_stride, const void *v_new, int64_t v_stride, hipStream_t stream)
{
    int rc = validate_append(s, v, n_new, rope, positions, q, q_stride, q_out, k, k_stride, v_new, v_stride);
    if (rc != SPD_OK)
        return rc;
    int64_t total = 0;
    for (int u = 0; u < v->n_users; ++u)
        total += n_new[u];
    if (total == 0)
        return SPD_OK;
    const OnDevice on(ctx->device);
    SPD_TRY(ctx, on.error);
    const int es = elt_size(s->dtype);
    const int64_t token_bytes = (int64_t)((q ? s->n_q_heads : 0) + 2 * s->n_kv_heads) * s->head_dim * es;
    const int group = tokens_per_group(total, token_bytes, ctx->n_cus);
    const bool paged = v->block_size != 0;
    AppendArgs a = {};
    a.turn = turn_args(rope, positions, total, false);
    a.q = static_cast<const char *>(q);
    a.k = static_cast<const char *>(k);
    a.v = static_cast<const char *>(v_new);
    a.q_out = static_cast<char *>(q_out);
    a.q_stride = q_stride * es;
    a.k_stride = k_stride * es;
    a.v_stride = v_stride * es;
    if (paged) {
        a.k_pool = static_cast<char *>(const_cast<void *>(v->k_pool));
        a.v_pool = static_cast<char *>(const_cast<void *>(v->v_pool));
        a.block_table = v->block_table;
        a.max_blocks = v->max_blocks;
        a.page_shift = page_shift(v->block_size);
        a.block_stride = v->block_stride * es;
    } else {
        a.k_ptrs = reinterpret_cast<char *const *>(const_cast<void *const *>(reinterpret_cast<const void *const *>(v->k_ptrs_dev)));
        a.v_ptrs = reinterpret_cast<char *const *>(const_cast<void *const *>(reinterpret_cast<const void *const *>(v->v_ptrs_dev)));
    }
    a.token_stride = v->token_stride * es;
    a.Hq = s->n_q_heads;
    a.Hkv = s->n_kv_heads;
    // Places are kept relative to the first user's, so that a decode loop's table serves all its steps.
    int first = 0;
    while (n_new[first] == 0)
        ++first;
    const int32_t base = v->lens[first] - n_new[first];
    a.grow = base;
    int64_t n_items = 0;
    for (int u = 0; u < v->n_users; ++u)
        n_items += (n_new[u] + group - 1) / group;
    auto fill = [&](AppendItem *it) {
        int32_t token = 0;
        for (int u = 0; u < v->n_users; ++u)
            for (int32_t i = 0; i < n_new[u]; i += group, ++it) {
                AppendItem x = {};
                if (!paged && !v->k_ptrs_dev) {
                    x.k_base = static_cast<char *>(const_cast<void *>(v->k_ptrs[u]));
                    x.v_base = static_cast<char *>(const_cast<void *>(v->v_ptrs[u]));
                }
                x.head_stride = (v->head_strides && !paged ? v->head_strides[u] : v->head_stride) * es;
                x.user = u;
                x.token = token;
                x.place = v->lens[u] - n_new[u] + i - base;
                x.count = std::min(group, n_new[u] - i);
                token += x.count;
                *it = x;
            }
    };
    AppendItems given;
    const AppendItem *items = nullptr;
    if (n_items <= kAppendByValue) {
        fill(given.it);
        a.by_value = 1;
    } else {
        TokensState *t = state_of(ctx);
        const bool in_graph = recording(stream);
        KeyWriter w(t->key, 64 + (size_t)v->n_users * (8 + kStorageBytes));
        const int32_t head[5] = {s->dtype, v->n_users, v->block_size, group, (!paged && v->k_ptrs_dev) ? 1 : 0};
        w.put(head);
        w.put(v->head_stride);
        for (int u = 0; u < v->n_users; ++u) {
            w.put(n_new[u]);
            w.put(n_new[u] > 0 ? v->lens[u] - base : 0);
            put_storage(w, v, u, n_new[u] > 0);
        }
        w.done();
        const uint64_t hash = hash_key(t->key.data(), t->key.size());
        TokEntry *e = find(t->entries[1], t->key, hash);
        if (e) {
            use_entry(t, *e, stream, in_graph);
        } else if (in_graph) {
            rc = cannot_record(ctx);
        } else {
            const size_t bytes = padded((size_t)n_items * sizeof(AppendItem));
            rc = new_entry(ctx, t, 1, bytes, stream, &e);
            if (rc == SPD_OK) {
                fill(reinterpret_cast<AppendItem *>(e->pinned));
                e->n_append = n_items;
                e->key = t->key;
                e->hash = hash;
                rc = upload(ctx, t, *e, bytes, stream);
            }
        }
        if (rc != SPD_OK)
            return rc;
        items = reinterpret_cast<const AppendItem *>(e->dev);
    }
    const bool once = total * token_bytes >= kOnceBytes;
    with_turn_kernel(s->dtype, s->head_dim, rope && rope->adjacent, once, [&](auto dt, auto d, auto adjacent, auto once) {
        in_parts(n_items, [&](int64_t first, unsigned n) {
            a.items = items ? items + first : nullptr;
            hipLaunchKernelGGL((append_kernel<dt(), d(), adjacent(), once()>), dim3(n), dim3(256), 0, stream, a, given);
        });
    });
    SPD_TRY(ctx, hipGetLastError());
    return SPD_OK;
}

}  // namespace
}  // namespace spd

extern "C" {

int spd_validate_rotate(int32_t dtype, int32_t head_dim, const spd_rope *rope, int32_t n_tokens, const int32_t *positions, int32_t n_heads,
                        const void *x, int64_t x_token_stride, const void *y, int64_t y_token_stride)
{
    return spd::host::validate_rotate(dtype, head_dim, rope, n_tokens, positions, n_heads, x, x_token_stride, y, y_token_stride);
}

int spd_validate_append(const spd_shape *shape, const spd_kv_view *view, const int32_t *n_new, const spd_rope *rope, const int32_t *positions,
                        const void *q, int64_t q_token_stride, const void *q_out, const void *k_new, int64_t k_token_stride, const void *v_new,
                        int64_t v_token_stride)
{
    return spd::host::validate_append(shape, view, n_new, rope, positions, q, q_token_stride, q_out, k_new, k_token_stride, v_new, v_token_stride);
}

int spd_validate_tokens(const spd_shape *shape, const void *q, int64_t q_token_stride, const spd_kv_view *view, const int32_t *n_new,
                        const spd_score *score, const void *out, int32_t out_dtype, const float *lse)
{
    return spd::host::validate_tokens(shape, q, q_token_stride, view, n_new, score, out, out_dtype, lse);
}

int spd_rotate(spd_ctx *ctx, int32_t dtype, int32_t head_dim, const spd_rope *rope, int32_t n_tokens, const int32_t *positions, int32_t n_heads,
               const void *x, int64_t x_token_stride, void *y, int64_t y_token_stride, int32_t transposed, void *hip_stream)
{
    using namespace spd;
    if (!ctx)
        return SPD_ERR_NULL;
    const int rc = host::validate_rotate(dtype, head_dim, rope, n_tokens, positions, n_heads, x, x_token_stride, y, y_token_stride);
    if (rc != SPD_OK || n_tokens == 0)
        return rc;
    if (transposed != 0 && transposed != 1)
        return SPD_ERR_SHAPE;
    ContextBase *c = context_base(ctx);
    const OnDevice on(c->device);
    SPD_TRY(c, on.error);
    const int es = host::elt_size(dtype);
    RotateArgs a = {};
    a.turn = turn_args(rope, positions, n_tokens, transposed != 0);
    a.x = static_cast<const char *>(x);
    a.y = static_cast<char *>(y);
    a.x_stride = x_token_stride * es;
    a.y_stride = y_token_stride * es;
    a.n_heads = n_heads;
    const int64_t token_bytes = (int64_t)n_heads * head_dim * es;
    a.per_group = tokens_per_group(n_tokens, token_bytes, c->n_cus);
    const int64_t groups = ((int64_t)n_tokens + a.per_group - 1) / a.per_group;
    const bool once = n_tokens * token_bytes >= kOnceBytes;
    with_turn_kernel(dtype, head_dim, rope->adjacent != 0, once, [&](auto dt, auto d, auto adjacent, auto once) {
        in_parts(groups, [&](int64_t first, unsigned n) {
            a.first = (int32_t)(first * a.per_group);
            hipLaunchKernelGGL((rotate_kernel<dt(), d(), adjacent(), once()>), dim3(n), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
        });
    });
    SPD_TRY(c, hipGetLastError());
    return SPD_OK;
}

int spd_append_tokens(spd_ctx *ctx, const spd_shape *shape, const spd_kv_view *view, const int32_t *n_new, const spd_rope *rope,
                      const int32_t *positions, const void *q, int64_t q_token_stride, void *q_out, const void *k_new, int64_t k_token_stride,
                      const void *v_new, int64_t v_token_stride, void *hip_stream)
try {
    if (!ctx)
        return SPD_ERR_NULL;
    return spd::append(spd::context_base(ctx), shape, view, n_new, rope, positions, q, q_token_stride, q_out, k_new, k_token_stride, v_new,
                       v_token_stride, static_cast<hipStream_t>(hip_stream));
} catch (...) {  // a failed host allocation: no C++ exception leaves the library
    return SPD_ERR_NOMEM;
}

int spd_partial_attn_tokens(spd_ctx *ctx, const spd_shape *shape, const void *q, int64_t q_token_stride, const spd_kv_view *view,
                            const int32_t *n_new, const spd_score *score, void *out, int32_t out_dtype, float *lse, void *hip_stream)
try {
    if (!ctx)
        return SPD_ERR_NULL;
    return spd::attend(spd::context_base(ctx), shape, q, q_token_stride, view, n_new, score, out, out_dtype, lse,
                       static_cast<hipStream_t>(hip_stream));
} catch (...) {
    return SPD_ERR_NOMEM;
}

}  // extern "C"
