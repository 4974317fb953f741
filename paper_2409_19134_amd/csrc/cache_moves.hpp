// Moves within caches: tokens that are kept move together in place, pages are copied.  Bound by the bytes that are moved (read and written together 5.8 TB/s
// past the caches, 4.6-4.9 through them), small calls by the launch and a chain of dependent reads (the count, the list, the page table, the keys).
#pragma once
#include "common.hpp"

namespace spd {

typedef __attribute__((address_space(1))) char global_char;  // (an address that came from memory: not one of LDS)
typedef __attribute__((address_space(1))) u32x4 global_u32x4;
typedef __attribute__((address_space(1))) const int32_t global_i32;

struct KeepUser {
    int64_t head_stride;      // bytes
    int32_t user, token;      // its number, and its first entry of the list
    int32_t begin, n;         // the place that entry 0 means, and how many places there are
};
// Users and layers travel with a launch's arguments, which cost the host by their size: few or many.  (Users times layers, K and V, heads and slices: a
// stream's number keeps to 32 bits.)
constexpr int kKeepUsers = 64, kKeepFew = 16;
template <int N>
struct KeepUsers {
    KeepUser it[N];
};
struct KeepLayer {
    char *kv[2];              // paged: the pools; else arrays of the users' buffers, on the device
    const int32_t *table;     // paged: [users][max_blocks], a width of its own for every layer
    int32_t max_blocks;
};
// A user's row of a layer's block table.
__host__ __device__ __forceinline__ const int32_t *keep_row(const KeepLayer &l, int user) { return l.table + (int64_t)user * l.max_blocks; }
constexpr int kKeepLayers = 32, kKeepFewLayers = 8;
template <int N>
struct KeepLayers {
    KeepLayer it[N];
};

struct KeepArgs {
    const int32_t *keep, *n_keep;
    int64_t token_stride, block_stride;  // bytes
    int32_t page_shift;
    int32_t n_heads, n_layers, slices;
    uint32_t first, n_streams;           // the launch's first stream's number, and how many there are
};

// Tokens kept, in place.  A stream is a slice of the channels of one head of K or V of one user and layer.  WAVES waves have it to themselves and go through
// the kept tokens in order, some at a time: all of them are read before any is written.  Place i gets what lay at keep[i] >= i: later entries
// are read at or behind their own places, so never where earlier ones were written, and nothing has to be asked of other workgroups.
// Measured: 4700 of 14000 tokens each of three users, two layers of 8 heads of 64, fp16, 84 MB read and written: 23 us, 3.6 TB/s, with sixteen waves to a stream and two slices
// of a row; with one wave 199.  (96 streams of K and V: more waves keep more reads in flight, and the slices of a row on one XCD share its cache lines, 30 us otherwise.)  The
// next reads under way while these are written: no gain.  The accepted 1-6 of 26 tokens of 32 users in eight layers, 3.7 MB: 4.5 us, one wave to a
// stream with two reads each (eight: 5.4, sixteen: 8.3).
template <int RB, bool PAGED, int WAVES, int USERS, int LAYERS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void keep_kernel(const KeepArgs a, const KeepUsers<USERS> users, const KeepLayers<LAYERS> layers)
{
    constexpr int kLoads = WAVES == 1 ? (RB > 256 ? 4 : 2) : 8;
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    uint32_t id = a.first + (WAVES == 1 ? blockIdx.x * 4u + (uint32_t)wave : blockIdx.x);
    int slice;
    if constexpr (WAVES == 1) {
        slice = (int)(id % (uint32_t)a.slices);
        id /= (uint32_t)a.slices;
    } else {  // (workgroups i and i + 8 run on one XCD: the slices of a cache line meet in its L2)
        const uint32_t eight = id / (8u * (uint32_t)a.slices), in = id - eight * 8u * (uint32_t)a.slices;
        slice = (int)(in / 8u);
        id = eight * 8u + in % 8u;
    }
    if (id >= a.n_streams)
        return;
    const int head = (int)(id % (uint32_t)a.n_heads);
    id /= (uint32_t)a.n_heads;
    const int kv = (int)(id & 1u);
    id >>= 1;
    const KeepLayer &layer = layers.it[id % (uint32_t)a.n_layers];
    const KeepUser u = users.it[id / (uint32_t)a.n_layers];
    const int count = uniform(min(max(a.n_keep[u.user], 0), u.n));
    const int pieces = RB / 16 / a.slices, rows = 64 / pieces;  // sixteen bytes to a lane; tokens to a load
    const int64_t lane_off = head * u.head_stride + (slice * pieces + lane % pieces) * 16;
    global_char *base;
    global_i32 *table = nullptr, *const keep = (global_i32 *)(a.keep + u.token);
    if constexpr (PAGED) {
        base = (global_char *)layer.kv[kv] + lane_off;
        table = (global_i32 *)keep_row(layer, u.user);
    } else {
        base = (global_char *)reinterpret_cast<char *const *>(layer.kv[kv])[u.user] + lane_off;
    }
    const int mine = (WAVES == 1 ? 0 : wave * rows) + lane / pieces, step = rows * (WAVES == 1 ? 1 : WAVES);
    auto at = [&](int place) __attribute__((always_inline)) {
        if constexpr (PAGED)
            return (int64_t)table[place >> a.page_shift] * a.block_stride + (int64_t)(place & ((1 << a.page_shift) - 1)) * a.token_stride;
        else
            return (int64_t)place * a.token_stride;
    };
    auto entries = [&](int i0, int (&from)[kLoads]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int i = i0 + j * step + mine;
            const int k = i < count ? keep[i] : -1;
            from[j] = k > i && k < u.n ? k : -1;  // (else in place already, or no such token)
        }
    };
    int from[kLoads];
    entries(0, from);
    for (int i0 = 0; i0 < count; i0 += step * kLoads) {
        u32x4 w[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            if (from[j] >= 0)
                w[j] = *(global_u32x4 *)(base + at(u.begin + from[j]));
        int next[kLoads];
        entries(i0 + step * kLoads, next);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the wave's reads are back before the first write ...
        if constexpr (WAVES > 1)
            __syncthreads();  // ... and all waves'
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            if (from[j] >= 0)
                *(global_u32x4 *)(base + at(u.begin + i0 + j * step + mine)) = w[j];
            from[j] = next[j];
        }
    }
}

constexpr int kPageLayers = 64, kPageFewLayers = 8;
template <int N>
struct PageLayers {
    char *kv[N][2];
};
struct PageArgs {
    const int32_t *pairs, *n_tokens;     // n_tokens: or nullptr
    int64_t token_stride, head_stride, block_stride;  // bytes
    int32_t n_pages, n_heads, n_layers, page_shift, token_major, parts;
    uint32_t first;                      // the launch's first workgroup's number
};

// Pages copied: a workgroup takes 4 KB of a page of K or V in one layer, sixteen bytes to a thread.  Many small workgroups: with one, two, four and eight
// pieces to a thread 1000 pages of 64 KB each of K and V in two layers take 90, 103, 102 and 134 us (524 MB read and written: 5.8 TB/s with one, past the caches).
// DENSE: a page's bytes lie end to end, tokens in order (or whole pages in any order).  ONCE: past the caches.
constexpr int kPagePieces = 256;
template <int RB, bool DENSE, bool ONCE, int LAYERS>
__global__ __launch_bounds__(256) void copy_pages_kernel(const PageArgs a, const PageLayers<LAYERS> layers)
{
    constexpr int C = RB / 16;
    uint32_t id = a.first + blockIdx.x;
    const int part = (int)(id % (uint32_t)a.parts);
    id /= (uint32_t)a.parts;
    const int kv = (int)(id & 1u);
    id >>= 1;
    char *const pool = layers.kv[id % (uint32_t)a.n_layers][kv];
    const uint32_t pair = id / (uint32_t)a.n_layers;
    const int from = uniform(a.pairs[2 * (size_t)pair]), to = uniform(a.pairs[2 * (size_t)pair + 1]);
    if ((unsigned)from >= (unsigned)a.n_pages || (unsigned)to >= (unsigned)a.n_pages || from == to)
        return;
    const int page = 1 << a.page_shift, n = a.n_tokens ? uniform(min(max(a.n_tokens[pair], 0), page)) : page;
    const char *const src = pool + from * a.block_stride;
    char *const dst = pool + to * a.block_stride;
    const int first = part * kPagePieces + (int)threadIdx.x;
    auto load = [](const char *p) __attribute__((always_inline)) {
        if constexpr (ONCE)
            return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
        else
            return *reinterpret_cast<const u32x4 *>(p);
    };
    auto store = [](char *p, u32x4 v) __attribute__((always_inline)) {
        if constexpr (ONCE)
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
        else
            *reinterpret_cast<u32x4 *>(p) = v;
    };
    if constexpr (DENSE) {
        if (first < n * a.n_heads * C)
            store(dst + (int64_t)first * 16, load(src + (int64_t)first * 16));
    } else {
        const int row = first / C;
        const int token = a.token_major ? row / a.n_heads : row & (page - 1);
        const int head = a.token_major ? row - token * a.n_heads : row >> a.page_shift;
        const int64_t off = token * a.token_stride + head * a.head_stride + first % C * 16;
        if (token < n && head < a.n_heads)
            store(dst + off, load(src + off));
    }
}

}  // namespace spd
