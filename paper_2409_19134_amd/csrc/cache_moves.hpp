// Moves within caches: tokens that are kept move together in place, pages are copied.  Bound by the bytes that are moved.
#pragma once
#include "common.hpp"

namespace spd {

struct KeepUser {
    int64_t head_stride;      // bytes
    int32_t user, token;      // its number, and its first entry of the list
    int32_t begin, n;         // the place that entry 0 means, and how many places there are
};
constexpr int kKeepUsers = 64;  // (times layers, K and V, heads and slices: a wave's number keeps to 32 bits)
struct KeepUsers {
    KeepUser it[kKeepUsers];
};
struct KeepLayer {
    char *kv[2];              // paged: the pools; else arrays of the users' buffers, on the device
    const int32_t *table;     // paged
};
constexpr int kKeepLayers = 32;
struct KeepLayers {
    KeepLayer it[kKeepLayers];
};

struct KeepArgs {
    const int32_t *keep, *n_keep;
    int64_t token_stride, block_stride;  // bytes
    int32_t max_blocks, page_shift;
    int32_t n_heads, n_layers, slices;
    uint32_t first, n_waves;             // the launch's first wave's number, and how many there are
};

// Tokens kept, in place.  A wave has a slice of the channels of one head of K or V of one user and layer to itself and goes through the kept tokens in
// order, some at a time: all of them are read before any is written.  Place i gets what lay at keep[i] >= i: later entries read at or behind their own
// places, so never where earlier ones have written, and nothing has to be asked of other waves.
template <int RB, bool PAGED>
__global__ __launch_bounds__(256) void keep_kernel(const KeepArgs a, const KeepUsers users, const KeepLayers layers)
{
    constexpr int kLoads = 8;
    const int lane = threadIdx.x & 63;
    uint32_t id = a.first + blockIdx.x * 4u + (uint32_t)uniform((int)(threadIdx.x >> 6));
    if (id >= a.n_waves)
        return;
    const int slice = (int)(id % (uint32_t)a.slices);
    id /= (uint32_t)a.slices;
    const int head = (int)(id % (uint32_t)a.n_heads);
    id /= (uint32_t)a.n_heads;
    const int kv = (int)(id & 1u);
    id >>= 1;
    const KeepLayer &layer = layers.it[id % (uint32_t)a.n_layers];
    const KeepUser &u = users.it[id / (uint32_t)a.n_layers];
    const int count = min(max(a.n_keep[u.user], 0), u.n);
    char *base;
    const int32_t *table = nullptr;
    if constexpr (PAGED) {
        base = layer.kv[kv];
        table = layer.table + (int64_t)u.user * a.max_blocks;
    } else {
        base = reinterpret_cast<char *const *>(layer.kv[kv])[u.user];
    }
    const int pieces = RB / 16 / a.slices, rows = 64 / pieces;  // sixteen bytes to a lane; tokens to a load
    base += head * u.head_stride + (slice * pieces + lane % pieces) * 16;
    const int mine = lane / pieces;
    auto at = [&](int place) __attribute__((always_inline)) {
        if constexpr (PAGED)
            return (int64_t)table[place >> a.page_shift] * a.block_stride + (int64_t)(place & ((1 << a.page_shift) - 1)) * a.token_stride;
        else
            return (int64_t)place * a.token_stride;
    };
    for (int i0 = 0; i0 < count; i0 += rows * kLoads) {
        u32x4 w[kLoads];
        int from[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int i = i0 + j * rows + mine;
            int k = -1;
            if (i < count) {
                k = a.keep[u.token + i];
                if (k <= i || k >= u.n)  // in place already, or no such token
                    k = -1;
            }
            from[j] = k;
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            if (from[j] >= 0)
                w[j] = *reinterpret_cast<const u32x4 *>(base + at(u.begin + from[j]));
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // all lanes' reads are back before the first write
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            if (from[j] >= 0)
                *reinterpret_cast<u32x4 *>(base + at(u.begin + i0 + j * rows + mine)) = w[j];
    }
}

constexpr int kPageLayers = 64;
struct PageLayers {
    char *kv[kPageLayers][2];
};
struct PageArgs {
    const int32_t *pairs, *n_tokens;     // n_tokens: or nullptr
    int64_t token_stride, head_stride, block_stride;  // bytes
    int32_t n_pages, n_heads, n_layers, page_shift, token_major, parts;
    uint32_t first;                      // the launch's first workgroup's number
};
constexpr int kPageLoads = 8, kPagePieces = 256 * kPageLoads;  // sixteen bytes each, of a workgroup

// Pages copied: a workgroup takes 32 KB of a page of K or V in one layer.
template <int RB>
__global__ __launch_bounds__(256) void copy_pages_kernel(const PageArgs a, const PageLayers layers)
{
    constexpr int C = RB / 16;
    uint32_t id = a.first + blockIdx.x;
    const int part = (int)(id % (uint32_t)a.parts);
    id /= (uint32_t)a.parts;
    const int kv = (int)(id & 1u);
    id >>= 1;
    char *const pool = layers.kv[id % (uint32_t)a.n_layers][kv];
    const uint32_t pair = id / (uint32_t)a.n_layers;
    const int from = a.pairs[2 * pair], to = a.pairs[2 * pair + 1];
    if ((unsigned)from >= (unsigned)a.n_pages || (unsigned)to >= (unsigned)a.n_pages || from == to)
        return;
    const int page = 1 << a.page_shift, n = a.n_tokens ? min(max(a.n_tokens[pair], 0), page) : page;
    const char *const src = pool + from * a.block_stride;
    char *const dst = pool + to * a.block_stride;
    u32x4 w[kPageLoads];
    int64_t off[kPageLoads];
#pragma unroll
    for (int j = 0; j < kPageLoads; ++j) {
        const int i = part * kPagePieces + j * 256 + (int)threadIdx.x, row = i / C;
        const int token = a.token_major ? row / a.n_heads : row & (page - 1);
        const int head = a.token_major ? row - token * a.n_heads : row >> a.page_shift;
        off[j] = token < n && head < a.n_heads ? token * a.token_stride + head * a.head_stride + i % C * 16 : -1;
        if (off[j] >= 0)
            w[j] = *reinterpret_cast<const u32x4 *>(src + off[j]);
    }
#pragma unroll
    for (int j = 0; j < kPageLoads; ++j)
        if (off[j] >= 0)
            *reinterpret_cast<u32x4 *>(dst + off[j]) = w[j];
}

}  // namespace spd
