// A tree of drafted tokens from its parents: every token's branch as a set of bits, its depth and its position.  A few bytes a token: bound by the
// launch and by the chain of dependent reads.
//
// branch(i) = {i} u branch(parent(i)), by doubling: with jump_k(i) the 2^k-th parent, sets grow as s(i) |= s(jump_k(i)), k = 0, 1, ..., until no
// token has such a parent: log2 of the depth steps instead of its number.  Sets only ever gain members of the branch, so it does not matter
// whether a step reads another token's set before or after that one's own step.  The depth is the set's size less one.
#pragma once
#include "common.hpp"

namespace spd {

struct PlanUser {
    int32_t token, n, first;  // its first token among all, how many, the position of tokens without a parent
};
constexpr int kPlanUsers = 128;
struct PlanUsers {
    PlanUser it[kPlanUsers];
};

struct PlanArgs {
    const int32_t *parents;
    uint64_t *seen;
    int32_t *depth, *positions;  // positions: or nullptr
    int32_t words;
};

// A token's parent, or -1: what is not an earlier token's number stands for none.
__device__ __forceinline__ int plan_parent(const PlanArgs &a, const PlanUser &u, int i)
{
    const int p = a.parents[u.token + i];
    return p >= 0 && p < i ? p : -1;
}

// Up to 64 tokens: one to a lane, sets and jumps in registers.
__global__ __launch_bounds__(64) void plan_small_kernel(const PlanArgs a, const PlanUsers users)
{
    const PlanUser u = users.it[blockIdx.x];
    const int i = threadIdx.x;
    const bool live = i < u.n;
    int jump = live ? plan_parent(a, u, i) : -1;
    uint64_t set = 1ull << i;
    while (__builtin_amdgcn_ballot_w64(jump >= 0) != 0) {
        const int from = max(jump, 0);
        const uint64_t other = __shfl(set, from);
        const int next = __shfl(jump, from);
        if (jump >= 0) {
            set |= other;
            jump = next;
        }
    }
    if (!live)
        return;
    const int64_t t = u.token + i;
    uint64_t *const out = a.seen + t * a.words;
    out[0] = set;
    for (int w = 1; w < a.words; ++w)
        out[w] = 0;
    const int depth = __builtin_popcountll(set) - 1;
    a.depth[t] = depth;
    if (a.positions)
        a.positions[t] = u.first + depth;
}

// Up to 64 * SPD_MAX_TREE_WORDS tokens: first every jump table, by all threads, then the waves take the words of the sets in turn; depths are summed over them.
constexpr int kPlanThreads = 512;
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(const PlanArgs a, const PlanUsers users)
{
    constexpr int kMost = 64 * SPD_MAX_TREE_WORDS, kSteps = 10, kWaves = kPlanThreads / 64;
    static_assert(1 << kSteps >= kMost);
    __shared__ int16_t jumps[kSteps][kMost];
    __shared__ uint64_t sets[kWaves][kMost];
    __shared__ int sizes[kMost];
    const PlanUser u = users.it[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n = u.n;
    for (int i = tid; i < n; i += kPlanThreads) {
        jumps[0][i] = (int16_t)plan_parent(a, u, i);
        sizes[i] = 0;
    }
    int steps = 0;  // tables that hold a jump
    for (;;) {
        bool any = false;
        __syncthreads();
        for (int i = tid; i < n; i += kPlanThreads) {
            const int j = jumps[steps][i];
            any = any || j >= 0;
            if (steps + 1 < kSteps)
                jumps[steps + 1][i] = j >= 0 ? jumps[steps][j] : (int16_t)-1;
        }
        if (__syncthreads_or(any) == 0)
            break;
        if (++steps == kSteps)
            break;
    }
    for (int w = wave; w < a.words; w += kWaves) {
        for (int i = lane; i < n; i += 64)
            sets[wave][i] = i >> 6 == w ? 1ull << (i & 63) : 0ull;
        // (the wave's own part of LDS: its reads and writes stay in order)
        for (int k = 0; k < steps; ++k) {
            __builtin_amdgcn_wave_barrier();
            for (int i = lane; i < n; i += 64) {
                const int j = jumps[k][i];
                if (j >= 0)
                    sets[wave][i] |= sets[wave][j];
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        for (int i = lane; i < n; i += 64) {
            const uint64_t s = sets[wave][i];
            a.seen[(int64_t)(u.token + i) * a.words + w] = s;
            if (s)
                atomicAdd(&sizes[i], __builtin_popcountll(s));
        }
    }
    __syncthreads();
    for (int i = tid; i < n; i += kPlanThreads) {
        a.depth[u.token + i] = sizes[i] - 1;
        if (a.positions)
            a.positions[u.token + i] = u.first + sizes[i] - 1;
    }
}

}  // namespace spd
