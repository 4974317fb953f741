// A tree of drafted tokens from its parents: every token's branch as a set of bits, its depth and its position.  A few bytes a token: bound by the
// launch and by the chain of dependent reads.
//
// branch(i) = {i} u branch(parent(i)), by doubling: with jump_k(i) the 2^k-th parent, sets grow as s(i) |= s(jump_k(i)), k = 0, 1, ..., until no
// token has such a parent: log2 of the depth steps instead of its number.  Sets only ever gain members of the branch, so it does not matter
// whether a step reads another token's set before or after that one's own step.  The depth is the set's size less one.
// Measured: one user's 13 tokens 1.4 us (a call 6: the host's), 256 users' 100-500 tokens in sets of eight words 8.8 us, one workgroup to a unit: its chain of steps,
// a barrier each with LDS reads between them (two barriers a step: 10.1; a word of the sets to a wave, token after token: 12 us for 128 users).
#pragma once
#include "common.hpp"

namespace spd {

struct PlanUser {
    int32_t token, n, first;  // its first token among all, how many, the position of tokens without a parent
};
// Users travel with a launch's arguments, which cost the host by their size: few or many.
constexpr int kPlanUsers = 256, kPlanFew = 16;
template <int N>
struct PlanUsers {
    PlanUser it[N];
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
template <int N>
__global__ __launch_bounds__(64) void plan_small_kernel(const PlanArgs a, const PlanUsers<N> users)
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

// More tokens, up to `MOST` words of sets in all: every word of every set is a thread's, four or sixteen to a thread; the sets wait in LDS in the order in
// which they are written.
constexpr int kPlanThreads = 1024;
template <int MOST, int N>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(const PlanArgs a, const PlanUsers<N> users)
{
    constexpr int kMine = MOST / kPlanThreads;
    __shared__ uint64_t sets[MOST];
    __shared__ int16_t jumps[2][64 * SPD_MAX_TREE_WORDS];
    __shared__ int more[16];  // for every step: whether some token still has a jump (a tree of 2^10 tokens takes eleven steps at most)
    const PlanUser u = users.it[blockIdx.x];
    const int tid = threadIdx.x, W = a.words, n = u.n, n_sets = n * W;  // (n is at most kPlanThreads)
    int mine = tid < n ? plan_parent(a, u, tid) : -1;
    if (tid < n)
        jumps[0][tid] = (int16_t)mine;
    int token[kMine];
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
        const int e = m * kPlanThreads + tid;
        token[m] = e / W;
        const int word = e - token[m] * W;
        if (e < n_sets)
            sets[e] = token[m] >> 6 == word ? 1ull << (token[m] & 63) : 0ull;
        token[m] = e < n_sets ? token[m] : -1;
    }
    if (tid < 16)
        more[tid] = 0;
    __syncthreads();
    for (int step = 0, now = 0;; ++step, now ^= 1) {
        if (__builtin_amdgcn_ballot_w64(mine >= 0) != 0 && (tid & 63) == 0)
            more[step] = 1;
        __syncthreads();  // (the step before this one is done everywhere, too)
        if (more[step] == 0)
            break;
        uint64_t other[kMine];
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int e = m * kPlanThreads + tid, j = token[m] >= 0 ? jumps[now][token[m]] : -1;
            other[m] = j >= 0 ? sets[e - (token[m] - j) * W] : 0ull;
        }
        mine = mine >= 0 ? jumps[now][mine] : -1;
        if (tid < n)
            jumps[now ^ 1][tid] = (int16_t)mine;
#pragma unroll
        for (int m = 0; m < kMine; ++m)
            if (other[m])
                sets[m * kPlanThreads + tid] |= other[m];
    }
    uint64_t *const out = a.seen + (int64_t)u.token * W;
#pragma unroll
    for (int m = 0; m < kMine; ++m)
        if (token[m] >= 0)
            out[m * kPlanThreads + tid] = sets[m * kPlanThreads + tid];
    if (tid >= n)
        return;
    int depth = -1;
    for (int w = 0; w < W; ++w)
        depth += __builtin_popcountll(sets[tid * W + w]);
    a.depth[u.token + tid] = depth;
    if (a.positions)
        a.positions[u.token + tid] = u.first + depth;
}

}  // namespace spd
