// Argument checks of the calls for several tokens per user, and the tables that their kernels read (host only, no HIP calls).
#pragma once
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <tuple>
#include <utility>
#include <vector>

#include "host_checks.hpp"
#include "tokens.hpp"

namespace spd::host {

constexpr int32_t kMaxPosition = 1 << 30;
constexpr int64_t kMaxStrideBytes = (int64_t)1 << 28;
constexpr int32_t kMaxLayers = 1024;  // views of one call

inline bool token_stride_ok(int64_t stride, int64_t heads, int head_dim, int es)
{
    return stride >= heads * head_dim && stride <= ((int64_t)1 << 40) && (stride * es) % 16 == 0;
}

inline int validate_rope(const spd_rope *r, int head_dim)
{
    if (!r)
        return SPD_ERR_NULL;
    if (r->n_axes < 1 || r->n_axes > 3 || r->n_pairs < 8 || r->n_pairs % 8 != 0 || r->n_pairs > head_dim / 2)
        return SPD_ERR_SHAPE;
    if ((r->adjacent != 0 && r->adjacent != 1) || !std::isfinite(r->amplitude))
        return SPD_ERR_SHAPE;
    if (!r->inv_freq)
        return SPD_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(r->inv_freq) & 3u)
        return SPD_ERR_ALIGN;
    if (r->pair_axis)
        for (int j = 0; j < r->n_pairs; ++j)
            if (r->pair_axis[j] >= r->n_axes)
                return SPD_ERR_SHAPE;
    return SPD_OK;
}

inline int validate_rotate(int32_t dtype, int32_t head_dim, const spd_rope *rope, int32_t n_tokens, const int32_t *positions, int32_t n_heads,
                           const void *x, int64_t x_stride, const void *y, int64_t y_stride)
{
    if (dtype != SPD_F32 && dtype != SPD_BF16 && dtype != SPD_F16)
        return SPD_ERR_SHAPE;
    if (head_dim != 64 && head_dim != 128)
        return SPD_ERR_SHAPE;
    const int rc = validate_rope(rope, head_dim);
    if (rc != SPD_OK)
        return rc;
    if (n_heads < 1 || n_heads > 65535)
        return SPD_ERR_SHAPE;
    if (n_tokens < 0)
        return SPD_ERR_LEN;
    if (n_tokens == 0)
        return SPD_OK;
    if (!positions || !x || !y)
        return SPD_ERR_NULL;
    const int es = elt_size(dtype);
    if (!aligned16(x) || !aligned16(y) || (reinterpret_cast<uintptr_t>(positions) & 3u) || !token_stride_ok(x_stride, n_heads, head_dim, es) ||
        !token_stride_ok(y_stride, n_heads, head_dim, es) || (x == y && x_stride != y_stride))
        return SPD_ERR_ALIGN;
    return SPD_OK;
}

// Counts of new tokens: *total on return.
inline int validate_counts(const spd_shape *s, const spd_kv_view *v, const int32_t *n_new, bool inside_view, int64_t *total)
{
    *total = 0;
    if (v->n_users > 0 && !n_new)
        return SPD_ERR_NULL;
    for (int u = 0; u < v->n_users; ++u) {
        if (n_new[u] < 0 || n_new[u] > kMaxLen || (inside_view && n_new[u] > v->lens[u]))
            return SPD_ERR_LEN;
        *total += n_new[u];
    }
    if (*total * s->n_q_heads > 0x7fffffffll)
        return SPD_ERR_LEN;
    return SPD_OK;
}

inline int validate_append(const spd_shape *s, const spd_kv_view *v, const int32_t *n_new, const spd_rope *rope, const int32_t *positions,
                           const void *q, int64_t q_stride, const void *q_out, const void *k, int64_t k_stride, const void *v_new, int64_t v_stride)
{
    int rc = validate_shape(s);
    if (rc == SPD_OK)
        rc = validate_view(s, v);
    if (rc == SPD_OK && rope)
        rc = validate_rope(rope, s->head_dim);
    int64_t total = 0;
    if (rc == SPD_OK)
        rc = validate_counts(s, v, n_new, true, &total);
    if (rc != SPD_OK || total == 0)
        return rc;
    if ((rope && !positions) || (q != nullptr) != (q_out != nullptr) || !k || !v_new)
        return SPD_ERR_NULL;
    const int es = elt_size(s->dtype);
    if ((reinterpret_cast<uintptr_t>(positions) & 3u) || !aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(v_new))
        return SPD_ERR_ALIGN;
    if ((q && !token_stride_ok(q_stride, s->n_q_heads, s->head_dim, es)) || !token_stride_ok(k_stride, s->n_kv_heads, s->head_dim, es) ||
        !token_stride_ok(v_stride, s->n_kv_heads, s->head_dim, es) || (q && q == q_out && q_stride != (int64_t)s->n_q_heads * s->head_dim))
        return SPD_ERR_ALIGN;
    return SPD_OK;
}

constexpr float kMaxCap = 1e30f;  // cap log2(e) stays finite, and what scale / cap times a product loses below 2^-126 is below 2^-26 of a score

inline int32_t first_key_position(const spd_score *c, int u) { return c && c->k_pos ? c->k_pos[u] : 0; }

// Sets of a tree's tokens: `words` of 64 bits each hold every user's tokens.
inline int validate_tree_counts(int32_t n_users, const int32_t *n_new, int32_t words)
{
    if (words < 1 || words > SPD_MAX_TREE_WORDS)
        return SPD_ERR_SHAPE;
    for (int u = 0; u < n_users; ++u)
        if (n_new[u] > 64 * words)
            return SPD_ERR_LEN;
    return SPD_OK;
}

// tree: nullptr without one.
inline int validate_tokens(const spd_shape *s, const void *q, int64_t q_stride, const spd_kv_view *v, const int32_t *n_new, const spd_score *c,
                           const void *out, int32_t out_dtype, const float *lse, const spd_tree *tree = nullptr)
{
    int rc = validate_shape(s);
    if (rc == SPD_OK)
        rc = validate_view(s, v);
    if (rc != SPD_OK)
        return rc;
    if (out_dtype != SPD_F32 && out_dtype != s->dtype)
        return SPD_ERR_SHAPE;
    // the kernels' products of a token's or page's number and its stride are 32 by 32 bits
    if (v->token_stride > kMaxStrideBytes / elt_size(s->dtype) || (v->block_size != 0 && v->block_stride > kMaxStrideBytes / elt_size(s->dtype)))
        return SPD_ERR_ALIGN;
    if (c && (!(c->cap >= 0.f) || !(c->cap <= kMaxCap) || (c->causal != 0 && c->causal != 1)))
        return SPD_ERR_SHAPE;
    if (c && c->cap > 0.f && s->scale != 0.f) {  // the kernels' factor scale / cap in all its 24 bits, four times it finite
        const float in = std::fabs(s->scale) / c->cap;
        if (!std::isnormal(in) || !std::isfinite(4.f * in))
            return SPD_ERR_SHAPE;
    }
    if (c && (c->window < 0 || c->window > kMaxPosition))
        return SPD_ERR_LEN;
    int64_t total = 0;
    rc = validate_counts(s, v, n_new, !(c && c->q_pos), &total);
    if (rc == SPD_OK && tree)
        rc = validate_tree_counts(v->n_users, n_new, tree->n_words);
    if (rc != SPD_OK)
        return rc;
    for (int u = 0; u < v->n_users; ++u) {
        const int64_t k0 = first_key_position(c, u);
        if (k0 < 0 || k0 + v->lens[u] > kMaxPosition)
            return SPD_ERR_LEN;
        if (c && c->q_pos && (c->q_pos[u] < 0 || (int64_t)c->q_pos[u] + n_new[u] > kMaxPosition))
            return SPD_ERR_LEN;
        if (c && c->prefix && (c->prefix[u] < 0 || c->prefix[u] > kMaxPosition))
            return SPD_ERR_LEN;
    }
    if (c && ((reinterpret_cast<uintptr_t>(c->slopes) & 3u) || (reinterpret_cast<uintptr_t>(c->ranges) & 7u)))
        return SPD_ERR_ALIGN;
    if (total == 0)
        return SPD_OK;
    if (!q || !out || !lse || (tree && (!tree->seen || !tree->depth)))
        return SPD_ERR_NULL;
    if (tree && ((reinterpret_cast<uintptr_t>(tree->seen) & 7u) || (reinterpret_cast<uintptr_t>(tree->depth) & 3u)))
        return SPD_ERR_ALIGN;
    if (!aligned16(q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(lse) & 3u) ||
        !token_stride_ok(q_stride, s->n_q_heads, s->head_dim, elt_size(s->dtype)))
        return SPD_ERR_ALIGN;
    return SPD_OK;
}

inline int validate_tree_plan(int32_t n_users, const int32_t *n_new, const int32_t *parents, const int32_t *first, int32_t words, const uint64_t *seen,
                              const int32_t *depth, const int32_t *positions)
{
    if (n_users < 0)
        return SPD_ERR_LEN;
    if (n_users > 0 && !n_new)
        return SPD_ERR_NULL;
    int64_t total = 0;
    for (int u = 0; u < n_users; ++u) {
        if (n_new[u] < 0)
            return SPD_ERR_LEN;
        total += n_new[u];
    }
    if (total > 0x7fffffffll)
        return SPD_ERR_LEN;
    const int rc = validate_tree_counts(n_users, n_new, words);
    if (rc != SPD_OK)
        return rc;
    if (total == 0)
        return SPD_OK;
    if (!parents || !seen || !depth || (first != nullptr) != (positions != nullptr))
        return SPD_ERR_NULL;
    if (first)
        for (int u = 0; u < n_users; ++u)
            if (first[u] < 0 || (int64_t)first[u] + n_new[u] > kMaxPosition)
                return SPD_ERR_LEN;
    if ((reinterpret_cast<uintptr_t>(seen) & 7u) || ((reinterpret_cast<uintptr_t>(parents) | reinterpret_cast<uintptr_t>(depth) |
                                                       reinterpret_cast<uintptr_t>(positions)) & 3u))
        return SPD_ERR_ALIGN;
    return SPD_OK;
}

// Layers' views that one call takes: alike but for where their caches and block tables lie.
inline int validate_layers(const spd_shape *s, const spd_kv_view *views, int32_t n_views)
{
    int rc = validate_shape(s);
    if (rc != SPD_OK)
        return rc;
    if (n_views < 0 || n_views > kMaxLayers)
        return SPD_ERR_LEN;
    return n_views > 0 && !views ? SPD_ERR_NULL : SPD_OK;
}

// Whether a cache is among the layers' twice (one of K and V counts too): its tokens would move twice.  Pages: the same pool under the same block table (that
// tables which lie apart name other pages is for the caller to see to).  Buffers: the same array of pointers on the device, or the same buffer of a user whose tokens
// move (buffers_twice: the arrays on the device are copies of the host's).
inline bool tables_twice(const spd_kv_view *views, int32_t n_views)
{
    std::pair<const void *, const void *> caches[2 * kMaxLayers];
    auto end = caches;
    for (int i = 0; i < n_views; ++i) {
        const spd_kv_view &v = views[i];
        const bool paged = v.block_size != 0;
        *end++ = paged ? std::make_pair(v.k_pool, (const void *)v.block_table) : std::make_pair((const void *)v.k_ptrs_dev, (const void *)nullptr);
        *end++ = paged ? std::make_pair(v.v_pool, (const void *)v.block_table) : std::make_pair((const void *)v.v_ptrs_dev, (const void *)nullptr);
    }
    std::sort(caches, end);
    return std::adjacent_find(caches, end) != end;
}
inline bool buffers_twice(const spd_kv_view *views, int32_t n_views, const int32_t *n_last)
{
    // A set of addresses, emptied for the next user by the user's number beside each.
    constexpr int kMost = 4 * kMaxLayers;
    const void *place[kMost];
    int32_t owner[kMost];
    int bits = 3;
    while ((1 << bits) < 4 * n_views)
        ++bits;
    std::fill(owner, owner + (1 << bits), -1);
    for (int32_t u = 0; u < views[0].n_users; ++u) {
        if (n_last[u] == 0)
            continue;
        for (int i = 0; i < n_views; ++i)
            for (const void *p : {views[i].k_ptrs[u], views[i].v_ptrs[u]}) {
                uint32_t at = (uint32_t)((uint64_t)reinterpret_cast<uintptr_t>(p) * 0x9e3779b97f4a7c15ull >> (64 - bits));
                for (; owner[at] == u; at = (at + 1) & ((1u << bits) - 1))  // (half of the places are free)
                    if (place[at] == p)
                        return true;
                owner[at] = u;
                place[at] = p;
            }
    }
    return false;
}

// buffers: with the check for buffers that are given twice, which a call that remembers them makes once.
inline int validate_keep(const spd_shape *s, const spd_kv_view *views, int32_t n_views, const int32_t *n_last, const int32_t *keep, const int32_t *n_keep,
                         bool buffers = true)
{
    int rc = validate_layers(s, views, n_views);
    for (int i = 0; rc == SPD_OK && i < n_views; ++i) {
        const spd_kv_view &v = views[i], &v0 = views[0];
        rc = validate_view(s, &v);
        if (rc != SPD_OK || i == 0)
            continue;
        if (v.n_users != v0.n_users || v.block_size != v0.block_size || v.token_stride != v0.token_stride || v.head_stride != v0.head_stride ||
            (v.block_size != 0 && v.block_stride != v0.block_stride) || (v.head_strides != nullptr) != (v0.head_strides != nullptr) ||
            (v.k_ptrs_dev != nullptr) != (v0.k_ptrs_dev != nullptr))
            return SPD_ERR_SHAPE;
        for (int u = 0; u < v.n_users; ++u)
            if (v.lens[u] != v0.lens[u] || (v.head_strides && v.block_size == 0 && v.lens[u] > 0 && v.head_strides[u] != v0.head_strides[u]))
                return SPD_ERR_SHAPE;
    }
    if (rc != SPD_OK || n_views == 0)
        return rc;
    int64_t total = 0;
    rc = validate_counts(s, &views[0], n_last, true, &total);
    if (rc != SPD_OK || total == 0)
        return rc;
    if (!keep || !n_keep)
        return SPD_ERR_NULL;
    const bool paged = views[0].block_size != 0;
    if (((paged || views[0].k_ptrs_dev) && tables_twice(views, n_views)) || (!paged && buffers && buffers_twice(views, n_views, n_last)))
        return SPD_ERR_SHAPE;
    return (reinterpret_cast<uintptr_t>(keep) | reinterpret_cast<uintptr_t>(n_keep)) & 3u ? SPD_ERR_ALIGN : SPD_OK;
}

inline int validate_pages(const spd_shape *s, const spd_kv_view *views, int32_t n_views, int32_t n_pages, int32_t n_pairs, const int32_t *pairs,
                          const int32_t *n_tokens)
{
    const int rc = validate_layers(s, views, n_views);
    if (rc != SPD_OK)
        return rc;
    if (n_pages < 0 || n_pairs < 0)
        return SPD_ERR_LEN;
    const int es = elt_size(s->dtype);
    for (int i = 0; i < n_views; ++i) {
        const spd_kv_view &v = views[i], &v0 = views[0];
        if (page_shift(v.block_size) < 0 || v.block_size != v0.block_size || v.token_stride != v0.token_stride || v.head_stride != v0.head_stride ||
            v.block_stride != v0.block_stride)
            return SPD_ERR_SHAPE;
        if (n_pages == 0 || n_pairs == 0)
            continue;
        if (!v.k_pool || !v.v_pool)
            return SPD_ERR_NULL;
        if (!aligned16(v.k_pool) || !aligned16(v.v_pool) || v.token_stride < s->head_dim || (v.token_stride * es) % 16 != 0 || v.head_stride < 0 ||
            (v.head_stride * es) % 16 != 0 || v.block_stride <= 0 || (v.block_stride * es) % 16 != 0)
            return SPD_ERR_ALIGN;
    }
    if (n_views == 0 || n_pages == 0 || n_pairs == 0)
        return SPD_OK;
    if (!pairs)
        return SPD_ERR_NULL;
    return (reinterpret_cast<uintptr_t>(pairs) & 7u) || (reinterpret_cast<uintptr_t>(n_tokens) & 3u) ? SPD_ERR_ALIGN : SPD_OK;
}

// A user of a call as the schedule sees it: positions relative to the view's first key.
struct TokUserPlan {
    int32_t n_tok = 0, len = 0, q_pos = 0, prefix = 0, k_pos = 0;
};

inline void plan_users(const spd_kv_view *v, const int32_t *n_new, const spd_score *c, std::vector<TokUserPlan> &plan)
{
    plan.resize((size_t)v->n_users);
    for (int u = 0; u < v->n_users; ++u) {
        TokUserPlan &p = plan[(size_t)u];
        p.n_tok = n_new[u];
        p.len = v->lens[u];
        p.k_pos = first_key_position(c, u);
        p.q_pos = c && c->q_pos ? c->q_pos[u] - p.k_pos : p.len - p.n_tok;
        p.prefix = c && c->prefix ? std::max(0, c->prefix[u] - p.k_pos) : 0;
    }
}

// Which kernel takes a user's rows, and in tiles of how many.
enum class TokKernel { kFew16 = 0, kFew32 = 1, kMany = 2 };
constexpr int kTokKernels = 3;
inline int tile_rows(TokKernel k) { return k == TokKernel::kFew16 ? 16 : k == TokKernel::kFew32 ? 32 : kManyRows; }

// How many rows (tokens times query heads of a group) the few kernel takes: 16 or 32 to a tile, each K/V byte read once for all of them.
inline TokKernel kernel_for(int64_t rows)
{
    return rows <= 16 ? TokKernel::kFew16 : rows <= 32 ? TokKernel::kFew32 : TokKernel::kMany;
}

// The keys that a tile's rows can see by what the host knows (causal order, windows, prefixes), without ranges: [lo, hi) less [gap_lo, gap_hi).
struct TokSpan {
    int32_t lo = 0, hi = 0, gap_lo = 0, gap_hi = 0;
};
inline TokSpan tile_span(const TokUserPlan &p, int causal, int window, int token_first, int token_last)
{
    const int64_t qa = (int64_t)p.q_pos + token_first, qb = (int64_t)p.q_pos + token_last;
    int64_t lo = 0, hi = p.len;
    if (window) {
        lo = std::max<int64_t>(lo, qa - window + 1);
        if (!causal)
            hi = std::min<int64_t>(hi, qb + window);
    }
    if (causal)
        hi = std::min<int64_t>(hi, qb + 1);
    const int64_t pre = std::min<int64_t>(p.prefix, p.len);
    TokSpan s;
    if (hi <= lo) {  // the prefix alone
        s.hi = (int32_t)pre;
        s.gap_lo = s.gap_hi = s.hi;
        return s;
    }
    if (pre <= 0 || pre >= lo) {
        s.lo = pre > 0 ? 0 : (int32_t)lo;
        s.hi = (int32_t)std::max(hi, pre);
        s.gap_lo = s.gap_hi = s.hi;
        return s;
    }
    s.lo = 0;
    s.hi = (int32_t)hi;
    s.gap_lo = (int32_t)pre;
    s.gap_hi = (int32_t)lo;
    return s;
}

// The steps (of `step` keys) of a span, in order, the gap's left out: how many, and the key at which the i-th begins.
struct TokSteps {
    int32_t first = 0, before = 0, second = 0, n = 0;  // first step, steps before the gap, the step behind it, all steps
    TokSteps(const TokSpan &s, int step)
    {
        if (s.hi <= s.lo)
            return;
        first = s.lo / step;
        const int32_t end = (s.hi + step - 1) / step;
        const int32_t gap0 = (s.gap_lo + step - 1) / step, gap1 = s.gap_hi / step;
        if (gap1 > gap0) {
            before = gap0 - first;
            second = gap1;
            n = before + end - gap1;
        } else {
            before = n = end - first;
        }
    }
    int64_t begin(int32_t i, int step) const { return (int64_t)(i < before ? first + i : second + i - before) * step; }
};

struct TokTables {
    std::vector<TokUser> users;
    std::vector<TokItem> items[kTokKernels];  // the launch order
    std::vector<TokJoin> joins[kTokKernels];
    int64_t slots[kTokKernels] = {0, 0, 0};
    std::vector<TreeItem> tree[kTokKernels];  // trees' items, in the place of the others
    // The tables serve longer lengths and later queries as well, any of them (growable), or where lengths grow by no more than positions (following).
    bool growable = false, following = false;
    bool half = false;  // trees: the tiles of many rows are of 64
    int64_t n_items() const
    {
        int64_t n = 0;
        for (int k = 0; k < kTokKernels; ++k)
            n += (int64_t)(items[k].size() + tree[k].size());
        return n;
    }
};

// Workgroups that run side by side on a compute unit, as the rule below counts them: three of the few kernel's 16-row form, two of the others.  That is what fits
// with 128 channels (149-158 registers; 179-246).  With 64 channels more may fit (16 rows three to five, 93-134 registers; 32 rows three or four; many rows two or
// three, 145-170), but counting three there made calls no faster, or 5 % slower.
inline int resident(TokKernel k) { return k == TokKernel::kFew16 ? 3 : 2; }

struct TokTile {
    int32_t user, kv_head, row0, n_rows, steps, first;  // first: index into the spans
};

// Tiles cut into stretches of at most `chunk` steps: how many stretches in all, and how long the longest is.
struct Cut {
    int64_t n = 0, longest = 0;
    Cut(const std::vector<TokTile> &tiles, int64_t chunk)
    {
        for (const TokTile &t : tiles) {
            const int64_t k = std::max<int64_t>(1, (t.steps + chunk - 1) / chunk);
            n += k;
            longest = std::max(longest, (t.steps + k - 1) / k);
        }
    }
};

// The longest stretch to cut tiles into, by what the call then takes in steps of one workgroup (`at_once` of them run side by side): tiles left whole, as long
// as the longest or as the average and the unevenness at the end; one round of stretches, as long as the longest of them; several rounds,
// shorter and so more even.  A stretch costs `overhead` steps (its start, its partial and the join).  No stretch is shorter than `least`.
// Few rows, us per call by the stretches' length: 64 users of 512-4096 keys, 8 KV heads of 64 (512 tiles, 48 steps for each of 768 workgroups): one round of up to
// 75 steps 84.6, 24 steps 65.5, 16 steps 63.7; 24 users of 8192-32768 keys, 8 KV heads (165 steps): one round of up to 183 343, 64 steps 354, 24 steps 368;
// 16 users of 512-4096 keys (12 steps): one round of up to 13 34.7, 24 steps 37.8, 10 steps 38.2.
// Many rows: 4096 causal tokens, 16 query heads of one KV head of 128, bf16 (512 tiles of up to 64 steps, 32 each on average): whole 104, 16 steps 116; 2048
// tokens, 32 heads in groups of four, fp32 (the same steps): whole 473, 16 steps 394.
inline int64_t stretch_steps(const std::vector<TokTile> &tiles, int64_t at_once, int64_t least, double overhead)
{
    int64_t total = 0;
    for (const TokTile &t : tiles)
        total += t.steps;
    const double average = (double)total / (double)at_once, uneven = 0.35;
    const int64_t longest = Cut(tiles, (int64_t)1 << 40).longest;
    if (longest <= least)
        return least;
    int64_t best = longest;
    double time = std::max((double)longest, average + uneven * (double)longest);
    if ((int64_t)tiles.size() < at_once) {  // the shortest with which one round takes them all
        int64_t lo = least, hi = longest;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (Cut(tiles, mid).n <= at_once)
                hi = mid;
            else
                lo = mid + 1;
        }
        const double t = (double)Cut(tiles, lo).longest + overhead;
        if (t < time) {
            best = lo;
            time = t;
        }
    }
    for (int rounds : {2, 3, 5}) {
        const int64_t c = std::max<int64_t>({least, 12, (int64_t)(average / rounds)});
        const double t = average * (1 + overhead / (double)c) + overhead + uneven * (double)c;
        if (c < longest && (double)Cut(tiles, c).n >= 2.5 * (double)at_once && t < 0.97 * time) {
            best = c;
            time = t;
        }
    }
    return best;
}

constexpr int kXcds = 8;

// tree: a user's tokens lie at any depth, in any order, so every tile's rows may see what any of the user's can.
inline void build_tok_tables(const spd_shape *s, const spd_kv_view *v, const std::vector<TokUserPlan> &plan, int causal, int window, int n_cus,
                             TokTables &T, bool tree = false)
{
    const int G = s->n_q_heads / s->n_kv_heads, Hkv = s->n_kv_heads, es = elt_size(s->dtype);
    const bool addresses = v->block_size == 0 && !v->k_ptrs_dev;
    T.users.resize(plan.size());
    T.growable = T.following = true;
    int32_t tok0 = 0;
    // Trees of few rows go in one launch, in tiles of 32 where any of them needs those.
    TokKernel few = TokKernel::kFew16;
    for (const TokUserPlan &p : plan)
        if ((int64_t)p.n_tok * G > 16 && (int64_t)p.n_tok * G <= 32)
            few = TokKernel::kFew32;
    // Trees of many rows go in tiles of 64 where tiles of 128 would be a fifth emptier.  24 users of 900-8000 keys, 32 heads in groups of four of 128, bf16, results in
    // fp32, us per call in tiles of 128 / 64: 14-16 tokens 136 / 117, 9-32 tokens 141 / 150, 28-32 tokens (results in bf16) 113 / 139.  fp32, six users' 60-64
    // tokens, 8 heads of 64 55 / 39.
    if (tree && has_half(s->dtype, s->head_dim)) {
        int64_t whole = 0, halves = 0;  // rows of all tiles, by the keys they go over
        for (const TokUserPlan &p : plan)
            if ((int64_t)p.n_tok * G > 32) {
                const int64_t rows = (int64_t)p.n_tok * G;
                whole += (rows + kManyRows - 1) / kManyRows * kManyRows * p.len;
                halves += (rows + kHalfRows - 1) / kHalfRows * kHalfRows * p.len;
            }
        T.half = (double)halves < 0.8 * (double)whole;
    }
    std::vector<TokTile> tiles[kTokKernels];
    std::vector<TokSteps> spans;
    for (size_t u = 0; u < plan.size(); ++u) {
        const TokUserPlan &p = plan[u];
        TokUser &d = T.users[u];
        d = TokUser();
        if (addresses && p.len > 0) {
            d.k_base = static_cast<const char *>(v->k_ptrs[u]);
            d.v_base = static_cast<const char *>(v->v_ptrs[u]);
        }
        d.head_stride = (v->head_strides && v->block_size == 0 && p.len > 0 ? v->head_strides[u] : v->head_stride) * es;
        d.tok0 = tok0;
        d.n_tok = p.n_tok;
        d.len = p.len;
        d.q_pos = p.q_pos;
        d.prefix = p.prefix;
        d.k_pos = p.k_pos;
        tok0 += p.n_tok;
        const int64_t rows = (int64_t)p.n_tok * G;
        if (rows == 0)
            continue;
        const TokKernel k = tree && rows <= 32 ? few : kernel_for(rows);
        // A schedule serves longer lengths and later queries as well where a tile's keys end with the view and not with its own causal order.  Where
        // its windows begin behind the view's last key, its keys end with the prefix (or there are none): keys that come into a window
        // would lie in no stretch, so its lengths may only grow with its positions, windows ahead.
        T.following = T.following && k != TokKernel::kMany && p.len > 0 && (!causal || p.q_pos + p.n_tok >= p.len) && !(window && !causal);
        T.growable = T.growable && T.following;
        const int step = k == TokKernel::kMany ? many_keys(s->dtype, T.half) : kFewKeys, cap = k == TokKernel::kMany && T.half ? kHalfRows : tile_rows(k);
        for (int64_t r0 = 0; r0 < rows; r0 += cap) {
            const int64_t r1 = std::min<int64_t>(rows, r0 + cap);
            const TokSpan span = tree ? tile_span(p, causal, window, 0, p.n_tok - 1) : tile_span(p, causal, window, (int)(r0 / G), (int)((r1 - 1) / G));
            T.growable = T.growable && span.hi == p.len;
            spans.emplace_back(span, step);
            for (int h = 0; h < Hkv; ++h)
                tiles[(int)k].push_back(TokTile{(int32_t)u, h, (int32_t)r0, (int32_t)(r1 - r0), spans.back().n, (int32_t)spans.size() - 1});
        }
    }
    for (int k = 0; k < kTokKernels; ++k) {
        std::vector<TokTile> &tl = tiles[k];
        if (tl.empty())
            continue;
        const bool many = k == (int)TokKernel::kMany;
        const int step = many ? many_keys(s->dtype, T.half) : kFewKeys;
        const int64_t at_once = (int64_t)n_cus * (tree && !many ? tree_resident(s->dtype, s->head_dim, tile_rows((TokKernel)k)) : resident((TokKernel)k));
        // (a step of many rows is short for its partial's 64 KB; fp32 steps take longer)
        const double overhead = k == (int)TokKernel::kFew16 && !tree ? 2.5 : many && s->dtype != SPD_F32 ? 10.0 : 5.0;
        // (Many rows of a tree, down to one step: small calls leave the device empty.  One user's 16 tokens over 1531 keys, us per call with one step at least / two / four /
        // eight: 14.7 / 15.9 / 20.6 / 30.6; three users' 5-130 tokens, fp32, 21.7 / 27.5 / 38.7 / 53.4.)
        const int64_t chunk = stretch_steps(tl, at_once, tree && many ? 1 : 4, overhead);
        // The longest stretches first.  The many kernel's tiles of one head read the same keys: they go to one XCD (workgroup i
        // runs on XCD i % 8), whose L2 then holds them; heads in order of their work, each to the XCD with least so far.  Where that would
        // leave XCDs idle (their number divides that of the heads badly, and these are few) a head's tiles are dealt out to several.
        // (Head after head on an XCD, so that fewer share its L2 at a time, us against this: 4096 causal tokens, 24 heads of 64 with their own KV heads
        // 116 / 84; four prompts of 900-4096 tokens 340 / 331; 16384 tokens, 32 heads of 128 with their own KV heads, 8 MB each, 2106 / 2090.)
        struct Queued {
            TokItem item;
            int32_t steps;
        };
        std::vector<std::vector<Queued>> queue(many ? kXcds : 1);
        std::vector<int64_t> load(queue.size(), 0);
        std::vector<int64_t> weight(plan.size() * (size_t)Hkv, 0);  // of a user's head
        for (const TokTile &t : tl)
            weight[(size_t)t.user * Hkv + t.kv_head] += t.steps + 1;
        size_t heads = 0;
        for (int64_t w : weight)
            heads += w > 0;
        std::stable_sort(tl.begin(), tl.end(), [&](const TokTile &a, const TokTile &b) {
            const size_t ga = (size_t)a.user * Hkv + a.kv_head, gb = (size_t)b.user * Hkv + b.kv_head;
            if (many && ga != gb)
                return weight[ga] != weight[gb] ? weight[ga] > weight[gb] : ga < gb;
            return a.steps > b.steps;
        });
        const size_t parts = !many || heads % kXcds == 0 || heads >= 4 * kXcds ? 1 : (4 * kXcds + heads - 1) / heads;
        std::vector<size_t> dealt_to(parts, 0);
        size_t last_head = (size_t)-1, at = 0;
        for (const TokTile &t : tl) {
            const size_t g = (size_t)t.user * Hkv + t.kv_head;
            if (many && g != last_head) {
                for (size_t &q : dealt_to) {
                    q = (size_t)(std::min_element(load.begin(), load.end()) - load.begin());
                    load[q] += weight[g] / (int64_t)parts + 1;
                }
                last_head = g;
                at = 0;
            }
            const size_t q = dealt_to[at++ % parts];
            const TokSteps &sp = spans[(size_t)t.first];
            const int64_t n = std::max<int64_t>(1, (t.steps + chunk - 1) / chunk);
            const int64_t slot = n > 1 ? T.slots[k] : -1;
            for (int64_t j = 0; j < n; ++j) {
                TokItem it;
                it.user = t.user;
                it.kv_head = t.kv_head;
                it.row0 = t.row0;
                it.n_rows = t.n_rows;
                const int32_t s0 = (int32_t)(t.steps * j / n), s1 = (int32_t)(t.steps * (j + 1) / n);
                it.k_begin = it.k_end = 0;
                if (s1 > s0) {
                    it.k_begin = (int32_t)sp.begin(s0, step);
                    it.k_end = (int32_t)std::min<int64_t>(sp.begin(s1 - 1, step) + step, plan[(size_t)t.user].len);
                }
                it.to_len = s1 > s0 && j == n - 1 && it.k_end == plan[(size_t)t.user].len;
                it.slot = n > 1 ? (int32_t)(slot + j) : -1;
                queue[q].push_back(Queued{it, s1 - s0});
            }
            if (n > 1) {
                T.joins[k].push_back(TokJoin{t.user, t.kv_head, t.row0, t.n_rows, (int32_t)slot, (int32_t)n, {0, 0}});
                T.slots[k] += n;
            }
        }
        // Few rows of a tree: the heads of a stretch side by side (one user's 4 tokens over 6000 keys, heads of 64 / 128, us per call: 11.7 / 14.7, head by head 13.3 / 15.2),
        // but not where long stretches' neighbours would ask for halves of the same 256 bytes at once from several XCDs (24 users' 2-4 tokens over 900-8000 keys, token-major heads of 64,
        // fp16: 56.8, head by head 49.8).
        const bool halves = v->head_stride < v->token_stride && s->head_dim * es < 256;
        const bool side_by_side = tree && !many && !(halves && chunk > 8);
        size_t longest = 0;
        for (auto &x : queue) {
            std::stable_sort(x.begin(), x.end(), [&](const Queued &a, const Queued &b) {
                if (a.steps != b.steps || !side_by_side)
                    return a.steps > b.steps;
                return std::tie(a.item.user, a.item.row0, a.item.k_begin) < std::tie(b.item.user, b.item.row0, b.item.k_begin);
            });
            longest = std::max(longest, x.size());
        }
        const TokItem nothing = {0, 0, 0, 0, 0, 0, -1, 0};
        if (tree) {
            T.tree[k].reserve(longest * queue.size());
            for (size_t i = 0; i < longest; ++i)
                for (const auto &x : queue)
                    T.tree[k].push_back(i < x.size() ? TreeItem{x[i].item, T.users[(size_t)x[i].item.user]} : TreeItem{nothing, TokUser()});
            continue;
        }
        T.items[k].reserve(longest * queue.size());
        for (size_t i = 0; i < longest; ++i)
            for (const auto &x : queue)
                T.items[k].push_back(i < x.size() ? x[i].item : nothing);
    }
}

}  // namespace spd::host
