// Shared declarations of the calls for several new tokens per user: the tables that the host builds and the kernels read,
// the kernels' arguments, and what happens to a score between <q, k> and the softmax.
#pragma once
#include "common.hpp"

namespace spd {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// A user as the kernels read it, indexed by user.  Positions are relative to the view's first key.
struct TokUser {
    const char *k_base, *v_base;  // contiguous without device pointer tables: the user's buffers; else nullptr
    int64_t head_stride;          // bytes
    int32_t tok0, n_tok;          // its first new token among all, and how many
    int32_t len;                  // keys (grows with TokArgs::grow_len)
    int32_t q_pos;                // position of its first new token (grows with grow_q)
    int32_t prefix;               // keys below it are seen by every query
    int32_t k_pos;                // position of key 0, for the ranges
    int32_t pad[4];
};
static_assert(sizeof(TokUser) == 64);

// A tile of query rows (row = token * G + query head of the group, counted from the user's first token) over a stretch of its keys.
struct TokItem {
    int32_t user, kv_head;
    int32_t row0, n_rows;
    int32_t k_begin, k_end;  // k_begin is a multiple of the kernel's step; so is k_end unless it is the view's length
    int32_t slot;            // where its partial goes, or -1: it writes the result
    int32_t to_len;          // 1: k_end is the view's length (grows with it)
};
static_assert(sizeof(TokItem) == 32);

// A tile whose keys were split: partials slot .. slot + n_chunks - 1.
struct TokJoin {
    int32_t user, kv_head, row0, n_rows, slot, n_chunks, pad[2];
};
static_assert(sizeof(TokJoin) == 32);

struct ScoreArgs {
    float c;                  // |scale| log2(e)
    float cap_in, cap_out;    // |scale| / cap, cap log2(e); cap_out 0: no cap
    uint32_t q_and, q_xor;    // applied to the queries' bits: 0 for scale 0 (c is then 1), the sign bits for a negative scale
    const float *slopes;      // [Hq] or nullptr
    const int32_t *ranges;    // [T][2] or nullptr
    int32_t causal, window;
};

struct TokArgs {
    const TokItem *items;
    const TokUser *users;
    const char *q;
    int64_t q_stride;                  // bytes between tokens
    const char *const *k_ptrs;         // device pointer tables, or nullptr
    const char *const *v_ptrs;
    const char *k_pool, *v_pool;       // paged, else nullptr
    const int32_t *block_table;
    int64_t block_stride, token_stride;  // bytes
    int32_t max_blocks, page_shift;
    int32_t Hq, G;
    int32_t grow_len, grow_q;
    char *out;
    int32_t out_f32;
    float *lse;
    float *part_o;    // [slot][rows of a tile][D]
    float2 *part_lse; // [slot][rows of a tile]: log2 of the sum, and what the final lse adds to it (natural log)
    ScoreArgs score;
};

// A query row's masks and bias (slope: its head's, 0 without).  It sees the keys in [mlo, mlo + mn) and in [plo, plo + pn).
struct RowMask {
    int mlo, plo;
    unsigned mn, pn;
    int q_pos;
    int dist0;      // its distance to the nearest key it sees: the bias is taken relative to that one, so that far rows lose nothing
    float slope2;   // slope log2(e)
};

__host__ __device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

__host__ __device__ __forceinline__ RowMask row_mask(const ScoreArgs &s, const TokUser &u, int len, int q_pos, int token, float slope)
{
    RowMask r;
    int rlo = 0, rhi = len;
    if (s.ranges) {  // positions; those of keys are not negative
        const int2 v = reinterpret_cast<const int2 *>(s.ranges)[u.tok0 + token];
        rlo = max(max(v.x, 0) - u.k_pos, 0);
        rhi = min(max(v.y, 0) - u.k_pos, len);
    }
    int wlo = rlo, whi = rhi;
    if (s.window) {
        wlo = max(rlo, q_pos - s.window + 1);
        if (!s.causal)
            whi = min(rhi, q_pos + s.window);
    }
    if (s.causal)
        whi = min(rhi, q_pos + 1);
    r.mlo = wlo;
    r.mn = (unsigned)max(whi - wlo, 0);
    r.plo = rlo;
    r.pn = (unsigned)max(min(rhi, u.prefix) - rlo, 0);
    r.q_pos = q_pos;
    r.dist0 = 0;
    r.slope2 = 0.f;
    if (s.slopes) {
        r.slope2 = slope * kLog2e;
        int d = 0x7fffffff;
        if (r.mn)
            d = abs(q_pos - clampi(q_pos, r.mlo, r.mlo + (int)r.mn - 1));
        if (r.pn)
            d = min(d, abs(q_pos - clampi(q_pos, r.plo, r.plo + (int)r.pn - 1)));
        r.dist0 = d == 0x7fffffff ? 0 : d;
    }
    return r;
}

__host__ __device__ __forceinline__ bool sees(const RowMask &r, int key)
{
    return (unsigned)(key - r.mlo) < r.mn || (unsigned)(key - r.plo) < r.pn;
}

// What a tile of rows sees: [any_lo, any_hi) some row, [full_lo, full_hi) every row's window; prefixes end at pre_hi, windows begin at win_lo.
struct Limits {
    int any_lo = 0x7fffffff, any_hi = 0, full_lo = 0, full_hi = 0x7fffffff, pre_hi = 0, win_lo = 0x7fffffff;
    __host__ __device__ __forceinline__ void add(const RowMask &m)
    {
        if (m.mn) {
            any_lo = min(any_lo, m.mlo);
            any_hi = max(any_hi, m.mlo + (int)m.mn);
            win_lo = min(win_lo, m.mlo);
        }
        if (m.pn) {
            any_lo = min(any_lo, m.plo);
            any_hi = max(any_hi, m.plo + (int)m.pn);
            pre_hi = max(pre_hi, m.plo + (int)m.pn);
        }
        full_lo = max(full_lo, m.mlo);
        full_hi = min(full_hi, m.mlo + (int)m.mn);
    }
    __host__ __device__ __forceinline__ void add(const Limits &o)
    {
        any_lo = min(any_lo, o.any_lo);
        any_hi = max(any_hi, o.any_hi);
        full_lo = max(full_lo, o.full_lo);
        full_hi = min(full_hi, o.full_hi);
        pre_hi = max(pre_hi, o.pre_hi);
        win_lo = min(win_lo, o.win_lo);
    }
    __device__ __forceinline__ void to(int (&v)[6]) const
    {
        v[0] = any_lo, v[1] = any_hi, v[2] = full_lo, v[3] = full_hi, v[4] = pre_hi, v[5] = win_lo;
    }
    static __device__ __forceinline__ Limits from(const int (&v)[6])
    {
        Limits l;
        l.any_lo = v[0], l.any_hi = v[1], l.full_lo = v[2], l.full_hi = v[3], l.pre_hi = v[4], l.win_lo = v[5];
        return l;
    }
    __device__ __forceinline__ Limits of_lane_xor(int x) const
    {
        Limits o;
        o.any_lo = __shfl_xor(any_lo, x);
        o.any_hi = __shfl_xor(any_hi, x);
        o.full_lo = __shfl_xor(full_lo, x);
        o.full_hi = __shfl_xor(full_hi, x);
        o.pre_hi = __shfl_xor(pre_hi, x);
        o.win_lo = __shfl_xor(win_lo, x);
        return o;
    }
    __device__ __forceinline__ Limits uniform_of() const
    {
        Limits o;
        o.any_lo = uniform(any_lo);
        o.any_hi = uniform(any_hi);
        o.full_lo = uniform(full_lo);
        o.full_hi = uniform(full_hi);
        o.pre_hi = uniform(pre_hi);
        o.win_lo = uniform(win_lo);
        return o;
    }
};
// ... without ranges, from the first and the last row's positions: both ends of a row's window move up with its position (the any-limits also hold
// where neither of the two rows sees a key, but one between them does).
__host__ __device__ __forceinline__ Limits tile_limits(const ScoreArgs &s, const TokUser &u, int len, int q_first, int q_last)
{
    auto begin = [&](int q) { return s.window ? max(0, q - s.window + 1) : 0; };
    auto end = [&](int q) { return min(len, s.causal ? q + 1 : s.window ? q + s.window : len); };
    Limits l;
    const int lo = begin(q_first), hi = end(q_last), pre = min(u.prefix, len);
    if (lo < hi) {
        l.any_lo = l.win_lo = lo;
        l.any_hi = hi;
    }
    if (pre > 0) {
        l.any_lo = 0;
        l.any_hi = max(l.any_hi, pre);
        l.pre_hi = pre;
    }
    l.full_lo = begin(q_last);
    l.full_hi = end(q_first);
    return l;
}

// The steps (of `step` keys) that `waves` waves take in turn over a stretch [k_begin, k_end) of a tile's keys: from the first key that some row sees,
// over the gap between the prefixes and the windows, to the last.  Places at or behind `hi` are hi: nothing is read there, and sums with
// them stay in 32 bits.
struct KeyWalk {
    int lo, hi, gap_lo, gap_hi, step, round;
    __host__ __device__ __forceinline__ KeyWalk(const Limits &l, int k_begin, int k_end, int step_, int waves)
        : lo(max(k_begin, l.any_lo / step_ * step_)), hi(min(k_end, l.any_hi)), gap_lo(l.pre_hi), gap_hi(l.win_lo), step(step_), round(step_ * waves)
    {
        if (lo >= hi)
            lo = hi = 0;
    }
    __host__ __device__ __forceinline__ int over_gap(int t) const  // in whole rounds, so that the waves stay apart
    {
        if (t >= gap_lo && t < hi && gap_hi - step >= t)
            t += (min(gap_hi, hi + round) - t) / round * round;
        return min(t, hi);
    }
    __host__ __device__ __forceinline__ int first(int wave) const { return lo < hi ? over_gap(lo + wave * step) : hi; }
    __host__ __device__ __forceinline__ int next(int t) const { return over_gap(t + round); }  // t < hi
};

// A row's view of a run of keys from key0 on, made anew for every run: without the detour the compiler keeps every key's differences to the row's
// limits in registers, over all runs.
struct RunMask {
    int m, p, q;
    __device__ __forceinline__ RunMask(const RowMask &r, int key0) : m(key0 - r.mlo), p(key0 - r.plo), q(r.q_pos - key0) { asm("" : "+v"(m), "+v"(p), "+v"(q)); }
    __device__ __forceinline__ bool sees(const RowMask &r, int i) const { return (unsigned)(m + i) < r.mn || (unsigned)(p + i) < r.pn; }
};

// tanh from its definition by one exponential, (1 - e) / (1 + e) with e = exp(-2|x|): off by a few 1e-8 of 1.  Near zero, where that is much of
// the value (a cap far above the scores), the series instead (x^13's term is 2e-9 of x at 0.3).
__device__ __forceinline__ float tanh_of(float x)
{
    const float a = fabsf(x), y = x * x;
    const float e = fast_exp2(-2.f * kLog2e * a);
    float p = fmaf(y, -1382.f / 155925.f, 62.f / 2835.f);
    p = fmaf(y, p, -17.f / 315.f);
    p = fmaf(y, p, 2.f / 15.f);
    p = fmaf(y, p, -1.f / 3.f);
    return a < 0.3f ? fmaf(x * y, p, x) : copysignf((1.f - e) * fast_rcp(1.f + e), x);
}

// A product <q, k> with its cap, in units of log2.
__device__ __forceinline__ float capped(float s, const ScoreArgs &a) { return tanh_of(s * a.cap_in) * a.cap_out; }
// ... and the bias of a key `apart` positions from its query, less that of the row's nearest key.
__device__ __forceinline__ float biased(float x, const RowMask &r, int apart) { return fmaf(-r.slope2, (float)(abs(apart) - r.dist0), x); }

// A product <q, k> with its cap and bias, in units of log2 (MOD) or as it is (the factor c comes with the exponential then).
template <bool MOD>
__device__ __forceinline__ float modified(float s, const ScoreArgs &a, const RowMask &r, int apart)
{
    if constexpr (!MOD)
        return s;
    const float x = a.cap_out != 0.f ? capped(s, a) : s * a.c;
    return a.slopes ? biased(x, r, apart) : x;
}

// A key that a row does not see must not reach it, and zero times infinity is NaN: where some row does not see some key, non-finite values
// of V go into the product as zeros, and the rows that do see them get them added afterwards (rare, so from memory again).
template <int DT>
__device__ __forceinline__ uint32_t nonfinite(uint32_t dword)  // zero unless one of the dword's values is
{
    if constexpr (DT == SPD_F32) {
        return (dword & 0x7f800000u) == 0x7f800000u ? 1u : 0u;
    } else {
        constexpr uint32_t exp = DT == SPD_F16 ? 0x7c007c00u : 0x7f807f80u, one = DT == SPD_F16 ? 0x04000400u : 0x00800080u;
        return ((dword & exp) + one) & 0x80008000u;
    }
}
template <int DT>
__device__ __forceinline__ uint32_t finite_part(uint32_t dword)
{
    const uint32_t bad = nonfinite<DT>(dword);
    if constexpr (DT == SPD_F32)
        return bad ? 0u : dword;
    else
        return dword & ~((bad & 0x8000u ? 0xffffu : 0u) | (bad & 0x80000000u ? 0xffff0000u : 0u));
}
// Channel `ch` of the row at v if it is not finite, else zero.
template <int DT>
__device__ __forceinline__ float nonfinite_part(const char *v, int ch)
{
    float x;
    if constexpr (DT == SPD_F32)
        x = reinterpret_cast<const float *>(v)[ch];
    else if constexpr (DT == SPD_BF16)
        x = (float)reinterpret_cast<const __bf16 *>(v)[ch];
    else
        x = (float)reinterpret_cast<const _Float16 *>(v)[ch];
    return nonfinite<SPD_F32>(__float_as_uint(x)) ? x : 0.f;
}

// Offset of a user's token in its cache (table: its row of the block table, nullptr: contiguous).
__device__ __forceinline__ int64_t token_offset(const TokArgs &a, const int32_t *table, int t)
{
    if (table)
        return (int64_t)table[t >> a.page_shift] * a.block_stride + (int64_t)(t & ((1 << a.page_shift) - 1)) * a.token_stride;
    return (int64_t)t * a.token_stride;
}

// Base addresses of a user's head.
__device__ __forceinline__ void kv_bases(const TokArgs &a, const TokUser &u, int user, int kv_head, const char *&k, const char *&v)
{
    const int64_t off = (int64_t)kv_head * u.head_stride;
    if (a.k_pool) {
        k = a.k_pool + off;
        v = a.v_pool + off;
    } else if (a.k_ptrs) {
        k = reinterpret_cast<const char *>(user_base(a.k_ptrs, user)) + off;
        v = reinterpret_cast<const char *>(user_base(a.v_ptrs, user)) + off;
    } else {
        k = u.k_base + off;
        v = u.v_base + off;
    }
}

template <class T>
__device__ __forceinline__ T scalar_load(const T *p, int idx)
{
    static_assert(sizeof(T) % 4 == 0);
    T r;
    const const_u32_ptr w = (const_u32_ptr)(uintptr_t)(p + idx);
    uint32_t words[sizeof(T) / 4];
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 4; ++i)
        words[i] = w[i];
    __builtin_memcpy(&r, words, sizeof r);
    return r;
}

// Four consecutive channels of a result row, from the normalised sums.
template <int DT>
__device__ __forceinline__ void store4(const TokArgs &a, int64_t at, f32x4 v)
{
    if (a.out_f32) {
        *reinterpret_cast<f32x4 *>(a.out + at * 4) = v;
    } else if constexpr (DT == SPD_BF16) {
        typedef __bf16 b4 __attribute__((ext_vector_type(4)));
        b4 w = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
        *reinterpret_cast<b4 *>(a.out + at * 2) = w;
    } else if constexpr (DT == SPD_F16) {
        typedef _Float16 h4 __attribute__((ext_vector_type(4)));
        h4 w = {(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
        *reinterpret_cast<h4 *>(a.out + at * 2) = w;
    }
}

// Launches (host): `rows` is the row capacity of the few kernel's tiles, 16 or 32.
__attribute__((visibility("hidden"))) void launch_tokens_few(int dtype, int head_dim, bool paged, int rows, bool modified, int64_t n_items,
                                                             const TokArgs &a, hipStream_t stream);
__attribute__((visibility("hidden"))) void launch_tokens_many(int dtype, int head_dim, bool modified, int64_t n_items, const TokArgs &a,
                                                              hipStream_t stream);
constexpr int kManyRows = 128;  // rows of a tile of the many kernel
__host__ __device__ constexpr int many_keys(int dtype) { return dtype == SPD_F32 ? 32 : 64; }  // keys of its steps
constexpr int kFewKeys = 32;    // keys that the few kernel's stretches are multiples of

}  // namespace spd
