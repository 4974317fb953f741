// Rotary positions, and the append of new tokens to a cache with the rotation on the way.  Bound by the bytes that are turned or copied.
//
// A workgroup takes a few tokens.  It first forms their cosines and sines, one (token, pair) to a thread, into LDS: the heads of a token
// share them.  Then every thread keeps one place of a head - sixteen bytes and, for pairs half a rotation apart, the sixteen that turn with
// them - and goes through the tokens' heads with its cosines and sines in registers.
// An angle is position * inv_freq: a product of 31 and 24 bits, formed in 64, as turns, of which only the fraction is kept; cosine and sine
// of that are fp32.
#pragma once
#include "common.hpp"

namespace spd {

struct TurnArgs {
    const int32_t *positions;  // [axes][tokens]
    const float *inv_freq;     // [pairs]
    uint64_t axis[2];          // two bits a pair
    int32_t n_tokens, n_pairs; // pairs 0: nothing turns
    float amplitude, sign;     // sign -1: the transposed map
};

struct RotateArgs {
    TurnArgs turn;
    const char *x;
    char *y;
    int64_t x_stride, y_stride;  // bytes between tokens
    int32_t n_heads;
    int32_t per_group;           // tokens of a workgroup, up to kTurnTokens
};

// New tokens of one user that lie next to each other: up to kTurnTokens of them.
struct AppendItem {
    char *k_base, *v_base;   // contiguous without device pointer tables: the user's buffers; else nullptr
    int64_t head_stride;     // bytes
    int32_t user, token;     // the first of them among all new tokens
    int32_t place, count;    // its place in the user's cache (grows with AppendArgs::grow)
};
static_assert(sizeof(AppendItem) == 40);

struct AppendArgs {
    TurnArgs turn;
    const char *q, *k, *v;
    char *q_out;                        // nullptr: no queries
    int64_t q_stride, k_stride, v_stride;  // bytes between tokens
    char *k_pool, *v_pool;              // paged, else nullptr
    char *const *k_ptrs, *const *v_ptrs;   // device pointer tables, or nullptr
    const int32_t *block_table;
    int64_t block_stride, token_stride;
    int32_t max_blocks, page_shift;
    int32_t Hq, Hkv;
    int32_t grow;
    int32_t by_value;                   // items travel with the arguments
    const AppendItem *items;
};
constexpr int kTurnTokens = 4;
constexpr int kAppendByValue = 16;  // items that travel with the arguments: a call for few users has nothing to upload (arguments of
                                     // 48 items cost the host more than looking its table up: 32 users 5.0 us, 4.1 with the table)
struct AppendItems {
    AppendItem it[kAppendByValue];
};

// One dword of an element pair <-> floats.
template <int DT>
__device__ __forceinline__ float elt_get(const u32x4 &w, int e)
{
    if constexpr (DT == SPD_F32)
        return __uint_as_float(w[e]);
    else if constexpr (DT == SPD_BF16)
        return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    else {
        const uint16_t b = (uint16_t)(e % 2 ? w[e / 2] >> 16 : w[e / 2]);
        return (float)__builtin_bit_cast(_Float16, b);
    }
}
template <int DT>
__device__ __forceinline__ u32x4 elt_pack(const float *f)
{
    u32x4 w;
    if constexpr (DT == SPD_F32) {
        for (int e = 0; e < 4; ++e)
            w[e] = __float_as_uint(f[e]);
    } else if constexpr (DT == SPD_BF16) {
        bf16x8 b;
        for (int e = 0; e < 8; ++e)
            b[e] = (__bf16)f[e];
        w = __builtin_bit_cast(u32x4, b);
    } else {
        typedef _Float16 h8 __attribute__((ext_vector_type(8)));
        h8 b;
        for (int e = 0; e < 8; ++e)
            b[e] = (_Float16)f[e];
        w = __builtin_bit_cast(u32x4, b);
    }
    return w;
}

// Where a thread stands in a head: `off` (and `off2`, the other channels of its pairs), bytes; `pair` the first of its pairs.
template <int DT, int D, bool ADJACENT>
struct TurnPlace {
    static constexpr int ES = DT == SPD_F32 ? 4 : 2, VE = 16 / ES, NP = ADJACENT ? VE / 2 : VE;  // elements of 16 bytes, pairs of a thread
    int off, off2, pair;
    bool turns, idle;
    __device__ __forceinline__ TurnPlace(int unit, int n_pairs)
    {
        const int turning = ADJACENT ? 2 * n_pairs / VE : n_pairs / VE;
        turns = unit < turning;
        idle = !turns && unit - turning >= (D - 2 * n_pairs) / VE;
        pair = unit * NP;
        off = turns ? unit * 16 : (2 * n_pairs + (unit - turning) * VE) * ES;
        off2 = off + n_pairs * ES;
    }
};
// Places of a head, rounded up to a power of two (so that a thread's place and head are bits of its number).
__host__ __device__ inline int turn_places(int es, int D, bool adjacent, int n_pairs)
{
    const int ve = 16 / es, n = (adjacent ? 2 * n_pairs : n_pairs) / ve + (D - 2 * n_pairs) / ve;
    int p = 1;
    while (p < n)
        p *= 2;
    return p;
}

// Cosines and sines of `count` tokens from `token` on.
__device__ __forceinline__ void fill_turns(float2 (*cs)[64], const TurnArgs &t, int token, int count)
{
    for (int i = threadIdx.x; i < count * 64; i += 256) {
        const int k = i / 64, pair = i % 64;
        if (pair >= t.n_pairs)
            continue;
        const int axis = (int)(t.axis[pair / 32] >> (2 * (pair % 32))) & 3;
        const double turns = (double)t.positions[(int64_t)axis * t.n_tokens + token + k] * ((double)t.inv_freq[pair] * 0.15915494309189533577);
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        cs[k][pair] = float2{c * t.amplitude, s * t.amplitude * t.sign};
    }
}

// A thread's cosines and sines of one token.
template <int NP>
struct Turns {
    float c[NP], s[NP];
    __device__ __forceinline__ void read(const float2 *cs, int pair, bool turns)
    {
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const float2 v = turns ? cs[pair + j] : float2{1.f, 0.f};
            c[j] = v.x;
            s[j] = v.y;
        }
    }
};

// Turns (or copies) the thread's place of one head.
template <int DT, bool ADJACENT, class Place>
__device__ __forceinline__ void turn_head(const Place &p, const Turns<Place::NP> &t, const char *src, char *dst)
{
    typedef const u32x4 __attribute__((address_space(1))) *in;
    typedef u32x4 __attribute__((address_space(1))) *out;
    u32x4 a = *(in)(uintptr_t)(src + p.off);
    if (p.turns) {
        constexpr int VE = Place::VE;
        if constexpr (ADJACENT) {
            float f[VE];
#pragma unroll
            for (int j = 0; j < VE / 2; ++j) {
                const float x0 = elt_get<DT>(a, 2 * j), x1 = elt_get<DT>(a, 2 * j + 1);
                f[2 * j] = x0 * t.c[j] - x1 * t.s[j];
                f[2 * j + 1] = x0 * t.s[j] + x1 * t.c[j];
            }
            a = elt_pack<DT>(f);
        } else {
            const u32x4 b = *(in)(uintptr_t)(src + p.off2);
            float f[VE], g[VE];
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const float x0 = elt_get<DT>(a, j), x1 = elt_get<DT>(b, j);
                f[j] = x0 * t.c[j] - x1 * t.s[j];
                g[j] = x0 * t.s[j] + x1 * t.c[j];
            }
            a = elt_pack<DT>(f);
            *(out)(uintptr_t)(dst + p.off2) = elt_pack<DT>(g);
        }
    }
    *(out)(uintptr_t)(dst + p.off) = a;
}

template <int DT, int D, bool ADJACENT>
__global__ __launch_bounds__(256) void rotate_kernel(const RotateArgs a)
{
    typedef TurnPlace<DT, D, ADJACENT> Place;
    __shared__ float2 cs[kTurnTokens][64];
    const int token0 = blockIdx.x * a.per_group, count = min(a.per_group, a.turn.n_tokens - token0);
    fill_turns(cs, a.turn, token0, count);
    __syncthreads();
    const int places = turn_places(Place::ES, D, ADJACENT, a.turn.n_pairs);
    const Place p((int)threadIdx.x & (places - 1), a.turn.n_pairs);
    if (p.idle)
        return;
    const int head0 = (int)threadIdx.x / places, heads = 256 / places;
    for (int k = 0; k < count; ++k) {
        Turns<Place::NP> t;
        t.read(cs[k], p.pair, p.turns);
        const char *src = a.x + (int64_t)(token0 + k) * a.x_stride;
        char *dst = a.y + (int64_t)(token0 + k) * a.y_stride;
#pragma unroll 4
        for (int head = head0; head < a.n_heads; head += heads)
            turn_head<DT, ADJACENT>(p, t, src + (int64_t)head * (D * Place::ES), dst + (int64_t)head * (D * Place::ES));
    }
}

template <int DT, int D, bool ADJACENT>
__global__ __launch_bounds__(256) void append_kernel(const AppendArgs a, const AppendItems given)
{
    typedef TurnPlace<DT, D, ADJACENT> Place;
    constexpr int HB = D * Place::ES;
    __shared__ float2 cs[kTurnTokens][64];
    const AppendItem it = a.by_value ? given.it[blockIdx.x] : a.items[blockIdx.x];
    fill_turns(cs, a.turn, it.token, it.count);
    __syncthreads();
    const int places = turn_places(Place::ES, D, ADJACENT, a.turn.n_pairs);
    const Place p((int)threadIdx.x & (places - 1), a.turn.n_pairs), whole((int)threadIdx.x & (D / Place::VE - 1), 0);
    const int head0 = (int)threadIdx.x / places, heads = 256 / places;
    char *k_base = it.k_base, *v_base = it.v_base;
    if (a.k_pool) {
        k_base = a.k_pool;
        v_base = a.v_pool;
    } else if (a.k_ptrs) {
        k_base = a.k_ptrs[it.user];
        v_base = a.v_ptrs[it.user];
    }
    const int Hq = a.q_out ? a.Hq : 0;
    for (int k = 0; k < it.count; ++k) {
        const int64_t token = it.token + k;
        const int at = it.place + a.grow + k;
        int64_t off;
        if (a.k_pool)
            off = (int64_t)a.block_table[(int64_t)it.user * a.max_blocks + (at >> a.page_shift)] * a.block_stride +
                  (int64_t)(at & ((1 << a.page_shift) - 1)) * a.token_stride;
        else
            off = (int64_t)at * a.token_stride;
        if (!p.idle) {
            Turns<Place::NP> t;
            t.read(cs[k], p.pair, p.turns);
            const char *q = a.q + token * a.q_stride, *kn = a.k + token * a.k_stride;
            char *qo = a.q_out + token * a.Hq * HB;
#pragma unroll 4
            for (int head = head0; head < Hq + a.Hkv; head += heads) {
                const int kh = head - Hq;
                if (kh < 0)
                    turn_head<DT, ADJACENT>(p, t, q + (int64_t)head * HB, qo + (int64_t)head * HB);
                else
                    turn_head<DT, ADJACENT>(p, t, kn + (int64_t)kh * HB, k_base + off + (int64_t)kh * it.head_stride);
            }
        }
        constexpr int kPieces = D / Place::VE;
        for (int head = (int)threadIdx.x / kPieces; head < a.Hkv; head += 256 / kPieces)
            copy16(v_base + off + (int64_t)head * it.head_stride + whole.off, a.v + token * a.v_stride + (int64_t)head * HB + whole.off);
    }
}

}  // namespace spd
