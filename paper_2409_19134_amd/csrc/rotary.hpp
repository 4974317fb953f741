// Rotary positions, and the append of new tokens to a cache with the rotation on the way.  Bound by the bytes that are turned or copied.
//
// A workgroup takes a few tokens.  It first forms their cosines and sines, one (token, pair) to a thread, into LDS: the heads of a token
// share them.  Then every thread keeps one place of a head - sixteen bytes and, for pairs half a rotation apart, the sixteen that turn with
// them - and goes through all heads of all the tokens, one after the other: what is read may be what the store before it wrote (in place), so the compiler
// keeps a head's loads behind the stores of the one before.  What is in flight is many waves' (seven or eight to a SIMD), not many loads of one.
// An angle is position * inv_freq: a product of 31 and 24 bits, formed in 64, as turns, of which only the fraction is kept; cosine and sine
// of that are fp32.
// Measured: 20240 tokens of 40 heads (bf16, 128 channels; 414 MB read and written) 68.4 us, 6.1 TB/s, where a large copy reaches 4.9.
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
    int32_t first;               // the launch's first token
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

// Sixteen bytes; ONCE: they do not come back soon, or are not read again soon (see kOnceBytes).
template <bool ONCE>
__device__ __forceinline__ u32x4 piece_load(const char *p)
{
    typedef const u32x4 __attribute__((address_space(1))) *in;
    return ONCE ? __builtin_nontemporal_load((in)(uintptr_t)p) : *(in)(uintptr_t)p;
}
template <bool ONCE>
__device__ __forceinline__ void piece_store(char *p, u32x4 v)
{
    typedef u32x4 __attribute__((address_space(1))) *out;
    if constexpr (ONCE)
        __builtin_nontemporal_store(v, (out)(uintptr_t)p);
    else
        *(out)(uintptr_t)p = v;
}

// Turns (or copies) the thread's place of one head.
template <int DT, bool ADJACENT, bool ONCE, class Place>
__device__ __forceinline__ void turn_head(const Place &p, const float2 *cs, const char *src, char *dst)
{
    constexpr int VE = Place::VE, NP = Place::NP;
    u32x4 a = piece_load<ONCE>(src + p.off);
    if (p.turns) {
        u32x4 b = a;
        if constexpr (!ADJACENT)
            b = piece_load<ONCE>(src + p.off2);
        float f[VE], g[VE];
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const float2 t = cs[p.pair + j];
            if constexpr (ADJACENT) {
                const float x0 = elt_get<DT>(a, 2 * j), x1 = elt_get<DT>(a, 2 * j + 1);
                f[2 * j] = x0 * t.x - x1 * t.y;
                f[2 * j + 1] = x0 * t.y + x1 * t.x;
            } else {
                const float x0 = elt_get<DT>(a, j), x1 = elt_get<DT>(b, j);
                f[j] = x0 * t.x - x1 * t.y;
                g[j] = x0 * t.y + x1 * t.x;
            }
        }
        a = elt_pack<DT>(f);
        if constexpr (!ADJACENT)
            piece_store<ONCE>(dst + p.off2, elt_pack<DT>(g));
    }
    piece_store<ONCE>(dst + p.off, a);
}

template <int DT, int D, bool ADJACENT, bool ONCE>
__global__ __launch_bounds__(256) void rotate_kernel(const RotateArgs a)
{
    typedef TurnPlace<DT, D, ADJACENT> Place;
    __shared__ float2 cs[kTurnTokens][64];
    const int token0 = a.first + (int)blockIdx.x * a.per_group, count = min(a.per_group, a.turn.n_tokens - token0);
    fill_turns(cs, a.turn, token0, count);
    __syncthreads();
    const int places = turn_places(Place::ES, D, ADJACENT, a.turn.n_pairs), step = 256 / places;
    const Place p((int)threadIdx.x & (places - 1), a.turn.n_pairs);
    if (p.idle)
        return;
    // the heads of the tokens, one after the other
    int k = 0, head = (int)threadIdx.x / places;
#pragma unroll 4
    for (int at = head; at < count * a.n_heads; at += step, head += step) {
        while (head >= a.n_heads) {
            head -= a.n_heads;
            ++k;
        }
        const int64_t off = (int64_t)head * (D * Place::ES), token = token0 + k;
        turn_head<DT, ADJACENT, ONCE>(p, cs[k], a.x + token * a.x_stride + off, a.y + token * a.y_stride + off);
    }
}

template <int DT, int D, bool ADJACENT, bool ONCE>
__global__ __launch_bounds__(256) void append_kernel(const AppendArgs a, const AppendItems given)
{
    typedef TurnPlace<DT, D, ADJACENT> Place;
    constexpr int HB = D * Place::ES;
    __shared__ float2 cs[kTurnTokens][64];
    __shared__ int64_t places_of[kTurnTokens];  // the tokens' offsets in the cache
    const AppendItem it = a.by_value ? given.it[blockIdx.x] : a.items[blockIdx.x];
    if ((int)threadIdx.x < it.count) {
        const int at = it.place + a.grow + (int)threadIdx.x;
        places_of[threadIdx.x] = a.k_pool ? (int64_t)a.block_table[(int64_t)it.user * a.max_blocks + (at >> a.page_shift)] * a.block_stride +
                                                (int64_t)(at & ((1 << a.page_shift) - 1)) * a.token_stride
                                          : (int64_t)at * a.token_stride;
    }
    fill_turns(cs, a.turn, it.token, it.count);
    __syncthreads();
    char *k_base = it.k_base, *v_base = it.v_base;
    if (a.k_pool) {
        k_base = a.k_pool;
        v_base = a.v_pool;
    } else if (a.k_ptrs) {
        k_base = a.k_ptrs[it.user];
        v_base = a.v_ptrs[it.user];
    }
    const int places = turn_places(Place::ES, D, ADJACENT, a.turn.n_pairs), step = 256 / places;
    const Place p((int)threadIdx.x & (places - 1), a.turn.n_pairs);
    if (!p.idle) {
        const int Hq = a.q_out ? a.Hq : 0, heads = Hq + a.Hkv;
        int k = 0, head = (int)threadIdx.x / places;
#pragma unroll 4
        for (int i = head; i < it.count * heads; i += step, head += step) {
            while (head >= heads) {
                head -= heads;
                ++k;
            }
            const int64_t token = it.token + k;
            const int kh = head - Hq;
            const char *src = kh < 0 ? a.q + token * a.q_stride + (int64_t)head * HB : a.k + token * a.k_stride + (int64_t)kh * HB;
            char *dst = kh < 0 ? a.q_out + (token * a.Hq + head) * HB : k_base + places_of[k] + kh * it.head_stride;
            turn_head<DT, ADJACENT, ONCE>(p, cs[k], src, dst);
        }
    }
    constexpr int kPieces = D / Place::VE, kHeads = 256 / kPieces;
    const int off = ((int)threadIdx.x & (kPieces - 1)) * 16;
    int k = 0, head = (int)threadIdx.x / kPieces;
#pragma unroll 4
    for (int i = head; i < it.count * a.Hkv; i += kHeads, head += kHeads) {
        while (head >= a.Hkv) {
            head -= a.Hkv;
            ++k;
        }
        piece_store<ONCE>(v_base + places_of[k] + head * it.head_stride + off,
                          piece_load<ONCE>(a.v + (it.token + k) * a.v_stride + (int64_t)head * HB + off));
    }
}

}  // namespace spd
