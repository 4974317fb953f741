// Partial attention of many query rows (a prompt, a chunk of one, many tokens to check) over one (user, KV head)'s keys.  Bound by the matrix
// products: 4 D operations per (row, key) pair.
//
// A workgroup takes 128 rows (row = token * G + query head of the group, so K and V are shared by the group's heads too), 32 to a wave, and goes
// through the keys in tiles of 64 (fp32: 32).  All in 32x32 blocks:
//   S^T = K Q^T    A operand K from LDS (a lane: a key, 16 bytes of its channels), B operand Q in registers (a lane: a row).  The result has a
//                  row's scores in the two lanes that share l % 32: sixteen keys of every 32 each, so the softmax needs one exchange per tile.
//   O^T += V^T P^T B operand P^T: a lane's own scores in the order in which they arrived (keys 8 (i / 4) + 4 (l / 32) + i % 4), rounded to the
//                  type; A operand V^T with its keys in that same order: 16-bit types by transposed LDS reads (ds_read_b64_tr_b16: four
//                  keys of sixteen channels to sixteen lanes), fp32 by single values.  O^T has a row per lane again: its factors need no exchange.
// P enters rounded once where results are rounded to 16 bits too; for fp32 results in three bf16 or two fp16 terms.
// The running maximum is only raised when a row's scores pass it by 2^8 (sums and P then hold values up to 2^8, the quotient is the same):
// most tiles leave the sums alone.
// K and V tiles are loaded to registers one tile ahead and stored to the other of two LDS buffers after the products: one barrier a tile.  16-byte
// pieces of a row are stored at places xor-ed with the row's number, so that neither the reads of K (16 bytes of eight rows at once) nor the
// transposed reads of V (32 bytes of four rows) meet in a bank.
// Masks: a tile that all rows of a wave see whole costs nothing, others are masked element by element, tiles that no row sees are left out.
#include "tokens.hpp"

namespace spd {
namespace {

template <int DT>
struct Block;
template <>
struct Block<SPD_BF16> {
    typedef __bf16 type;
    typedef __bf16 vec8 __attribute__((ext_vector_type(8)));
    static constexpr int kTerms = 3;
    static __device__ __forceinline__ f32x16 mfma(vec8 a, vec8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Block<SPD_F16> {
    typedef _Float16 type;
    typedef _Float16 vec8 __attribute__((ext_vector_type(8)));
    static constexpr int kTerms = 2;
    static __device__ __forceinline__ f32x16 mfma(vec8 a, vec8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Block<SPD_F32> {
    static constexpr int kTerms = 1;
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) uint32_t lds_u32;

constexpr float kRaise = 8.f;   // log2 of what a row's largest P may be
// P carries 2^kShift: fp16's keep to [2^-24, 65504] with a maximum of 2^(kRaise + 7)
template <int DT>
constexpr float kShift = DT == SPD_F16 ? 7.f : 0.f;

template <int DT, int D, bool EXACT, bool MOD>
__global__ __launch_bounds__(256, 2) void tokens_many_kernel(const TokArgs a)
{
    constexpr bool kF32 = DT == SPD_F32;
    constexpr int kBytes = kF32 ? 4 : 2, RB = D * kBytes, BN = many_keys(DT), NB = BN / 32, C = RB / 16, KK = RB / 32, CB = D / 32;
    constexpr int kTile = BN * RB, kPieces = BN * C / 256;
    constexpr int kTerms = EXACT ? Block<DT>::kTerms : 1;
    __shared__ __attribute__((aligned(16))) char lds[2][2][kTile];  // [buffer][K, V]
    __shared__ int lds_bounds[4][4];
    __shared__ uint32_t lds_bad[2][4];

    const TokItem it = scalar_load(a.items, blockIdx.x);
    if (it.n_rows == 0)
        return;  // (fills up the launch order)
    const TokUser u = scalar_load(a.users, it.user);
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    const int len = u.len + a.grow_len, q_pos0 = u.q_pos + a.grow_q;
    const int k_end = it.k_end + (it.to_len ? a.grow_len : 0);

    // the lane's row, its query and masks (rows behind the last repeat it and are not stored)
    const int my_row = min(it.row0 + wave * 32 + n, it.row0 + it.n_rows - 1);
    const int token = my_row / a.G, head = it.kv_head * a.G + (my_row - token * a.G);
    const RowMask mask = row_mask(a.score, u, len, q_pos0 + token, token, head);
    u32x4 q[KK];
    {
        const char *qr = a.q + (int64_t)(u.tok0 + token) * a.q_stride + (int64_t)head * RB + h * 16;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                q[kk][j] = (reinterpret_cast<const u32x4 *>(qr + kk * 32)[0][j] & a.score.q_and) ^ a.score.q_xor;
    }
    // keys that some row sees; where prefixes end and windows begin; keys that every row's window holds: of the wave, of the workgroup
    int any_lo = 0x7fffffff, any_hi = 0, pre_hi = 0, win_lo = 0x7fffffff, full_lo = mask.mlo, full_hi = mask.mlo + (int)mask.mn;
    if (mask.mn) {
        any_lo = mask.mlo;
        any_hi = mask.mlo + (int)mask.mn;
        win_lo = mask.mlo;
    }
    if (mask.pn) {
        any_lo = min(any_lo, mask.plo);
        any_hi = max(any_hi, mask.plo + (int)mask.pn);
        pre_hi = mask.plo + (int)mask.pn;
    }
#pragma unroll
    for (int x = 1; x < 32; x *= 2) {
        any_lo = min(any_lo, __shfl_xor(any_lo, x));
        any_hi = max(any_hi, __shfl_xor(any_hi, x));
        pre_hi = max(pre_hi, __shfl_xor(pre_hi, x));
        win_lo = min(win_lo, __shfl_xor(win_lo, x));
        full_lo = max(full_lo, __shfl_xor(full_lo, x));
        full_hi = min(full_hi, __shfl_xor(full_hi, x));
    }
    const int my_lo = uniform(any_lo), my_hi = uniform(any_hi), my_pre = uniform(pre_hi), my_win = uniform(win_lo);
    full_lo = uniform(full_lo);
    full_hi = uniform(full_hi);
    if (lane == 0) {
        lds_bounds[wave][0] = my_lo;
        lds_bounds[wave][1] = my_hi;
        lds_bounds[wave][2] = my_pre;
        lds_bounds[wave][3] = my_win;
    }
    __syncthreads();
    int lo = 0x7fffffff, hi = 0, gap_lo = 0, gap_hi = 0x7fffffff;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        lo = min(lo, lds_bounds[w][0]);
        hi = max(hi, lds_bounds[w][1]);
        gap_lo = max(gap_lo, lds_bounds[w][2]);
        gap_hi = min(gap_hi, lds_bounds[w][3]);
    }
    lo = max(it.k_begin, uniform(lo) / BN * BN);
    hi = min(k_end, uniform(hi));
    gap_lo = uniform(gap_lo);
    gap_hi = uniform(gap_hi);

    float mc = -INFINITY, l = 0.f;  // running maximum in units of log2 (both lanes of a row), the lane's part of the sum
    f32x16 acc[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            acc[cb][i] = 0.f;

    const char *k_base, *v_base;
    kv_bases(a, u, it.user, it.kv_head, k_base, v_base);
    const int32_t *table = a.k_pool ? a.block_table + (int64_t)it.user * a.max_blocks : nullptr;
    const int t_last = hi - 1;

    u32x4 sk[kPieces], sv[kPieces];
    auto load = [&](int kt) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int id = j * 256 + tid, t = min(kt + id / C, t_last);
            const int64_t off = token_offset(a, table, t) + (id % C) * 16;
            typedef const u32x4 __attribute__((address_space(1))) *global_ptr;
            sk[j] = *(global_ptr)(uintptr_t)(k_base + off);
            sv[j] = *(global_ptr)(uintptr_t)(v_base + off);
        }
    };
    auto k_place = [](int row, int c) { return row * RB + ((c ^ (row & (C < 16 ? C - 1 : 15))) * 16); };
    auto v_place = [](int row, int c) {
        const int x = kF32 ? (row & 4) << 1 : C == 16 ? (row & 7) << 1 : ((row >> 1) & 3) << 1;
        return row * RB + ((c ^ x) * 16);
    };
    auto store = [&](int buf, bool look) {
        if (look) {
            uint32_t any = 0;
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    any |= nonfinite<DT>(sv[j][i]);
            const bool bad = __builtin_amdgcn_ballot_w64(any != 0) != 0;
            if (bad)
#pragma unroll
                for (int j = 0; j < kPieces; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sv[j][i] = finite_part<DT>(sv[j][i]);
            if (lane == 0)
                lds_bad[buf][wave] = bad;
        }
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int id = j * 256 + tid;
            *reinterpret_cast<u32x4 *>(&lds[buf][0][k_place(id / C, id % C)]) = sk[j];
            *reinterpret_cast<u32x4 *>(&lds[buf][1][v_place(id / C, id % C)]) = sv[j];
        }
    };
    // tiles that no row sees between the prefixes and the windows are passed over
    auto next = [&](int kt) {
        kt += BN;
        if (kt >= gap_lo && kt + BN <= gap_hi)
            kt = gap_hi / BN * BN;
        return kt;
    };
    // a tile that some row of the workgroup may not see whole (wave by wave would do; this is what is known everywhere)
    __shared__ int lds_full[4][2];
    if (lane == 0) {
        lds_full[wave][0] = full_lo;
        lds_full[wave][1] = full_hi;
    }
    __syncthreads();
    const int all_lo = uniform(max(max(lds_full[0][0], lds_full[1][0]), max(lds_full[2][0], lds_full[3][0])));
    const int all_hi = uniform(min(min(lds_full[0][1], lds_full[1][1]), min(lds_full[2][1], lds_full[3][1])));
    auto partly = [&](int kt) { return kt < all_lo || kt + BN > all_hi; };

    const float c = MOD ? 1.f : a.score.c;
    // lane parts of the LDS places: K row n, piece 2 kk + h; V (16-bit) keys 4 h + i / 4 of sixteen channels' pieces; V (fp32) channel n
    const int k_lane = k_place(n, h);
    const int vi = lane & 15, v_row = 4 * h + vi / 4;
    const int v_lane = kF32 ? 0 : v_place(v_row, ((lane >> 4) & 1) * 2 + ((vi & 3) >> 1)) + (vi & 1) * 8;

    auto compute = [&](int buf, int kt) {
        f32x16 s[NB];
        lds_char *const kp = (lds_char *)&lds[buf][0][0], *const vp = (lds_char *)&lds[buf][1][0];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[nb][i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const u32x4 w = *(lds_u32x4 *)(kp + ((k_lane ^ (kk * 32)) + nb * 32 * RB));
                if constexpr (kF32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[nb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w[e]), __uint_as_float(q[kk][e]), s[nb], 0, 0, 0);
                } else {
                    typedef typename Block<DT>::vec8 vec8;
                    s[nb] = Block<DT>::mfma(__builtin_bit_cast(vec8, w), __builtin_bit_cast(vec8, q[kk]), s[nb]);
                }
            }
        const bool masked = kt < full_lo || kt + BN > full_hi;
        const int key0 = kt + 4 * h;
        if constexpr (MOD)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[nb][i] = modified<true, EXACT>(s[nb][i], a.score, mask, key0 + nb * 32 + 8 * (i / 4) + i % 4);
        if (masked)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[nb][i] = sees(mask, key0 + nb * 32 + 8 * (i / 4) + i % 4) ? s[nb][i] : -INFINITY;
        float mt = s[0][0];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                mt = fmaxf(mt, s[nb][i]);
        mt = wave_xor_max<32>(mt) * c;
        if (__builtin_amdgcn_ballot_w64(mt > mc + kRaise) != 0) {  // (mc is -inf at first)
            const float m_new = fmaxf(mc, mt);
            const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(mc - m_new);
            mc = m_new;
            l *= alpha;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                acc[cb] *= alpha;
        }
        const float m_p = (mc == -INFINITY ? 0.f : mc) - kShift<DT>;
        float ps = 0.f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[nb][i] = fast_exp2(fmaf(s[nb][i], c, -m_p));
                ps += s[nb][i];
            }
        l += ps;
        if constexpr (kF32) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i)
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) {
                        const int key = nb * 32 + 8 * (i / 4) + 4 * h + i % 4;
                        const uint32_t v = *(lds_u32 *)(vp + (v_place(key, cb * 8 + n / 4) + n % 4 * 4));
                        acc[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(v), s[nb][i], acc[cb], 0, 0, 0);
                    }
        } else {
            typedef typename Block<DT>::vec8 vec8;
            typedef typename Block<DT>::type E;
#pragma unroll
            for (int mb = 0; mb < 2 * NB; ++mb) {
                vec8 w[kTerms];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float left = s[mb / 2][8 * (mb & 1) + e];
#pragma unroll
                    for (int t = 0; t < kTerms; ++t) {
                        w[t][e] = (E)left;
                        left -= (float)w[t][e];
                    }
                }
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {  // sixteen keys' V^T of 32 channels: two transposed reads
                    lds_char *const p = vp + ((v_lane ^ (cb * 64)) + 16 * mb * RB);
                    union {
                        s16x4 half[2];
                        vec8 v;
                    } r;
                    r.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
                    r.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 8 * RB));
#pragma unroll
                    for (int t = 0; t < kTerms; ++t)
                        acc[cb] = Block<DT>::mfma(r.v, w[t], acc[cb]);
                }
            }
        }
        if (partly(kt) && uniform((int)(lds_bad[buf][0] | lds_bad[buf][1] | lds_bad[buf][2] | lds_bad[buf][3])) != 0) {
#pragma unroll 1
            for (int key = kt; key <= min(kt + BN - 1, t_last); ++key) {
                if (!sees(mask, key))
                    continue;
                const char *v = v_base + token_offset(a, table, key);
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        acc[cb][i] += nonfinite_part<DT>(v, cb * 32 + 8 * (i / 4) + 4 * h + i % 4);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    };

    if (lo < hi) {
        int kt = lo, buf = 0;
        if (kt >= gap_lo && kt + BN <= gap_hi)  // (a stretch can begin in the gap)
            kt = gap_hi / BN * BN;
        if (kt < hi) {
            load(kt);
            store(0, partly(kt));
        }
        __syncthreads();
        while (kt < hi) {
            const int following = next(kt);
            if (following < hi)
                load(following);
            if (kt < my_hi && kt + BN > my_lo)  // (some tiles only other waves' rows see)
                compute(buf, kt);
            if (following < hi)
                store(buf ^ 1, partly(following));
            __syncthreads();
            buf ^= 1;
            kt = following;
        }
    }

    const float total = wave_xor_sum<32>(l);
    const bool stored = wave * 32 + n < it.n_rows;
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const float lse2 = total == 0.f ? -INFINITY : (mc == -INFINITY ? 0.f : mc) + fast_log2(total) - kShift<DT>;
    const float offset = MOD ? -mask.slope * (float)mask.dist0 : 0.f;
    if (!stored)
        return;
    const int64_t at = (int64_t)(u.tok0 + token) * a.Hq + head;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                o[i] = total == 0.f ? 0.f : acc[cb][g * 4 + i] * inv;
            const int ch = cb * 32 + 8 * g + 4 * h;
            if (it.slot >= 0)
                *reinterpret_cast<f32x4 *>(a.part_o + ((int64_t)it.slot * kManyRows + wave * 32 + n) * D + ch) = o;
            else
                store4<DT>(a, at * D + ch, o);
        }
    if (h == 0) {
        if (it.slot >= 0)
            a.part_lse[(int64_t)it.slot * kManyRows + wave * 32 + n] = float2{lse2, offset};
        else
            a.lse[at] = lse2 * kLn2 + offset;
    }
}

template <int DT, int D>
void launch(bool modified, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)n_items), block(256);
    if (DT == SPD_F32 || a.out_f32) {
        if (modified)
            hipLaunchKernelGGL((tokens_many_kernel<DT, D, true, true>), grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL((tokens_many_kernel<DT, D, true, false>), grid, block, 0, stream, a);
    } else if constexpr (DT != SPD_F32) {
        if (modified)
            hipLaunchKernelGGL((tokens_many_kernel<DT, D, false, true>), grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL((tokens_many_kernel<DT, D, false, false>), grid, block, 0, stream, a);
    }
}
template <int DT>
void launch(int head_dim, bool modified, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    if (head_dim == 64)
        launch<DT, 64>(modified, n_items, a, stream);
    else
        launch<DT, 128>(modified, n_items, a, stream);
}

}  // namespace

void launch_tokens_many(int dtype, int head_dim, bool modified, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    if (dtype == SPD_F32)
        launch<SPD_F32>(head_dim, modified, n_items, a, stream);
    else if (dtype == SPD_BF16)
        launch<SPD_BF16>(head_dim, modified, n_items, a, stream);
    else
        launch<SPD_F16>(head_dim, modified, n_items, a, stream);
}

}  // namespace spd
