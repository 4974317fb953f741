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
// K and V tiles go from memory straight into the other of two LDS buffers while this one's products run (no registers in between): one wait and one
// barrier a tile.  16-byte pieces of a row are stored at places xor-ed with the row's number, so that neither
// the reads of K (16 bytes of eight rows at once) nor the transposed reads of V (32 bytes of four rows) meet in a bank.
// Masks: a tile that all rows of a wave see whole costs nothing, others are masked element by element, tiles that no row sees are left out.
// Measured, 32 query heads in groups of four of 128 channels, bf16, results in bf16: 8192 tokens of documents over a cache of 16384 919-985 us, 1.0 PFLOP/s
// of what the masks leave; 16384 causal tokens 1938-2060 us, 1.07-1.13; 4096 causal tokens 148-170 us, 0.81-0.93: two tiles to a place, of which the last to end
// leave their neighbours' places empty for 30 us, and 3 us to begin a tile, 3 to end it.  A library product of 8192^3
// reaches 1.12.  With results in fp32 (P in three terms) the first takes 1564-1650, 4096 causal tokens 240-255.
// Of the first in bf16 (966 when it was taken apart) the loads are 118, the exponentials and maxima 104, LDS reads 24; matrix instructions and
// barriers alone need 673.  Tried: the next tile's scores between this tile's weights, 962-988; one V buffer and three waves per SIMD, spills, 1134.
// fp32: 252 tokens of six users over 4474 earlier ones, 64 heads in groups of eight, 2033 us, 112 TFLOP/s, with a cap 2260; 2048 causal tokens, groups of
// four, 375 us, 92 (a library product: 154; the matrix units are busy 71 % of a busy unit's time, and tiles of 128 rows compute what the diagonal masks).
//
// Trees (the forms kTree and kTreeHalf).  A query's position is its depth's.  Keys in front of the tree go by the same rules as ever; of the tree's own, in the last
// tiles, a row takes 64 bits of its set at once, shifted to the tile's first key, and their positions (for biases, windows shorter than the tree, ranges) wait in LDS.
// A workgroup's item brings its user along, and the first tile is asked for before the queries and masks are read: a chain of three dependent reads less
// where a call is a few steps of latency (one user's 16 tokens over 1531 keys, 8 KV heads of 128, 18.0 us with the join, 12.2 with this and stretches down to one step).
// Measured, 32 query heads in groups of four of 128 channels, bf16: 24 users' 50-64 tokens over 900-8000 keys 167-171 us (0.61-0.62 PFLOP/s, 478 MB at 2.8-2.9 TB/s; the matrix
// units are busy 41 % of a busy unit's time and the waves wait 32 % of theirs; with all keys in the L2 156), 28-32 tokens 111-115 (4.1 TB/s); 64 query heads, fp16 with a cap, 8
// users' 31-48 tokens over 8192-32768 keys 332-347 us.
// Tried for trees: equal pieces of all tiles' steps, a workgroup taking several tiles and up to four workgroups of an XCD a head's keys side by side: 24 users' 50-64 tokens
// 168 / 169 without, 28-32 tokens 127 / 112; four tiles of 32 keys in flight 190 / 169; a tile's page numbers read one tile ahead 167 / 164.
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
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) uint32_t lds_u32;

// Sixteen bytes from every lane's offset behind `from` to its place behind `to` (both the wave's) without a trip through registers.  Not by the builtin: the compiler then waits
// for all of them in front of every LDS read that it cannot tell from them.  Nothing but all_loads_done() and a barrier orders reads behind them.
// `to` travels in M0, as an operand: the compiler writes that register and knows when (the wait state behind the write is the asm's).
__device__ __forceinline__ void load_to_lds(const char *from, uint32_t lane_off, uint32_t to)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(to), "v"(lane_off), "s"(from) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const char *p) { return (uint32_t)uniform((int)(uint32_t)(uintptr_t)(lds_char *)p); }
__device__ __forceinline__ void all_loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// What happens to a score.  kCapped: a cap alone, for results of 16 bits: two multiplications, an addition, an exponential and a reciprocal, of which
// the softmax's own multiplication takes the last (the general form, with a copied sign, the series near zero and the bias, takes eighteen; four prompts of
// 900-4096 tokens with 32 heads of 128, us per call: 330, generally 421).  It is off by 2^-23 of twice the cap: up to a cap of 64, 2^-16, little beside a rounded P's 2^-12
// to 2^-9, but 24-bit results would show it, and a cap far above the scores would leave nothing of them.
enum { kPlain = 0, kCapped = 1, kGeneral = 2 };
constexpr float kCappedMost = 64.f * kLog2e;

constexpr float kRaise = 8.f;   // log2 of what a row's largest P may be
// P carries 2^kShift: fp16's keep to [2^-24, 65504] with a maximum of 2^(kRaise + 7)
template <int DT>
constexpr float kShift = DT == SPD_F16 ? 7.f : 0.f;

// The kernel's forms.  kTree: for the tokens of a tree.  kTreeHalf: the same for up to 64 rows: two waves share 32 rows, each takes half of every tile's keys, and
// their sums are joined at the end.  (In the other form two of four waves, and with them two of a unit's four SIMDs, would have no rows: 24 users' 14-16 tokens,
// fp32 results, 117 us for 136; fp32, six users' 60-64 tokens of 8 heads of 64, 39 for 55.)
enum { kChain = 0, kTree = 1, kTreeHalf = 2 };

template <int DT, int D, int FORM>
struct Tiles {
    static constexpr int kBytes = many_keys(DT, FORM == kTreeHalf) * D * (DT == SPD_F32 ? 4 : 2);
    char (*k)[kBytes], (*v)[kBytes];  // two buffers of each, in LDS
};

// The kernel's arguments, in the tree form read anew where a tile's end or the tree's own keys need them: the loop over the keys has no scalar registers for them.
template <bool TREE>
__device__ __forceinline__ const TokArgs &arguments(const TokArgs &a)
{
    if constexpr (!TREE)
        return a;
    const __attribute__((address_space(4))) char *p = (const __attribute__((address_space(4))) char *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const TokArgs *)(const __attribute__((address_space(4))) TokArgs *)p;
}

// One item: a tile's rows over a stretch of keys.
template <int DT, int D, bool EXACT, int MOD, int FORM>
__device__ __forceinline__ void many_item(const TokArgs &a, const TokItem &it, const TokUser &u, const Tiles<DT, D, FORM> lds)
{
    constexpr bool kF32 = DT == SPD_F32, TREE = FORM != kChain, HALF = FORM == kTreeHalf;
    constexpr int kRows = HALF ? kHalfRows : kManyRows;
    constexpr int kBytes = kF32 ? 4 : 2, RB = D * kBytes, BN = many_keys(DT, HALF), NB = BN / 32 / (HALF ? 2 : 1), C = RB / 16, KK = RB / 32, CB = D / 32;
    constexpr int kPieces = BN * C / 256;
    constexpr int kTerms = EXACT ? Block<DT>::kTerms : 1;
    auto &k_lds = lds.k;
    auto &v_lds = lds.v;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    const int rows_of = (HALF ? wave & 1 : wave) * 32, keys_of = HALF ? (wave >> 1) * (BN / 2) : 0;  // the wave's rows of the tile, and keys of every step
    const int len = u.len + a.grow_len, q_pos0 = u.q_pos + a.grow_q;
    const int k_end = it.k_end + (it.to_len ? a.grow_len : 0);

    // the lane's row, its query and masks (rows behind the last repeat it and are not stored)
    // (In the tree form worked out anew where it is needed again: the loop has no registers for it.)
    struct Place {
        int token, head;
    };
    auto place = [&](int lane_) __attribute__((always_inline)) {
        const int my_row = min(it.row0 + rows_of + (lane_ & 31), it.row0 + it.n_rows - 1), token_ = my_row / a.G;
        return Place{token_, it.kv_head * a.G + (my_row - token_ * a.G)};
    };
    const Place mine_ = place(lane);
    const int token = mine_.token, head = mine_.head;
    auto place_again = [&]() __attribute__((always_inline)) {
        if constexpr (!TREE)
            return mine_;
        int l = lane;
        asm volatile("" : "+v"(l));
        return place(l);
    };
    const float slope = a.score.slopes ? a.score.slopes[head] : 0.f;
    RowMask mask;
    u32x4 q[KK];
    auto read_row = [&]() __attribute__((always_inline)) {
        mask = token_mask<TREE>(a, u, len, q_pos0, token, slope);
        const char *qr = a.q + (int64_t)(u.tok0 + token) * a.q_stride + (int64_t)head * RB + h * 16;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                q[kk][j] = (reinterpret_cast<const u32x4 *>(qr + kk * 32)[0][j] & a.score.q_and) ^ a.score.q_xor;
    };
    if constexpr (!TREE)
        read_row();
    else if (a.score.ranges)
        mask = token_mask<TREE>(a, u, len, q_pos0, token, slope);
    // what the wave's rows see, and the workgroup's: without ranges from the first and the last row's positions
    Limits mine, all;
    if (a.score.ranges) {
        __shared__ int lds_limits[4][6];
        mine.add(mask);
#pragma unroll
        for (int x = 1; x < 32; x *= 2)  // (the wave's halves hold the same rows)
            mine.add(mine.of_lane_xor(x));
        if (lane == 0)
            mine.to(lds_limits[wave]);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w)
            all.add(Limits::from(lds_limits[w]));
        mine = mine.uniform_of();
        all = all.uniform_of();
    } else {
        auto token_of = [&](int row) { return min(it.row0 + row, it.row0 + it.n_rows - 1) / a.G; };
        mine = token_limits<TREE>(a, u, len, q_pos0, token_of(rows_of), token_of(rows_of + 31));
        all = token_limits<TREE>(a, u, len, q_pos0, token_of(0), token_of(kRows - 1));
    }
    add_tree<TREE>(mine, a, u, len);
    add_tree<TREE>(all, a, u, len);
    const int tree_begin = TREE ? plain_keys<TREE>(a, u, len) : 0;
    auto in_tree = [&](int kt) { return TREE && a.tree.inside && kt + BN > tree_begin; };  // a tile that holds keys of the tree
    const KeyWalk walk(all, it.k_begin, k_end, BN, 1);
    const int hi = walk.hi;

    float mc = -INFINITY, l[2] = {0.f, 0.f};  // running maximum in units of log2 (both lanes of a row), the lane's part of the sum (in two)
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

    // A row's pieces of sixteen bytes lie at places xor-ed with this (see above): for sixteen rows in a row all different, and for four rows in a row
    // different in the bits that tell four neighbouring pieces' groups apart.
    auto swap = [](int row) __attribute__((always_inline)) {
        if constexpr (kF32)
            return row & 7;
        else
            return C == 16 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row & 1) << 1 | (row >> 2 & 1);
    };
    // A wave's share of a tile: kPieces runs of 64 pieces, kRun rows each (inside one page: they are aligned).  What is xor-ed is the same for all
    // its runs, so a lane's place in a run stays.
    constexpr int kRun = 64 / C;
    const int run_row = lane / C;
    const uint32_t stride = (uint32_t)a.token_stride, block_stride = (uint32_t)a.block_stride;  // (the host's checks keep them below 2^31)
    const uint32_t part = ((lane % C) ^ swap(wave * kRun + run_row)) * 16;
    const uint32_t run_off = (uint32_t)(wave * kRun + run_row) * stride + part;
    const bool by_offset = !table && stride < (1u << 26);  // (a tile's rows lie less than 2^32 bytes apart)
    auto load = [&](int kt, int buf) __attribute__((always_inline)) {
        const uint32_t k_to = lds_address(k_lds[buf]) + wave * 1024, v_to = lds_address(v_lds[buf]) + wave * 1024;
        if (by_offset && kt + BN <= hi) {
            const uint64_t row = (uint64_t)(uint32_t)kt * stride;
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
                load_to_lds(k_base + row, run_off + j * 4 * kRun * stride, k_to + j * 4096);
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
                load_to_lds(v_base + row, run_off + j * 4 * kRun * stride, v_to + j * 4096);
            return;
        }
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int t = min(kt + j * 4 * kRun + wave * kRun, t_last);
            uint64_t row;
            if (table)
                row = (uint64_t)(uint32_t)scalar_load_i32(table, t >> a.page_shift) * block_stride + (uint64_t)(uint32_t)(t & ((1 << a.page_shift) - 1)) * stride;
            else
                row = (uint64_t)(uint32_t)t * stride;
            const uint32_t off = (uint32_t)min(run_row, t_last - t) * stride + part;  // rows behind the last key re-read it (they are masked)
            load_to_lds(k_base + row, off, k_to + j * 4096);
            load_to_lds(v_base + row, off, v_to + j * 4096);
        }
    };
    // a tile that some row of the workgroup may not see whole
    auto partly = [&](int kt) { return kt < all.full_lo || kt + BN > all.full_hi; };
    const float c = MOD == kPlain ? a.score.c : MOD == kCapped ? 2.f * a.score.cap_out : 1.f, steep = 2.f * kLog2e * a.score.cap_in;
    // lane parts of the LDS places: K row n, piece 2 kk + h; V (16-bit) keys 4 h + i / 4 of sixteen channels' pieces
    const int k_lane_ = (keys_of + n) * RB + (h ^ swap(n)) * 16;
    const int vi = lane & 15, v_row = keys_of + 4 * h + vi / 4, v_piece = ((lane >> 4) & 1) * 2 + ((vi & 3) >> 1);
    const int v_lane[2] = {v_row * RB + (v_piece ^ swap(v_row)) * 16 + (vi & 1) * 8, (v_row + 8) * RB + (v_piece ^ swap(v_row + 8)) * 16 + (vi & 1) * 8};

    // Pieces of the two products.  K: the rows' pieces kk of 32 keys each; V (16-bit): sixteen keys' V^T of 32 channels, by two transposed reads; V
    // (fp32): one key's values (of each half of the wave).
    auto read_k = [&](const char *kbuf, int kk, u32x4 (&f)[NB]) __attribute__((always_inline)) {
        int k_lane = k_lane_;
        if constexpr (kF32)  // (sixteen addresses are not worth a register each)
            asm volatile("" : "+v"(k_lane));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            f[nb] = *(lds_u32x4 *)((lds_char *)kbuf + ((k_lane ^ (kk * 32)) + nb * 32 * RB));
    };
    auto multiply_k = [&](const u32x4 (&f)[NB], int kk, f32x16 (&x)[NB]) __attribute__((always_inline)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            if constexpr (kF32) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[nb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(f[nb][e]), __uint_as_float(q[kk][e]), kk + e ? x[nb] : f32x16{}, 0, 0, 0);
            } else {
                typedef typename Block<DT>::vec8 vec8;
                x[nb] = Block<DT>::mfma(__builtin_bit_cast(vec8, f[nb]), __builtin_bit_cast(vec8, q[kk]), kk ? x[nb] : f32x16{});
            }
        }
    };
    constexpr int kSteps = kF32 ? 16 * NB : 2 * NB;  // of the second product: a key (of each half), or sixteen
    typedef std::conditional_t<kF32, uint32_t, u32x4> vpiece;
    auto read_v = [&](const char *vbuf, int m, vpiece (&f)[CB]) __attribute__((always_inline)) {
        lds_char *const vp = (lds_char *)vbuf;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            if constexpr (kF32) {
                int key = keys_of + 8 * (m / 4) + 4 * h + m % 4;
                asm volatile("" : "+v"(key));
                f[cb] = *(lds_u32 *)(vp + (key * RB + ((cb * 8 + n / 4) ^ swap(key)) * 16 + n % 4 * 4));
            } else {
                union {
                    s16x4 half[2];
                    u32x4 w;
                } r;
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    r.half[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vp + ((v_lane[i] ^ (cb * 64)) + 16 * m * RB)));
                f[cb] = r.w;
            }
        }
    };
    auto multiply_v = [&](const vpiece (&f)[CB], int m, const f32x16 (&p)[NB]) __attribute__((always_inline)) {
        if constexpr (kF32) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                acc[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(f[cb]), p[m / 16][m % 16], acc[cb], 0, 0, 0);
        } else {
            typedef typename Block<DT>::vec8 vec8;
            typedef typename Block<DT>::type E;
            vec8 w[kTerms];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float left = p[m / 2][8 * (m & 1) + e];
#pragma unroll
                for (int t = 0; t < kTerms; ++t) {
                    w[t][e] = (E)left;
                    left -= (float)w[t][e];
                }
            }
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int t = 0; t < kTerms; ++t)
                    acc[cb] = Block<DT>::mfma(__builtin_bit_cast(vec8, f[cb]), w[t], acc[cb]);
        }
    };
    // Scores i0 .. i1 of a tile become weights.
    auto weigh = [&](f32x16 (&p)[NB], int i0, int i1) __attribute__((always_inline)) {
        const float m_p = (mc == -INFINITY ? 0.f : mc) - kShift<DT>;
#pragma unroll
        for (int i = i0; i < i1; ++i) {
            p[i / 16][i % 16] = fast_exp2(fmaf(p[i / 16][i % 16], c, -m_p));
            l[i % 2] += p[i / 16][i % 16];
        }
    };
    auto top_of = [&](const f32x16 (&x)[NB], int i0, int i1, float m) __attribute__((always_inline)) {
#pragma unroll
        for (int i = i0; i < i1; ++i)
            m = fmaxf(m, x[i / 16][i % 16]);
        return m;
    };
    // Cap, bias and masks of the tile at kt, and the running maximum with them (top: the lane's largest score as it came).
    __shared__ __attribute__((aligned(16))) int lds_pos[TREE ? 4 : 1][64];  // positions of a tile's keys where the tree's are among them
    auto positions = [&](int nb, int g) __attribute__((always_inline)) { return *reinterpret_cast<const i32x4 *>(&lds_pos[TREE ? wave : 0][nb * 32 + 8 * g + 4 * h]); };
    // A tile with keys of the tree: their positions into LDS, and which of the lane's are on its token's branch (bit i: key kt + keys_of + 4 h + i).
    auto branch_of = [&](int kt) __attribute__((always_inline)) {
        const TokArgs &b = arguments<TREE>(a);
        lds_pos[TREE ? wave : 0][lane] = tree_position(b, u, tree_begin, kt + keys_of + lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (a wave's own LDS accesses stay in order)
        const int my_token = place_again().token;
        uint64_t bits = tree_bits(b, u, tree_begin, my_token, kt + keys_of + 4 * h);
        if (tree_is_cut(b, u)) {
            const TreeCut cut(b, u, my_token);
#pragma unroll 1
            for (int g = 0; g < 4 * NB; ++g) {
                const i32x4 pos = positions(0, g);
                uint64_t left = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    left |= cut.leaves(mask.q_pos, pos[i]) ? 1ull << i : 0ull;
                bits &= ~(15ull << 8 * g) | left << 8 * g;
            }
        }
        return bits;
    };
    auto masks = [&](f32x16 (&x)[NB], int kt, float top, uint64_t branch) __attribute__((always_inline)) {
        const int first = kt + keys_of;
        const RunMask run(mask, first + 4 * h);
        const bool masked = first < mine.full_lo || first + 32 * NB > mine.full_hi;
        if constexpr (MOD == kCapped) {  // -1 / (1 + exp(2 s / cap)): twice the cap times that, and the cap, is cap tanh(s / cap)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    x[nb][i] = fast_rcp(-1.f - fast_exp2(x[nb][i] * steep));
        } else if constexpr (MOD == kGeneral) {
            // Before all of the wave's queries a key's distance grows by one from key to key: the bias is a line, one fma per score.
            const bool before = a.score.slopes && __builtin_amdgcn_ballot_w64(run.q < 32 * NB - 1) == 0 && !in_tree(kt);
            const float nearest = mask.slope2 * (float)(mask.dist0 - run.q);
            const float f = a.score.cap_out != 0.f ? 1.f : a.score.c;
            if (a.score.cap_out != 0.f)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        x[nb][i] = capped(x[nb][i], a.score);
            if (before) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        x[nb][i] = fmaf(x[nb][i], f, fmaf(mask.slope2, (float)(nb * 32 + 8 * (i / 4) + i % 4), nearest));
            } else if (a.score.slopes && in_tree(kt)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const i32x4 pos = positions(nb, g);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            x[nb][g * 4 + i] = biased(x[nb][g * 4 + i] * f, mask, mask.q_pos - pos[i]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
            } else if (a.score.slopes) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        x[nb][i] = biased(x[nb][i] * f, mask, run.q - (nb * 32 + 8 * (i / 4) + i % 4));
            }
        }
        if (masked)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = nb * 32 + 8 * (i / 4) + i % 4;
                    x[nb][i] = run.sees(mask, key) || (TREE && (branch >> key & 1u)) ? x[nb][i] : -INFINITY;
                }
        if (MOD != kPlain || masked)
            top = top_of(x, 0, 16 * NB, -INFINITY);
        const float mt = wave_xor_max<32>(top) * c;
        if (__builtin_amdgcn_ballot_w64(mt > mc + kRaise) != 0) {  // (mc is -inf at first)
            const float m_new = fmaxf(mc, mt);
            const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(mc - m_new);
            mc = m_new;
            l[0] *= alpha;
            l[1] *= alpha;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                acc[cb] *= alpha;
        }
    };
    // Sets a tile's non-finite values of V to zero (where some row does not see some key): whether there are any.
    auto clean = [&](char *vbuf) __attribute__((always_inline)) {
        uint32_t any = 0;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(vbuf + (j * 256 + tid) * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                any |= nonfinite<DT>(w[i]);
        }
        if (__syncthreads_or(any != 0) == 0)
            return false;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            u32x4 w = *reinterpret_cast<const u32x4 *>(vbuf + (j * 256 + tid) * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = finite_part<DT>(w[i]);
            *reinterpret_cast<u32x4 *>(vbuf + (j * 256 + tid) * 16) = w;
        }
        __syncthreads();
        return true;
    };
    auto add_nonfinite = [&](int kt) __attribute__((always_inline)) {
        const TokArgs &b = arguments<TREE>(a);
        const int my_token = TREE ? place_again().token : 0;
#pragma unroll 1
        for (int key = kt + keys_of; key <= min(kt + keys_of + 32 * NB - 1, t_last); ++key) {
            if (!sees(mask, key) && !(in_tree(kt) && tree_sees(b, u, tree_begin, my_token, mask.q_pos, key)))
                continue;
            const char *v = v_base + token_offset(b, table, key);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    acc[cb][i] += nonfinite_part<DT>(v, cb * 32 + 8 * (i / 4) + 4 * h + i % 4);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };

    int kt = walk.first(0), buf = 0;
    if (kt < hi) {
        load(kt, 0);
    }
    if constexpr (TREE)
        read_row();  // (while the first tile comes)
    const bool idle = TREE && rows_of >= it.n_rows;
    while (kt < hi) {
        all_loads_done();  // the wave's own ...
        __syncthreads();   // ... and everybody's; and everybody has done with the buffers that are loaded next
        const int following = walk.next(kt);
        if (following < hi) {
            load(following, buf ^ 1);
        }
        const bool bad = partly(kt) && clean(v_lds[buf]);
        const char *const kb = k_lds[buf], *const vb = v_lds[buf];
        if (!idle && kt + keys_of < mine.any_hi && kt + keys_of + 32 * NB > mine.any_lo) {  // (some tiles only other waves' rows see)
            uint64_t branch = 0;
            if (in_tree(kt))
                branch = branch_of(kt);
            f32x16 s[NB];
            // (pieces are read one ahead of their use)
            u32x4 kf[2][NB];
            read_k(kb, 0, kf[0]);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if (kk + 1 < KK)
                    read_k(kb, kk + 1, kf[(kk + 1) & 1]);
                multiply_k(kf[kk & 1], kk, s);
                if constexpr (kF32)
                    __builtin_amdgcn_sched_barrier(0);
            }
            vpiece vf[2][CB];
            constexpr bool kLate = TREE && MOD == kGeneral;  // (no registers for it in front of the masks)
            if constexpr (!kLate)
                read_v(vb, 0, vf[0]);
            masks(s, kt, top_of(s, 0, 16 * NB, -INFINITY), branch);
            if constexpr (kLate)
                read_v(vb, 0, vf[0]);
            weigh(s, 0, 16 * NB);
#pragma unroll
            for (int m = 0; m < kSteps; ++m) {
                if (m + 1 < kSteps)
                    read_v(vb, m + 1, vf[(m + 1) & 1]);
                multiply_v(vf[m & 1], m, s);
                if constexpr (kF32 || MOD == kGeneral)  // (no further reads ahead: these have no registers for them)
                    __builtin_amdgcn_sched_barrier(0);
            }
            if (bad)
                add_nonfinite(kt);
        }
        buf ^= 1;
        kt = following;
    }

    const Place at_end = place_again();
    float total = wave_xor_sum<32>(l[0] + l[1]);
    if constexpr (HALF) {  // the second halves' sums through LDS
        static_assert(CB * 4 * 64 * 16 <= Tiles<DT, D, FORM>::kBytes);
        __shared__ float lds_ml[2][2][64];
        __syncthreads();  // (everybody has done with the tiles)
        f32x4 *const part = reinterpret_cast<f32x4 *>(k_lds[wave & 1]);
        if (wave >= 2) {
            lds_ml[0][wave & 1][lane] = mc;
            lds_ml[1][wave & 1][lane] = total;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    part[(cb * 4 + g) * 64 + lane] = f32x4{acc[cb][g * 4], acc[cb][g * 4 + 1], acc[cb][g * 4 + 2], acc[cb][g * 4 + 3]};
        }
        __syncthreads();
        if (wave >= 2)
            return;
        const float other = lds_ml[0][wave][lane], m = fmaxf(mc, other);
        const float f0 = mc == -INFINITY ? 0.f : fast_exp2(mc - m), f1 = other == -INFINITY ? 0.f : fast_exp2(other - m);
        mc = m;
        total = total * f0 + lds_ml[1][wave][lane] * f1;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 o = part[(cb * 4 + g) * 64 + lane];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[cb][g * 4 + i] = acc[cb][g * 4 + i] * f0 + o[i] * f1;
            }
    }
    const bool stored = rows_of + n < it.n_rows;
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const float lse2 = total == 0.f ? -INFINITY : (mc == -INFINITY ? 0.f : mc) + fast_log2(total) - kShift<DT> + (MOD == kCapped ? a.score.cap_out : 0.f);
    const TokArgs &b = arguments<TREE>(a);
    const float offset = MOD == kGeneral && b.score.slopes ? -b.score.slopes[at_end.head] * (float)mask.dist0 : 0.f;
    if (!stored)
        return;
    const int64_t at = (int64_t)(u.tok0 + at_end.token) * b.Hq + at_end.head;
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
                *reinterpret_cast<f32x4 *>(b.part_o + ((int64_t)it.slot * kRows + rows_of + n) * D + ch) = o;
            else
                store4<DT>(b, at * D + ch, o);
        }
    if (h == 0) {
        if (it.slot >= 0)
            b.part_lse[(int64_t)it.slot * kRows + rows_of + n] = float2{lse2, offset};
        else
            b.lse[at] = lse2 * kLn2 + offset;
    }
}

template <int DT, int D, bool EXACT, int MOD, int FORM>
__global__ __launch_bounds__(256, 2) void tokens_many_kernel(const TokArgs a)
{
    __shared__ __attribute__((aligned(16))) char k_lds[2][Tiles<DT, D, FORM>::kBytes], v_lds[2][Tiles<DT, D, FORM>::kBytes];
    const Tiles<DT, D, FORM> lds = {k_lds, v_lds};
    if constexpr (FORM != kChain) {
        const TreeItem x = scalar_load(reinterpret_cast<const TreeItem *>(a.items), blockIdx.x);
        if (x.it.n_rows == 0)
            return;  // (fills up the launch order)
        many_item<DT, D, EXACT, MOD, FORM>(a, x.it, x.u, lds);
    } else {
        const TokItem it = scalar_load(a.items, blockIdx.x);
        if (it.n_rows == 0)
            return;  // (fills up the launch order)
        const TokUser u = scalar_load(a.users, it.user);
        many_item<DT, D, EXACT, MOD, FORM>(a, it, u, lds);
    }
}

template <int DT, int D, bool EXACT, int FORM>
void launch(bool modified, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)n_items), block(256);
    if (!modified)
        hipLaunchKernelGGL((tokens_many_kernel<DT, D, EXACT, kPlain, FORM>), grid, block, 0, stream, a);
    else if (!EXACT && !a.score.slopes && a.score.cap_out <= kCappedMost)
        hipLaunchKernelGGL((tokens_many_kernel<DT, D, EXACT, EXACT ? kGeneral : kCapped, FORM>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((tokens_many_kernel<DT, D, EXACT, kGeneral, FORM>), grid, block, 0, stream, a);
}
template <int DT, int D, int FORM>
void launch(bool modified, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    if (DT == SPD_F32 || a.out_f32)
        launch<DT, D, true, FORM>(modified, n_items, a, stream);
    else if constexpr (DT != SPD_F32)
        launch<DT, D, false, FORM>(modified, n_items, a, stream);
}
template <int DT, int D>
void launch(bool modified, bool tree, bool half, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    if constexpr (has_half(DT, D))
        if (half)
            return launch<DT, D, kTreeHalf>(modified, n_items, a, stream);
    tree ? launch<DT, D, kTree>(modified, n_items, a, stream) : launch<DT, D, kChain>(modified, n_items, a, stream);
}
template <int DT>
void launch(int head_dim, bool modified, bool tree, bool half, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    if (head_dim == 64)
        launch<DT, 64>(modified, tree, half, n_items, a, stream);
    else
        launch<DT, 128>(modified, tree, half, n_items, a, stream);
}

}  // namespace

void launch_tokens_many(int dtype, int head_dim, bool modified, bool tree, bool half, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    if (dtype == SPD_F32)
        launch<SPD_F32>(head_dim, modified, tree, half, n_items, a, stream);
    else if (dtype == SPD_BF16)
        launch<SPD_BF16>(head_dim, modified, tree, half, n_items, a, stream);
    else
        launch<SPD_F16>(head_dim, modified, tree, half, n_items, a, stream);
}

}  // namespace spd
