// Partial attention of a few query rows (16 or 32: a single token's query heads, or some tokens proposed for checking) over a stretch of one
// (user, KV head)'s keys.  Bound by the K/V bytes: each is read once for all rows.
//
// A workgroup of four waves takes a stretch; the waves take its 32-key steps in turn (16 keys with rows of 512 bytes) with the loads and
// the register layout of the streaming kernel (TileRegs, load_tile): S^T = K Q^T in 16x16 blocks whose columns are query rows, online
// softmax per column, O^T += V^T P^T with P straight from the registers that S^T arrived in.  Sums are fp32, and P enters the second product
// as three bf16 or two fp16 terms (24 and 22 bits), since partials are fp32 and V is read once however many products it goes through.
// Rows differ in what they see (causal order among the new tokens, windows, documents): a step that not every row sees whole is masked
// element by element, steps that none sees are left out.
// Measured (a read of 8 GB: 6.8 TB/s): one token of 24 users over 8192-32768 keys, 64 query heads in groups of eight, fp16 with a cap, 2.07 GB: 323 us, 6.4 TB/s;
// six tokens of 24 users over 900-8000 keys, groups of four, pages of 64, bf16, 459 MB: 85 us, 5.4 TB/s, of which the join is 5; one token of 16 users
// over 512-4096 keys with a distance bias, pages of 16, 150 MB: 33 us, 4.5 TB/s, the join 4.5: stretches of at most 13 steps, so a start (a table's
// entry, the page numbers, then the first keys: 3 us one behind the other) for a few us of loads.  One user's token over 1531 keys: 11 us, launches.
// Trees: as in the kernel for many rows; a step with keys of the tree takes a row's bits and, from memory, its eight keys' depths.  All tiles of a call are of 16 or all of 32
// rows: one launch.  Held to the registers of as many workgroups as its schedule counts on a unit (24 users' 2-4 tokens over 900-8000 keys, 128 channels, bf16: three take 86 us,
// two, where three are counted, 98).  40 users' 4-8
// tokens over 300-3000 keys, 8 KV heads of 64, fp16, 131 MB: 39 us, of which the join is 5; the waves wait for keys, 8 KB of them each, one step at a time.
#include "partial_mfma.hpp"
#include "tokens.hpp"

namespace spd {
namespace {

template <int DT>
constexpr int kTerms = DT == SPD_BF16 ? 3 : DT == SPD_F16 ? 2 : 1;

// The second product's right operand: a lane's probabilities of its NE keys, in as many terms as the type needs.
template <int DT, int NE>
struct Weights {
    typename Elt<DT>::vec8 t[kTerms<DT>];
    __device__ __forceinline__ explicit Weights(const float (&p)[NE])
    {
        static_assert(NE == 8);
        typedef typename Elt<DT>::type E;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float left = p[e];
#pragma unroll
            for (int k = 0; k < kTerms<DT>; ++k) {
                t[k][e] = (E)left;
                left -= (float)t[k][e];
            }
        }
    }
};
template <int NE>
struct Weights<SPD_F32, NE> {
    float t[NE];
    __device__ __forceinline__ explicit Weights(const float (&p)[NE])
    {
#pragma unroll
        for (int e = 0; e < NE; ++e)
            t[e] = p[e];
    }
};

// acc + V^T w for channel phase cc.
template <int DT, int D, int NA>
__device__ __forceinline__ f32x4 add_phase(const TileRegs<D * Elt<DT>::kBytes, NA> &T, int cc, const Weights<DT, 4 * NA> &w, f32x4 acc)
{
    if constexpr (DT == SPD_F32) {
#pragma unroll
        for (int e = 0; e < 4 * NA; ++e)
            acc = Elt<DT>::mfma(__uint_as_float(T.v[e].dword(cc)), w.t[e], acc);
    } else {
        typedef typename Elt<DT>::vec8 vec8;
        const unsigned sel = (cc & 1) ? 0x07060302u : 0x05040100u;  // odd channel: high halves, even: low halves
        u32x4 vt;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            vt[j] = __builtin_amdgcn_perm(T.v[2 * j + 1].dword(cc >> 1), T.v[2 * j].dword(cc >> 1), sel);
#pragma unroll
        for (int t = 0; t < kTerms<DT>; ++t)
            acc = Elt<DT>::mfma(__builtin_bit_cast(vec8, vt), w.t[t], acc);
    }
    return acc;
}

template <int DT>
__device__ __forceinline__ void keep_finite(VRow<128> &v)
{
    for (int i = 0; i < 2; ++i)
        v.w[i] = finite_part<DT>(v.w[i]);
}
template <int DT>
__device__ __forceinline__ void keep_finite(VRow<256> &v)
{
    for (int i = 0; i < 4; ++i)
        v.w[i] = finite_part<DT>(v.w[i]);
}
template <int DT>
__device__ __forceinline__ void keep_finite(VRow<512> &v)
{
    for (int i = 0; i < 4; ++i) {
        v.w0[i] = finite_part<DT>(v.w0[i]);
        v.w1[i] = finite_part<DT>(v.w1[i]);
    }
}

// One item: a tile's rows over a stretch of keys.
template <int DT, int D, bool PAGED, int NT, bool MOD, bool TREE>
__device__ __forceinline__ void few_item(const TokArgs &a, const TokItem &it, const TokUser &u)
{
    constexpr int kBytes = Elt<DT>::kBytes, RB = D * kBytes, NA = step_tiles(RB), NE = 4 * NA, kStep = 16 * NA, CP = D / 16;
    constexpr int kRows = 16 * NT;
    constexpr int kPitch = D + 4;  // floats of a staged row: the sixteen rows start in different banks
    __shared__ __attribute__((aligned(16))) float stage[4][16][kPitch];
    __shared__ float stage_ml[2][4][kRows];

    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int r = lane & 15, grp = lane >> 4;
    const int len = u.len + a.grow_len, q_pos0 = u.q_pos + a.grow_q;
    const int k_end = it.k_end + (it.to_len ? a.grow_len : 0);

    const char *k_base, *v_base;
    kv_bases(a, u, it.user, it.kv_head, k_base, v_base);

    // The lane's rows (those behind the last repeat it and are not stored).  What is loaded of them is asked for before the first keys: loads come back
    // in order, and the first products need no values yet.
    constexpr int kQ = RB / 64;
    RowMask mask[NT];
    int token[NT];
    float slope[NT];
    u32x4 q_raw[NT][kQ];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = min(it.row0 + nt * 16 + r, it.row0 + it.n_rows - 1);
        token[nt] = row / a.G;
        const int head = it.kv_head * a.G + (row - token[nt] * a.G);
        slope[nt] = MOD && a.score.slopes ? a.score.slopes[head] : 0.f;
        const char *qr = a.q + (int64_t)(u.tok0 + token[nt]) * a.q_stride + (int64_t)head * RB + grp * 16;
#pragma unroll
        for (int kk = 0; kk < kQ; ++kk)
            q_raw[nt][kk] = reinterpret_cast<const u32x4 *>(qr + kk * 64)[0];
    }
    // What the rows see: without ranges it follows from the first and the last row's positions.
    Limits lim;
    if (a.score.ranges) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            lim.add(token_mask<TREE>(a, u, len, q_pos0, token[nt], 0.f));
#pragma unroll
        for (int x = 1; x < 16; x *= 2)  // (the four lane groups hold the same rows)
            lim.add(lim.of_lane_xor(x));
        lim = lim.uniform_of();
    } else {
        lim = token_limits<TREE>(a, u, len, q_pos0, it.row0 / a.G, (it.row0 + it.n_rows - 1) / a.G);
    }
    add_tree<TREE>(lim, a, u, len);
    const int tree_begin = TREE ? plain_keys<TREE>(a, u, len) : 0;  // (without the tree inside the view: its end)
    const KeyWalk walk(lim, it.k_begin, k_end, kStep, 4);
    const int hi = walk.hi, full_lo = lim.full_lo, full_hi = min(lim.full_hi, hi);

    LaneConst L = {};
    L.r = r;
    L.grp = grp;
    L.kt = r >> 2;
    L.kc = grp;
    L.k_base = k_base;
    L.v_base = v_base;
    L.page_shift = a.page_shift;
    L.page_mask = (1 << a.page_shift) - 1;
    L.token_stride = a.token_stride;
    L.block_stride = a.block_stride;
    L.bt_row = PAGED ? a.block_table + (int64_t)it.user * a.max_blocks : nullptr;
    const int t_last = hi - 1;
    int tb = walk.first(wave);
    PagePair P = {};
    if (PAGED && tb < hi)
        P = load_pages(L, tb, t_last);

    // Two tiles' queries have no registers: every lane's pieces wait in LDS (the same for all waves).
    __shared__ __attribute__((aligned(16))) u32x4 q_lds[NT > 1 ? NT * kQ * 64 : 1];
    u32x4 qB[kQ];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int kk = 0; kk < kQ; ++kk) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                qB[kk][j] = (q_raw[nt][kk][j] & a.score.q_and) ^ a.score.q_xor;
            if (NT > 1 && wave == nt)
                q_lds[(nt * kQ + kk) * 64 + lane] = qB[kk];
        }
        mask[nt] = token_mask<TREE>(a, u, len, q_pos0, token[nt], slope[nt]);
    }
    if (NT > 1)
        __syncthreads();

    float mc[NT], l[NT];  // running maximum in units of log2 (of all rows' lanes alike), the lane's part of the sum
    f32x4 acc[NT][CP];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        mc[nt] = -INFINITY;
        l[nt] = 0.f;
#pragma unroll
        for (int cc = 0; cc < CP; ++cc)
            acc[nt][cc] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const float c = MOD ? 1.f : a.score.c;
    while (tb < hi) {
        TileRegs<RB, NA> T;
        load_tile<RB, NA, PAGED, false>(T, L, tb, t_last, P, walk.next(tb) - tb);
        const bool masked = tb < full_lo || tb + kStep > full_hi;
        const int t0 = tb + grp * NE;
        const bool in_tree = TREE && a.tree.inside && tb + kStep > tree_begin;
        int pos[TREE ? NE : 1];  // of a step with keys of the tree
        if (TREE && in_tree)
#pragma unroll
            for (int e = 0; e < NE; ++e)
                pos[e] = tree_position(a, u, tree_begin, t0 + e);
        float p[NT][NE];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if constexpr (NT > 1) {
                int at = nt * kQ * 64 + lane;
                asm volatile("" : "+v"(at));  // (read anew in every step)
#pragma unroll
                for (int kk = 0; kk < kQ; ++kk)
                    qB[kk] = q_lds[at + kk * 64];
            }
            f32x4 s[NA];
#pragma unroll
            for (int i = 0; i < NA; ++i)
                s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < RB / 64; ++kk)
#pragma unroll
                for (int i = 0; i < NA; ++i) {
                    if constexpr (kBytes == 4) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[i] = Elt<DT>::mfma(__uint_as_float(T.k[i][kk][e]), __uint_as_float(qB[kk][e]), s[i]);
                    } else {
                        typedef typename Elt<DT>::vec8 vec8;
                        s[i] = Elt<DT>::mfma(__builtin_bit_cast(vec8, T.k[i][kk]), __builtin_bit_cast(vec8, qB[kk]), s[i]);
                    }
                }
            float x[NE];
            const RunMask run(mask[nt], t0);
#pragma unroll
            for (int e = 0; e < NE; ++e)
                x[e] = modified<MOD>(s[e / 4][e % 4], a.score, mask[nt], TREE && in_tree ? mask[nt].q_pos - pos[e] : run.q - e);
            if (TREE && in_tree) {
                uint32_t branch = (uint32_t)tree_bits(a, u, tree_begin, token[nt], t0);
                if (tree_is_cut(a, u)) {
                    const TreeCut cut(a, u, token[nt]);
#pragma unroll
                    for (int e = 0; e < NE; ++e)
                        branch &= cut.leaves(mask[nt].q_pos, pos[e]) ? ~0u : ~(1u << e);
                }
#pragma unroll
                for (int e = 0; e < NE; ++e)
                    x[e] = run.sees(mask[nt], e) || (branch >> e & 1u) ? x[e] : -INFINITY;
            } else if (masked) {
#pragma unroll
                for (int e = 0; e < NE; ++e)
                    x[e] = run.sees(mask[nt], e) ? x[e] : -INFINITY;
            }
            float mt = x[0];
#pragma unroll
            for (int e = 1; e < NE; ++e)
                mt = fmaxf(mt, x[e]);
            mt = wave_xor_max<16>(mt);
            mt = wave_xor_max<32>(mt);
            const float m_new = fmaxf(mc[nt], mt * c);
            const float m_use = m_new == -INFINITY ? 0.f : m_new;  // (nothing seen yet)
            const float alpha = fast_exp2(mc[nt] - m_use);
            const float m_p = m_use - Elt<DT>::kPShift;
            float ps = 0.f;
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                p[nt][e] = fast_exp2(fmaf(x[e], c, -m_p));
                ps += p[nt][e];
            }
            l[nt] = l[nt] * alpha + ps;
            mc[nt] = m_new;
            if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
                for (int cc = 0; cc < CP; ++cc)
                    acc[nt][cc] *= alpha;
            }
            if (NT > 1)
                __builtin_amdgcn_sched_barrier(0);
        }
        bool bad = false;
        if (masked) {
            uint32_t any = 0;
#pragma unroll
            for (int e = 0; e < NE; ++e)
#pragma unroll
                for (int i = 0; i < RB / 64; ++i)
                    any |= nonfinite<DT>(T.v[e].dword(i));
            bad = __builtin_amdgcn_ballot_w64(any != 0) != 0;
            if (bad)
#pragma unroll
                for (int e = 0; e < NE; ++e)
                    keep_finite<DT>(T.v[e]);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const Weights<DT, NE> w(p[nt]);
#pragma unroll
            for (int cc = 0; cc < CP; ++cc)
                acc[nt][cc] = add_phase<DT, D, NA>(T, cc, w, acc[nt][cc]);
            if (NT > 1)  // (one tile's terms at a time: 32 rows have no registers for more)
                __builtin_amdgcn_sched_barrier(0);
        }
        if (bad) {
#pragma unroll 1
            for (int key = tb; key <= min(tb + kStep - 1, t_last); ++key) {
                const char *v = L.v_base + token_offset(a, L.bt_row, key);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if (!sees(mask[nt], key) && !(TREE && in_tree && tree_sees(a, u, tree_begin, token[nt], mask[nt].q_pos, key)))
                        continue;
#pragma unroll
                    for (int cc = 0; cc < CP; ++cc)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            acc[nt][cc][i] += nonfinite_part<DT>(v, o_channel<RB, CP>(grp * 4 + i, cc));
                }
            }
        }
        tb = walk.next(tb);
    }

    // the four waves' states, joined
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float sum = wave_xor_sum<16>(l[nt]);
        sum = wave_xor_sum<32>(sum);
        if (grp == 0) {
            stage_ml[0][wave][nt * 16 + r] = mc[nt];
            stage_ml[1][wave][nt * 16 + r] = sum;
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        if (nt > 0)
            __syncthreads();
#pragma unroll
        for (int cc = 0; cc < CP; ++cc)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                stage[wave][r][o_channel<RB, CP>(grp * 4 + i, cc)] = acc[nt][cc][i];
        __syncthreads();
        constexpr int kQuads = D / 4;  // a row's results, four channels to a thread
#pragma unroll
        for (int j = 0; j < 16 * kQuads / 256; ++j) {
            const int idx = j * 256 + tid, rr = idx / kQuads, ch = idx % kQuads * 4;
            if (nt * 16 + rr >= it.n_rows)
                continue;
            float m = stage_ml[0][0][nt * 16 + rr];
#pragma unroll
            for (int w = 1; w < 4; ++w)
                m = fmaxf(m, stage_ml[0][w][nt * 16 + rr]);
            const float m_use = m == -INFINITY ? 0.f : m;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = fast_exp2(stage_ml[0][w][nt * 16 + rr] - m_use), part = stage_ml[1][w][nt * 16 + rr];
                if (part != 0.f) {  // (a wave without keys of this row holds nothing)
                    sum += f * part;
                    o += f * *reinterpret_cast<const f32x4 *>(&stage[w][rr][ch]);
                }
            }
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            o = sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * inv;
            const float lse2 = sum == 0.f ? -INFINITY : m + fast_log2(sum) - Elt<DT>::kPShift;
            const int row = it.row0 + nt * 16 + rr, token = row / a.G, head = it.kv_head * a.G + (row - token * a.G);
            float offset = 0.f;
            if (MOD && a.score.slopes && ch == 0) {
                const RowMask mk = token_mask<TREE>(a, u, len, q_pos0, token, 0.f);
                offset = -a.score.slopes[head] * (float)mk.dist0;
            }
            if (it.slot >= 0) {
                *reinterpret_cast<f32x4 *>(a.part_o + ((int64_t)it.slot * kRows + nt * 16 + rr) * D + ch) = o;
                if (ch == 0)
                    a.part_lse[(int64_t)it.slot * kRows + nt * 16 + rr] = float2{lse2, offset};
            } else {
                const int64_t at = (int64_t)(u.tok0 + token) * a.Hq + head;
                store4<DT>(a, at * D + ch, o);
                if (ch == 0)
                    a.lse[at] = lse2 * kLn2 + offset;
            }
        }
    }
}

template <int DT, int D, bool PAGED, int NT, bool MOD, bool TREE>
__global__ __launch_bounds__(256, TREE ? tree_resident(DT, D, 16 * NT) : 2) void tokens_few_kernel(const TokArgs a)
{
    if constexpr (TREE) {
        const TreeItem x = scalar_load(reinterpret_cast<const TreeItem *>(a.items), blockIdx.x);
        few_item<DT, D, PAGED, NT, MOD, TREE>(a, x.it, x.u);
    } else {
        const TokItem it = scalar_load(a.items, blockIdx.x);
        const TokUser u = scalar_load(a.users, it.user);
        few_item<DT, D, PAGED, NT, MOD, TREE>(a, it, u);
    }
}

// Kernel template arguments from run-time values.
template <int DT, int D, bool PAGED, int NT>
void launch(bool modified, bool tree, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)n_items), block(256);
    if (tree && modified)
        hipLaunchKernelGGL((tokens_few_kernel<DT, D, PAGED, NT, true, true>), grid, block, 0, stream, a);
    else if (tree)
        hipLaunchKernelGGL((tokens_few_kernel<DT, D, PAGED, NT, false, true>), grid, block, 0, stream, a);
    else if (modified)
        hipLaunchKernelGGL((tokens_few_kernel<DT, D, PAGED, NT, true, false>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((tokens_few_kernel<DT, D, PAGED, NT, false, false>), grid, block, 0, stream, a);
}
template <int DT, int D>
void launch(bool paged, int rows, bool modified, bool tree, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    if (rows == 16)
        paged ? launch<DT, D, true, 1>(modified, tree, n_items, a, stream) : launch<DT, D, false, 1>(modified, tree, n_items, a, stream);
    else
        paged ? launch<DT, D, true, 2>(modified, tree, n_items, a, stream) : launch<DT, D, false, 2>(modified, tree, n_items, a, stream);
}
template <int DT>
void launch(int head_dim, bool paged, int rows, bool modified, bool tree, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    if (head_dim == 64)
        launch<DT, 64>(paged, rows, modified, tree, n_items, a, stream);
    else
        launch<DT, 128>(paged, rows, modified, tree, n_items, a, stream);
}

}  // namespace

void launch_tokens_few(int dtype, int head_dim, bool paged, int rows, bool modified, bool tree, int64_t n_items, const TokArgs &a, hipStream_t stream)
{
    if (dtype == SPD_F32)
        launch<SPD_F32>(head_dim, paged, rows, modified, tree, n_items, a, stream);
    else if (dtype == SPD_BF16)
        launch<SPD_BF16>(head_dim, paged, rows, modified, tree, n_items, a, stream);
    else
        launch<SPD_F16>(head_dim, paged, rows, modified, tree, n_items, a, stream);
}

}  // namespace spd
