// Host logic of the calls for several tokens per user: tables and masks for random users, checked key by key against the masks'
// definition - every row in one tile, every key that a row sees in exactly one of its tile's stretches, stretches inside the
// caches and on whole steps, partial slots given out once; the same after lengths and positions have grown.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <tuple>

#include "../../paper_2409_19134_amd/csrc/tokens_schedule.hpp"

using namespace spd;
using namespace spd::host;

#define REQUIRE(x)                                                                \
    do {                                                                          \
        if (!(x)) {                                                               \
            std::printf("round %d line %d: %s\n", round_, __LINE__, #x);          \
            std::exit(1);                                                         \
        }                                                                         \
    } while (0)

static bool by_definition(const spd_score &c, int u, int64_t pos_q, int64_t pos_k, const int32_t *range)
{
    if (range && (pos_k < range[0] || pos_k >= range[1]))
        return false;
    if (c.prefix && pos_k < c.prefix[u])
        return true;
    if (c.causal && pos_k > pos_q)
        return false;
    return c.window == 0 || std::llabs(pos_q - pos_k) < c.window;
}

int main()
{
    std::mt19937 rng(7);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    for (int round_ = 0; round_ < 400; ++round_) {
        const int heads[][2] = {{8, 8}, {8, 2}, {16, 1}, {5, 5}, {12, 3}, {14, 2}};
        const int *hd = heads[pick(0, 5)];
        spd_shape s = {pick(0, 2), hd[0], hd[1], pick(0, 1) ? 64 : 128, 0.1f};
        const int U = pick(1, 9), G = hd[0] / hd[1], n_cus = pick(0, 2) ? 256 : pick(1, 40);
        std::vector<int32_t> lens(U), n_new(U), prefix(U), q_pos(U), k_pos(U);
        spd_score c = {};
        c.causal = pick(0, 3) != 0;
        c.window = pick(0, 2) ? 0 : pick(1, 700);
        const bool given = pick(0, 3) == 0, tokens_small = pick(0, 1);
        for (int u = 0; u < U; ++u) {
            lens[u] = pick(0, 7) == 0 ? 0 : pick(0, 5) ? pick(0, 900) : pick(0, 6000);
            n_new[u] = tokens_small ? pick(0, 9) : pick(0, 3) ? pick(0, 700) : pick(0, 3);
            if (!given)
                n_new[u] = std::min(n_new[u], lens[u]);
            prefix[u] = pick(0, 1200);
            q_pos[u] = pick(0, 2000);
            k_pos[u] = pick(0, 1) ? 0 : pick(0, 900);
        }
        if (pick(0, 2) == 0)
            c.prefix = prefix.data();
        if (given)
            c.q_pos = q_pos.data();
        if (pick(0, 1))
            c.k_pos = k_pos.data();
        int64_t T = 0;
        for (int n : n_new)
            T += n;
        std::vector<int32_t> ranges((size_t)T * 2);
        for (auto &r : ranges)
            r = pick(0, 9) ? pick(-5, 7000) : (pick(0, 1) ? INT32_MIN : INT32_MAX);
        if (pick(0, 3) == 0)
            c.ranges = ranges.data();
        spd_kv_view v = {};
        std::vector<const void *> ptrs(U, reinterpret_cast<const void *>(0x1000));
        v.n_users = U;
        v.lens = lens.data();
        v.k_ptrs = v.v_ptrs = ptrs.data();
        v.token_stride = s.head_dim;
        v.head_stride = 7000 * s.head_dim;
        std::vector<TokUserPlan> plan;
        plan_users(&v, n_new.data(), &c, plan);
        TokTables t;
        build_tok_tables(&s, &v, plan, c.causal, c.window, n_cus, t);
        const int grow_len = t.growable && pick(0, 1) ? pick(0, kMaxLen > 64 ? 64 : 1) : 0, grow_q = t.growable && pick(0, 1) ? pick(0, 64) : 0;
        ScoreArgs a = {};
        a.causal = c.causal;
        a.window = c.window;
        a.ranges = c.ranges;
        std::map<std::tuple<int, int, int>, int> rows_seen;
        for (int k = 0; k < kTokKernels; ++k) {
            const int cap = tile_rows((TokKernel)k), step = k == (int)TokKernel::kMany ? many_keys(s.dtype) : kFewKeys;
            std::map<std::tuple<int, int, int>, std::vector<const TokItem *>> tiles;
            std::set<int> slots;
            for (const TokItem &it : t.items[k]) {
                if (it.n_rows == 0) {
                    REQUIRE(k == (int)TokKernel::kMany);
                    continue;
                }
                REQUIRE(it.user >= 0 && it.user < U && it.kv_head >= 0 && it.kv_head < s.n_kv_heads);
                REQUIRE(it.n_rows <= cap && it.row0 >= 0 && it.row0 + it.n_rows <= n_new[it.user] * G);
                REQUIRE(it.k_begin >= 0 && it.k_begin <= it.k_end && it.k_end <= lens[it.user] && it.k_begin % step == 0);
                REQUIRE(it.k_end % step == 0 || it.k_end == lens[it.user]);
                REQUIRE(!it.to_len || it.k_end == lens[it.user]);
                if (it.slot >= 0)
                    REQUIRE(it.slot < t.slots[k] && slots.insert(it.slot).second);
                tiles[{it.user, it.kv_head, it.row0}].push_back(&it);
            }
            REQUIRE((int64_t)slots.size() == t.slots[k]);
            size_t split = 0;
            for (auto &[id, items] : tiles) {
                const auto [u, h, row0] = id;
                split += items.size() > 1;
                REQUIRE(items.size() == 1 ? items[0]->slot < 0 : true);
                for (const TokItem *it : items)
                    REQUIRE(it->n_rows == items[0]->n_rows && (items.size() == 1 || it->slot >= 0));
                for (int r = 0; r < items[0]->n_rows; ++r)
                    ++rows_seen[{u, h, row0 + r}];
                if (items.size() > 1) {
                    int found = 0;
                    for (const TokJoin &j : t.joins[k])
                        if (j.user == u && j.kv_head == h && j.row0 == row0) {
                            ++found;
                            REQUIRE(j.n_rows == items[0]->n_rows && j.n_chunks == (int)items.size());
                            for (const TokItem *it : items)
                                REQUIRE(it->slot >= j.slot && it->slot < j.slot + j.n_chunks);
                        }
                    REQUIRE(found == 1);
                }
                if (h != 0 && h != s.n_kv_heads - 1)
                    continue;
                // what the kernels take from a tile's first and last row holds for all of them
                const TokUser &d = t.users[u];
                if (!c.ranges) {
                    const int len = d.len + grow_len, q0 = d.q_pos + grow_q, ta = row0 / G, tb = (row0 + items[0]->n_rows - 1) / G;
                    const Limits l = tile_limits(a, d, len, q0 + ta, q0 + tb);
                    for (int token = ta; token <= tb; ++token) {
                        const RowMask m = row_mask(a, d, len, q0 + token, token, 0.f);
                        if (m.mn)
                            REQUIRE(m.mlo >= l.any_lo && m.mlo >= l.win_lo && m.mlo + (int)m.mn <= l.any_hi);
                        if (m.pn)
                            REQUIRE(m.plo >= l.any_lo && m.plo + (int)m.pn <= l.any_hi && m.plo + (int)m.pn <= l.pre_hi);
                        if (l.full_lo < l.full_hi)
                            REQUIRE(m.mlo <= l.full_lo && m.mlo + (int)m.mn >= l.full_hi);
                    }
                }
                // the steps that a kernel's waves take: every key that a row sees in exactly one, none outside of the stretch
                {
                    const int len = d.len + grow_len, q0 = d.q_pos + grow_q, waves = k == (int)TokKernel::kMany ? 1 : 4;
                    const int kstep = waves == 4 && pick(0, 1) ? 16 : step;
                    Limits l = tile_limits(a, d, len, q0 + row0 / G, q0 + (row0 + items[0]->n_rows - 1) / G);
                    std::vector<RowMask> rows;
                    for (int r = 0; r < items[0]->n_rows; ++r)
                        rows.push_back(row_mask(a, d, len, q0 + (row0 + r) / G, (row0 + r) / G, 0.f));
                    if (c.ranges) {
                        l = Limits();
                        for (const RowMask &m : rows)
                            l.add(m);
                    }
                    for (const TokItem *it : items) {
                        const int end = it->k_end + (it->to_len ? grow_len : 0);
                        const KeyWalk walk(l, it->k_begin, end, kstep, waves);
                        REQUIRE(walk.lo >= 0 && walk.hi <= end && walk.hi <= len);
                        std::vector<int> taken((size_t)len + 1, 0);
                        for (int w = 0; w < waves; ++w)
                            for (int t = walk.first(w); t < walk.hi; t = walk.next(t)) {
                                REQUIRE(t >= it->k_begin && t % kstep == 0 && walk.next(t) > t && walk.next(t) <= walk.hi);
                                for (int key = t; key < std::min(t + kstep, walk.hi); ++key)
                                    ++taken[(size_t)key];
                            }
                        for (int key = it->k_begin; key < end; ++key) {
                            REQUIRE(taken[(size_t)key] <= 1);
                            for (size_t r = 0; r < rows.size(); r += 1 + rows.size() / 5)
                                REQUIRE(!sees(rows[r], key) || taken[(size_t)key] == 1);
                        }
                    }
                }
                // key by key, for the tile's first, last and some row between
                REQUIRE(d.n_tok == n_new[u] && d.len == lens[u]);
                const int len = d.len + grow_len;
                for (int r : {0, items[0]->n_rows / 2, items[0]->n_rows - 1}) {
                    const int token = (row0 + r) / G;
                    const RowMask m = row_mask(a, d, len, d.q_pos + grow_q + token, token, 0.f);
                    const int64_t pos_q = (int64_t)d.q_pos + grow_q + token + first_key_position(&c, u);
                    for (int key = 0; key < len; ++key) {
                        const bool want = by_definition(c, u, pos_q, (int64_t)key + first_key_position(&c, u),
                                                        c.ranges ? &ranges[2 * (size_t)(d.tok0 + token)] : nullptr);
                        REQUIRE(sees(m, key) == want);
                        int covered = 0;
                        for (const TokItem *it : items)
                            covered += key >= it->k_begin && key < it->k_end + (it->to_len ? grow_len : 0);
                        REQUIRE(covered <= 1 && (!want || covered == 1));
                    }
                    REQUIRE(!sees(m, -1) && !sees(m, len));
                }
            }
            REQUIRE(split == t.joins[k].size());
        }
        size_t rows = 0;
        for (int u = 0; u < U; ++u)
            rows += (size_t)n_new[u] * G * s.n_kv_heads;
        REQUIRE(rows_seen.size() == rows);
        for (auto &x : rows_seen)
            REQUIRE(x.second == 1);
    }
    std::printf("ok 400\n");
    return 0;
}
