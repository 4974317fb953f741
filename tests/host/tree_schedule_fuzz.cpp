// Host logic of the attention of trees: tables and masks for random users and trees, checked against the masks' definition - every row in one tile, every key
// that a row sees in exactly one of its tile's stretches and on the walk over it, its bits and masks as they should be, every item with
// its own user beside it, partial slots given out once, in the order of the keys.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
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

int main()
{
    std::mt19937 rng(11);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    for (int round_ = 0; round_ < 500; ++round_) {
        const int heads[][2] = {{8, 8}, {8, 2}, {16, 1}, {5, 5}, {12, 3}, {14, 2}};
        const int *hd = heads[pick(0, 5)];
        const spd_shape s = {pick(0, 2), hd[0], hd[1], pick(0, 1) ? 64 : 128, 0.1f};
        const int U = pick(1, round_ % 25 ? 9 : 150), G = hd[0] / hd[1], H = hd[1], n_cus = pick(0, 2) ? 256 : pick(1, 40), words = pick(1, 4);
        std::vector<int32_t> lens(U), n_new(U), prefix(U), q_pos(U), k_pos(U);
        const bool inside = pick(0, 3) != 0, small = pick(0, 1) != 0;
        spd_score c = {};
        c.causal = pick(0, 3) != 0;
        c.window = pick(0, 1) ? 0 : pick(0, 1) ? pick(1, 20) : pick(1, 700);
        int64_t T = 0;
        for (int u = 0; u < U; ++u) {
            n_new[u] = std::min(64 * words, small ? pick(0, 9) : pick(0, 3) ? pick(0, 200) : pick(0, 3));
            lens[u] = (pick(0, 7) == 0 ? 0 : pick(0, 5) ? pick(0, 900) : pick(0, 4000)) + (inside ? n_new[u] : 0);
            prefix[u] = pick(0, 1200);
            q_pos[u] = pick(0, 2000);
            k_pos[u] = pick(0, 1) ? 0 : pick(0, 900);
            T += n_new[u];
        }
        if (pick(0, 2) == 0)
            c.prefix = prefix.data();
        if (!inside)
            c.q_pos = q_pos.data();
        if (pick(0, 1))
            c.k_pos = k_pos.data();
        std::vector<int32_t> ranges((size_t)T * 2 + 2), depth((size_t)T + 1);
        std::vector<uint64_t> seen((size_t)T * (size_t)words + 1);
        for (auto &r : ranges)
            r = pick(-10, 1500);
        for (auto &d : depth)
            d = pick(0, 9) ? pick(0, 30) : pick(-5, 2000);
        for (auto &w : seen)
            w = ((uint64_t)rng() << 32 | rng()) & ((uint64_t)rng() << 32 | rng());
        const bool with_ranges = pick(0, 3) == 0;
        std::vector<const void *> ptrs((size_t)U, reinterpret_cast<const void *>(16));
        spd_kv_view v = {};
        v.n_users = U;
        v.lens = lens.data();
        v.k_ptrs = v.v_ptrs = ptrs.data();
        v.token_stride = v.head_stride = s.head_dim;
        std::vector<TokUserPlan> plan;
        plan_users(&v, n_new.data(), &c, plan);
        TokTables tables;
        build_tok_tables(&s, &v, plan, c.causal, c.window, n_cus, tables, true);
        TokArgs a = {};
        a.G = G;
        a.score.causal = c.causal;
        a.score.window = c.window;
        a.score.ranges = with_ranges ? ranges.data() : nullptr;
        a.tree.seen = seen.data();
        a.tree.depth = depth.data();
        a.tree.words = words;
        a.tree.inside = inside;
        std::map<std::pair<int, int>, std::vector<char>> rows_done;
        for (int k = 0; k < kTokKernels; ++k) {
            const bool half = k == (int)TokKernel::kMany && tables.half;
            const int step = k == (int)TokKernel::kMany ? many_keys(s.dtype, half) : s.dtype == SPD_F32 && s.head_dim == 128 ? 16 : 32;
            const int cap = half ? kHalfRows : tile_rows((TokKernel)k), waves = k == (int)TokKernel::kMany ? 1 : 4;
            const std::vector<TreeItem> &list = tables.tree[k];
            REQUIRE(tables.items[k].empty());
            std::vector<char> slots((size_t)tables.slots[k], 0);
            std::map<std::tuple<int, int, int>, std::vector<TokItem>> tiles;
            for (const TreeItem &x : list) {
                REQUIRE(x.it.n_rows > 0 || k == (int)TokKernel::kMany);  // (the many kernel's launch order is filled up)
                if (x.it.n_rows == 0)
                    continue;
                REQUIRE(std::memcmp(&x.u, &tables.users[(size_t)x.it.user], sizeof x.u) == 0 && x.it.n_rows <= cap);
                tiles[{x.it.user, x.it.kv_head, x.it.row0}].push_back(x.it);
            }
            std::map<std::tuple<int, int, int>, TokJoin> joins;
            for (const TokJoin &j : tables.joins[k])
                joins[{j.user, j.kv_head, j.row0}] = j;
            for (auto &[key, parts] : tiles) {
                const auto [user, head, row0] = key;
                std::sort(parts.begin(), parts.end(), [](const TokItem &x, const TokItem &y) { return x.slot < y.slot; });
                if (parts.size() > 1) {
                    const auto j = joins.find(key);
                    REQUIRE(j != joins.end() && j->second.slot == parts[0].slot && j->second.n_chunks == (int)parts.size() && j->second.n_rows == parts[0].n_rows);
                    for (size_t i = 0; i < parts.size(); ++i) {
                        REQUIRE(parts[i].slot == parts[0].slot + (int)i && !slots[(size_t)parts[i].slot]);
                        slots[(size_t)parts[i].slot] = 1;
                        REQUIRE(i == 0 || parts[i].k_begin >= parts[i - 1].k_end);
                    }
                } else {
                    REQUIRE(parts[0].slot == -1 && !joins.count(key));
                }
                for (const TokItem &it : parts)
                    REQUIRE(it.k_begin % 32 == 0 && it.k_begin >= 0 && it.k_end <= lens[(size_t)user] && it.row0 == row0 && it.n_rows == parts[0].n_rows);
                std::vector<char> &done = rows_done[{user, head}];
                done.resize((size_t)n_new[(size_t)user] * (size_t)G, 0);
                const TokUser &u = tables.users[(size_t)user];
                const int len = lens[(size_t)user], n = n_new[(size_t)user], base = inside ? len - n : len;
                // the walk over each stretch, as the kernels take it
                Limits lim;
                if (with_ranges)
                    for (int r = 0; r < parts[0].n_rows; ++r)
                        lim.add(token_mask<true>(a, u, len, u.q_pos, (row0 + r) / G, 0.f));
                else
                    lim = token_limits<true>(a, u, len, u.q_pos, row0 / G, (row0 + parts[0].n_rows - 1) / G);
                add_tree<true>(lim, a, u, len);
                std::vector<int> walked((size_t)len, 0);
                for (const TokItem &it : parts) {
                    const KeyWalk walk(lim, it.k_begin, it.k_end, step, waves);
                    for (int w = 0; w < waves; ++w)
                        for (int t = walk.first(w); t < walk.hi; t = walk.next(t))
                            for (int key_ = t; key_ < std::min(t + step, walk.hi); ++key_) {
                                REQUIRE(key_ >= it.k_begin && key_ < it.k_end);
                                ++walked[(size_t)key_];
                            }
                }
                for (int w : walked)
                    REQUIRE(w <= 1);
                for (int r = 0; r < parts[0].n_rows; ++r) {
                    const int row = row0 + r, token = row / G;
                    REQUIRE(row < (int)done.size() && !done[(size_t)row]);
                    done[(size_t)row] = 1;
                    if (r % G && r > 2)
                        continue;  // (the group's heads see the same)
                    const RowMask m = token_mask<true>(a, u, len, u.q_pos, token, 0.f);
                    const int d = clampi(depth[(size_t)(u.tok0 + token)], 0, n - 1);
                    const int64_t k0 = c.k_pos ? k_pos[(size_t)user] : 0, pos_q = (inside ? k0 + base : q_pos[(size_t)user]) + d;
                    REQUIRE(m.q_pos == pos_q - k0);
                    for (int key_ = 0; key_ < len; ++key_) {
                        const bool drafted = key_ >= base;
                        const int64_t pos_k = k0 + (drafted ? base + clampi(depth[(size_t)(u.tok0 + key_ - base)], 0, n - 1) : key_);
                        const int j = key_ - base;
                        bool see = drafted ? seen[(size_t)(u.tok0 + token) * (size_t)words + (size_t)(j / 64)] >> (j % 64) & 1 : !c.causal || pos_k <= pos_q;
                        see = see && (!c.window || std::llabs(pos_q - pos_k) < c.window);
                        see = see || (!drafted && c.prefix && pos_k < prefix[(size_t)user]);
                        if (with_ranges)
                            see = see && pos_k >= ranges[2 * (size_t)(u.tok0 + token)] && pos_k < ranges[2 * (size_t)(u.tok0 + token) + 1];
                        const bool by_masks = sees(m, key_) || (inside && tree_sees(a, u, base, token, m.q_pos, key_));
                        REQUIRE(see == by_masks);
                        REQUIRE(!see || walked[(size_t)key_] == 1);
                        // rows that are not masked element by element see every key there
                        REQUIRE(see || key_ < lim.full_lo || key_ >= lim.full_hi);
                        if (inside && key_ % 7 == 0) {  // 64 keys' bits at once
                            const uint64_t bits = tree_bits(a, u, base, token, key_);
                            for (int i = 0; i < 64; ++i) {
                                const int t = key_ + i - base;
                                const bool want = t >= 0 && t < n && (seen[(size_t)(u.tok0 + token) * (size_t)words + (size_t)(t / 64)] >> (t % 64) & 1);
                                REQUIRE((bits >> i & 1) == (uint64_t)want);
                            }
                        }
                    }
                }
            }
            for (char x : slots)
                REQUIRE(x);
        }
        for (int u = 0; u < U; ++u)
            for (int h = 0; n_new[(size_t)u] && h < H; ++h)
                for (char x : rows_done[{u, h}])
                    REQUIRE(x);
        for (int u = 0; u < U; ++u)
            REQUIRE(!n_new[(size_t)u] || rows_done.count({u, 0}));
    }
    std::puts("ok");
    return 0;
}
