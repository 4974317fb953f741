// Biases of trees are taken relative to the nearest key that a row sees: token_mask's distance to it, against all keys one by one, for random sets, depths and masks.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../../paper_2409_19134_amd/csrc/tokens.hpp"

using namespace spd;

int main()
{
    std::mt19937 rng(17);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    int far = 0;
    for (int round = 0; round < 20000; ++round) {
        const int words = pick(1, 3), n = pick(1, pick(0, 3) ? 12 : 64 * words), tok0 = pick(0, 3), past = pick(0, 4) ? pick(0, 300) : 0;
        const bool inside = pick(0, 4) != 0;
        std::vector<int32_t> depth((size_t)(tok0 + n)), ranges((size_t)(tok0 + n) * 2);
        std::vector<uint64_t> seen((size_t)(tok0 + n) * (size_t)words);
        for (auto &d : depth)
            d = pick(0, 5) ? pick(0, n) : pick(-3, 2000);
        const int kind = pick(0, 3);
        for (auto &w : seen)
            w = kind == 0 ? 0 : kind == 1 ? (uint64_t)rng() << 32 | rng() : ((uint64_t)rng() << 32 | rng()) & ((uint64_t)rng() << 32 | rng()) & ((uint64_t)rng() << 32 | rng());
        TokUser u = {};
        u.len = past + (inside ? n : 0);
        u.n_tok = n;
        u.tok0 = tok0;
        u.q_pos = inside ? past : pick(0, 400);
        u.k_pos = pick(0, 1) ? 0 : pick(0, 50);
        u.prefix = pick(0, 2) ? 0 : pick(0, u.len);
        for (auto &r : ranges)
            r = u.k_pos + pick(-10, past + n + 10);
        const float slope = 0.5f;
        TokArgs a = {};
        a.score.causal = pick(0, 3) != 0;
        a.score.window = pick(0, 1) ? 0 : pick(1, 60);
        a.score.ranges = pick(0, 1) ? ranges.data() : nullptr;
        a.score.slopes = &slope;
        a.tree.seen = seen.data();
        a.tree.depth = depth.data();
        a.tree.words = words;
        a.tree.inside = inside;
        const int base = inside ? past : u.len;
        for (int t = 0; t < n; ++t) {
            const RowMask m = token_mask<true>(a, u, u.len, u.q_pos, t, slope);
            int nearest = 0x7fffffff;
            for (int key = 0; key < u.len; ++key)
                if (sees(m, key) || (inside && tree_sees(a, u, base, t, m.q_pos, key)))
                    nearest = std::min(nearest, std::abs(m.q_pos - tree_position(a, u, base, key)));
            if (m.dist0 != (nearest == 0x7fffffff ? 0 : nearest)) {
                std::printf("round %d: token %d of %d behind %d: %d, the nearest key lies at %d\n", round, t, n, past, m.dist0, nearest);
                return 1;
            }
            far += inside && m.dist0 > 0;
        }
    }
    std::printf("%d tokens that do not see their own place\n", far);
    std::puts(far > 1000 ? "ok" : "too few");
    return 0;
}
