// The host side of the moves within caches on the runtime that is not there (see tokens_calls.cpp, whose stand-ins these are): the arguments of the launches are
// kept, and the kernel's way from them to a user's row of a block table is gone for every stream.  Run without a GPU by tests/test_cache_moves_calls.py.
#include <hip/hip_runtime.h>

#define hipLaunchKernel base_launch
#define main base_main
#include "tokens_calls.cpp"
#undef hipLaunchKernel
#undef main

#include "../../paper_2409_19134_amd/csrc/cache_moves.hpp"

struct Keep {
    KeepArgs a;
    std::vector<KeepUser> users;
    std::vector<KeepLayer> layers;
};
static std::vector<Keep> keeps;

extern "C" hipError_t hipLaunchKernel(const void *fn, dim3 grid, dim3 block, void **args, size_t lds, hipStream_t stream)
{
    if (names()[fn].find("keep_kernel") != std::string::npos) {
        Keep k;
        std::memcpy(&k.a, args[0], sizeof k.a);
        const int n_layers = k.a.n_layers, n_users = (int)(k.a.n_streams / (uint32_t)(2 * k.a.n_heads * n_layers));
        const KeepUser *u = static_cast<const KeepUsers<1> *>(args[1])->it;
        const KeepLayer *l = static_cast<const KeepLayers<1> *>(args[2])->it;
        if (k.a.first == 0)  // (the parts of a call of many streams have the same arguments)
            keeps.push_back(Keep{k.a, {u, u + n_users}, {l, l + n_layers}});
    }
    return base_launch(fn, grid, block, args, lds, stream);
}

// Views of several layers whose block tables have widths of their own: every user's pages are read from the row that its layer's width gives.
static void tables()
{
    SYM(spd_keep_tokens);
    std::mt19937 rng(3);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    for (int round = 0; round < 100; ++round) {
        spd_ctx *ctx = make();
        const int U = pick(1, round % 10 ? 9 : 150), n_views = pick(1, round % 7 ? 5 : 70);
        const spd_shape s = {pick(0, 2), 8, pick(0, 1) ? 2 : 8, pick(0, 1) ? 64 : 128, 0.1f};
        std::vector<int32_t> lens, n_last;
        for (int u = 0; u < U; ++u) {
            n_last.push_back(pick(0, 3) ? pick(0, 60) : pick(0, 700));
            lens.push_back(n_last.back() + pick(0, 40));
        }
        char *const nowhere = static_cast<char *>(kNowhere);
        const int need = (*std::max_element(lens.begin(), lens.end()) + 15) / 16;
        std::vector<spd_kv_view> views((size_t)n_views);
        for (int i = 0; i < n_views; ++i) {
            spd_kv_view &v = views[(size_t)i];
            v = {};
            v.n_users = U;
            v.lens = lens.data();
            v.token_stride = s.head_dim;
            v.head_stride = 16 * s.head_dim;
            v.block_stride = (int64_t)s.n_kv_heads * 16 * s.head_dim;
            v.block_size = 16;
            v.max_blocks = need + pick(0, 100);
            v.k_pool = nowhere + ((int64_t)(2 * i + 1) << 32);
            v.v_pool = nowhere + ((int64_t)(2 * i + 2) << 32);
            v.block_table = reinterpret_cast<const int32_t *>(nowhere + ((int64_t)(i + 1) << 20));
        }
        keeps.clear();
        if (const int rc = spd_keep_tokens_(ctx, &s, views.data(), n_views, n_last.data(), static_cast<const int32_t *>(kNowhere), static_cast<const int32_t *>(kNowhere), nullptr);
            rc != SPD_OK)
            FAIL("tables: the call fails: %d", rc);
        std::map<std::pair<int, int>, int> taken;  // (view, user)
        for (const Keep &k : keeps)
            for (const KeepLayer &l : k.layers) {
                int i = 0;
                while (i < n_views && views[(size_t)i].k_pool != l.kv[0])
                    ++i;
                if (i == n_views || l.kv[1] != views[(size_t)i].v_pool)
                    FAIL("tables: a layer's pools are no view's");
                const spd_kv_view &v = views[(size_t)i];
                for (const KeepUser &u : k.users) {
                    if (const int32_t *row = keep_row(l, u.user); row != v.block_table + (int64_t)u.user * v.max_blocks)
                        FAIL("tables: view %d of %d, user %d, %d blocks a user: the row begins at entry %lld", i, n_views, u.user, v.max_blocks, (long long)(row - v.block_table));
                    ++taken[{i, u.user}];
                }
            }
        for (int i = 0; i < n_views; ++i)
            for (int u = 0; u < U; ++u)
                if (taken[{i, u}] != (n_last[(size_t)u] > 0))
                    FAIL("tables: view %d, user %d is taken %d times", i, u, taken[{i, u}]);
        drop(ctx);
    }
}

// Buffers that are given twice, through the call that remembers tables of pointers: refused each time, whatever was remembered before and after.
static void twice()
{
    SYM(spd_keep_tokens);
    for (const bool dev : {false, true}) {
        spd_ctx *ctx = make();
        constexpr int U = 5, kViews = 3;
        const spd_shape s = {SPD_BF16, 8, 2, 64, 0.1f};
        const std::vector<int32_t> lens(U, 40), n_last = {4, 0, 9, 40, 1};
        std::vector<const void *> k[kViews], v[kViews];
        std::vector<spd_kv_view> views(kViews);
        for (int i = 0; i < kViews; ++i) {
            for (int u = 0; u < U; ++u) {
                k[i].push_back(static_cast<char *>(kNowhere) + ((int64_t)(2 * i) * U + u) * (1 << 20));
                v[i].push_back(static_cast<char *>(kNowhere) + ((int64_t)(2 * i + 1) * U + u) * (1 << 20));
            }
            spd_kv_view &x = views[(size_t)i];
            x = {};
            x.n_users = U;
            x.lens = lens.data();
            x.token_stride = 64;
            x.head_stride = 64 * 64;
            x.k_ptrs = k[i].data();
            x.v_ptrs = v[i].data();
            if (dev) {
                x.k_ptrs_dev = k[i].data();
                x.v_ptrs_dev = v[i].data();
            }
        }
        auto call = [&] {
            return spd_keep_tokens_(ctx, &s, views.data(), kViews, n_last.data(), static_cast<const int32_t *>(kNowhere), static_cast<const int32_t *>(kNowhere), nullptr);
        };
        for (int round = 0; round < 3; ++round)
            for (int u = 0; u < U; ++u) {
                const void *const own = v[2][(size_t)u];
                const size_t before = launches.size();
                const int uploaded = uploads;
                v[2][(size_t)u] = k[1][(size_t)u];
                const int rc = call();
                if (rc != (n_last[(size_t)u] ? SPD_ERR_SHAPE : SPD_OK) || (rc != SPD_OK && (launches.size() != before || uploads != uploaded)))
                    FAIL("twice: user %d of round %d: %d", u, round, rc);
                v[2][(size_t)u] = own;
                if (call() != SPD_OK)
                    FAIL("twice: the call without it fails");
            }
        drop(ctx);
    }
}

int main(int argc, char **argv)
{
    const std::string what = argc > 2 ? argv[2] : "";
    lib = argc > 2 ? dlopen(argv[1], RTLD_NOW) : nullptr;
    if (!lib)
        FAIL("cache_moves_calls <library> tables | twice");
    if (what == "tables")
        tables();
    else if (what == "twice")
        twice();
    else
        FAIL("no such part");
    std::printf("ok\n");
    return 0;
}
