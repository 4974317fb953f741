"""spd_keep_tokens and spd_copy_pages against indexing on the CPU, bit for bit: what is not named stays as it was."""
import numpy as np
import pytest
import torch

import token_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    import paper_2409_19134_amd as spd
    c = spd.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


LAYOUTS = ["hnd", "nhd", "exact", "tables", "paged_hnd16", "paged_nhd16", "paged_hnd64", "paged_nhd256"]


def _caches(spd, lens, H, d, dtype, layout, layers, seed):
    gen = torch.Generator().manual_seed(seed)
    rows = [[[torch.randn((l, H, d), generator=gen).to(dtype) for l in lens] for _ in range(2)] for _ in range(layers)]
    return rows, [ref.Cache(spd, k, v, layout, DEV, seed=seed + i) for i, (k, v) in enumerate(rows)]


def _kept(rows, n_last, keep, n_keep):
    """The same on the rows of one cache: gathered from what was there."""
    out, at = [], 0
    for t, n, m in zip(rows, n_last, n_keep):
        t, b = t.clone(), t.shape[0] - n
        old = t.clone()
        for i in range(min(max(m, 0), n)):
            k = int(keep[at + i])
            if i <= k < n:
                t[b + i] = old[b + k]
        at += n
        out.append(t)
    return out


def _lists(rng, n_last, kind):
    keep, count = [], []
    for n in n_last:
        if kind == "branch":
            m = int(rng.integers(0, min(n, 8) + 1))
            x = np.sort(rng.permutation(n)[:m])
        elif kind == "window":      # the first four and the last
            m = min(n, 4 + n // 3)
            x = np.concatenate([np.arange(min(4, m)), np.arange(n - max(0, m - 4), n)])
        elif kind == "any":      # any order, some more than once, some that name no token
            m = n
            x = np.array([int(rng.integers(-2, n + 3)) if rng.random() < 0.2 else int(rng.integers(i, n)) for i in range(n)], np.int64)
        else:
            m, x = n, np.arange(n)
            if kind == "one":      # all move up by one
                x = np.append(np.arange(1, n), [0])[:n]
        count.append(m)
        keep.append(np.concatenate([x, np.full(n - len(x), 1 << 30)]))
    return np.concatenate(keep).astype(np.int32), np.array(count, np.int32)


CASES = [([1], [0]), ([26, 5, 0, 64], [100, 3, 40, 0]), ([300, 0, 33], [0, 9, 31]), ([9] * 70, [2]), ([3000], [0]), ([700, 900], [16, 15])]


@pytest.mark.parametrize("dtype,H,d", [(torch.bfloat16, 8, 128), (torch.float16, 3, 64), (torch.float32, 2, 128), (torch.float32, 1, 64)])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_kept_tokens(ctx, case, layout, dtype, H, d):
    import paper_2409_19134_amd as spd
    n_last, past = CASES[case]
    lens = [n + past[u % len(past)] for u, n in enumerate(n_last)]
    shape = spd.make_shape(dtype, H, H, d, 1.0)
    for kind in ("branch", "window", "any", "one", "same"):
        rng = np.random.default_rng(case)
        layers = 1 if case > 2 else 3
        rows, caches = _caches(spd, lens, H, d, dtype, layout, layers, seed=case)
        keep, count = _lists(rng, n_last, kind)
        ctx.spd_keep_tokens(shape, [c.view for c in caches], n_last, torch.from_numpy(keep).to(DEV), torch.from_numpy(count).to(DEV))
        torch.cuda.synchronize()
        for c, (k, v) in zip(caches, rows):
            want = ref.Cache(spd, _kept(k, n_last, keep, count), _kept(v, n_last, keep, count), layout, "cpu", seed=0) if not c.page else None
            if want is None:      # the same pages
                want = ref.Cache.__new__(ref.Cache)
                want.table, want.page, want.head_major = c.table, c.page, c.head_major
                want.k, want.v = (torch.full(t.shape, float("nan"), dtype=t.dtype) for t in (c.k, c.v))
                for u, (a, b) in enumerate(zip(_kept(k, n_last, keep, count), _kept(v, n_last, keep, count))):
                    if len(a):
                        want.put(u, 0, a, b)
            for x, y in zip(c.bits(), want.bits()):
                assert torch.equal(x, y), kind


def test_counts_are_kept_to_the_lists(ctx):
    import paper_2409_19134_amd as spd
    rows, (c,) = _caches(spd, [40, 50, 60], 2, 64, torch.bfloat16, "hnd", 1, seed=3)
    n_last, keep = [10, 20, 30], np.concatenate([np.full(10, 9), np.full(20, 19), np.full(30, 29)]).astype(np.int32)
    for count in ([-5, 1 << 30, 7], [0, 0, 0], [11, 21, 31]):
        rows, (c,) = _caches(spd, [40, 50, 60], 2, 64, torch.bfloat16, "hnd", 1, seed=3)
        ctx.spd_keep_tokens(spd.make_shape(torch.bfloat16, 2, 2, 64, 1.0), [c.view], n_last, torch.from_numpy(keep).to(DEV),
                            torch.tensor(count, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        want = ref.Cache(spd, *(_kept(t, n_last, keep, count) for t in rows[0]), "hnd", "cpu")
        assert all(torch.equal(x, y) for x, y in zip(c.bits(), want.bits()))


def test_many_layers_recorded(ctx):
    """More layers and users than one launch takes; recorded into a graph and replayed with other lists in the same memory."""
    import paper_2409_19134_amd as spd
    U, layers = 70, 35
    shape = spd.make_shape(torch.bfloat16, 2, 2, 64, 1.0)
    for layout in ("hnd", "paged_nhd16"):
        n_last = [6] * U
        rows, caches = _caches(spd, [9] * U, 2, 64, torch.bfloat16, layout, layers, seed=1)
        views = [c.view for c in caches]
        keep, count = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (6 * U, U))
        ctx.spd_keep_tokens(shape, views, n_last, keep, count)      # (nothing is kept: nothing moves)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctx.spd_keep_tokens(shape, views, n_last, keep, count)
        now = [[[t.clone() for t in x] for x in kv] for kv in rows]
        for step in range(3):
            a, b = _lists(np.random.default_rng(step), n_last, "branch")
            keep.copy_(torch.from_numpy(a))
            count.copy_(torch.from_numpy(b))
            graph.replay()
            torch.cuda.synchronize()
            now = [[_kept(x, n_last, a, b) for x in kv] for kv in now]
        for c, (k, v) in zip(caches, now):
            for u in range(U):
                got = torch.stack([c._place(c.k, u, t).cpu() for t in range(9)])
                assert torch.equal(got, k[u])
                assert torch.equal(torch.stack([c._place(c.v, u, t).cpu() for t in range(9)]), v[u])


@pytest.mark.parametrize("dtype,H,d", [(torch.bfloat16, 8, 128), (torch.float16, 3, 64), (torch.float32, 5, 128)])
@pytest.mark.parametrize("layout", ["hnd", "nhd", "padded"])
@pytest.mark.parametrize("page,pairs,layers", [(16, 1, 1), (16, 40, 3), (64, 7, 2), (256, 3, 1), (16, 5, 70)])
def test_copied_pages(ctx, dtype, H, d, layout, page, pairs, layers):
    import paper_2409_19134_amd as spd
    gen, rng = torch.Generator().manual_seed(1), np.random.default_rng(2)
    total = 2 * pairs + 3
    shape = spd.make_shape(dtype, H, H, d, 1.0)
    for partial in (False, True):
        order = rng.permutation(total)
        p = np.stack([order[:pairs], order[pairs:2 * pairs]], 1).astype(np.int32)
        extra = np.array([[total, order[-1]], [order[-1], total], [-1, order[-2]], [order[-2], order[-2]], [1 << 30, -5]], np.int32)   # left out
        given = np.concatenate([p, extra])
        n = rng.integers(-2, page + 3, len(given)).astype(np.int32)
        views, pools, old = [], [], []
        for _ in range(layers):
            kv = []
            for _ in range(2):
                if layout == "hnd":
                    t = torch.randn((total, H, page, d), generator=gen).to(dtype)
                    strides = (d, page * d, H * page * d)
                elif layout == "nhd":
                    t = torch.randn((total, page, H, d), generator=gen).to(dtype)
                    strides = (H * d, d, H * page * d)
                else:      # room between tokens, heads and pages
                    t = torch.randn((total, H * (page + 1) * 2 * d), generator=gen).to(dtype)
                    strides = (2 * d, (page + 1) * 2 * d, H * (page + 1) * 2 * d)
                kv.append(t)
            old.append(kv)
            pools.append([t.to(DEV) for t in kv])
            views.append(spd.KVView([], strides[0], strides[1], k_pool=pools[-1][0], v_pool=pools[-1][1], block_size=page, block_stride=strides[2]))
        ctx.spd_copy_pages(shape, views, torch.from_numpy(given).to(DEV), torch.from_numpy(n).to(DEV) if partial else None)
        torch.cuda.synchronize()
        for kv, got in zip(old, pools):
            for x, y in zip(kv, got):
                want = x.clone()
                for (a, b), m in zip(p.tolist(), n.tolist()):
                    m = min(max(m, 0), page) if partial else page
                    if layout == "hnd":
                        want[b, :, :m] = x[a, :, :m]
                    elif layout == "nhd":
                        want[b, :m] = x[a, :m]
                    else:
                        for h in range(H):
                            for t in range(m):
                                o = h * strides[1] + t * strides[0]
                                want[b, o:o + d] = x[a, o:o + d]
                assert torch.equal(y.cpu().view(torch.uint8), want.view(torch.uint8))


def test_pools_of_more_than_four_gigabytes(ctx):
    """Pages whose first byte lies beyond 2^32, copied and moved within."""
    import paper_2409_19134_amd as spd
    H, d, page, pages = 8, 128, 16, 135000      # 32 KB a page, 4.4 GB a pool
    shape = spd.make_shape(torch.bfloat16, H, H, d, 1.0)
    pools = [torch.zeros((pages, page, H, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    last = pages - 1
    for i, t in enumerate(pools):
        t[last] = torch.randn((page, H, d), generator=torch.Generator().manual_seed(i)).bfloat16().to(DEV)
    want = [t[last].clone() for t in pools]
    table = torch.tensor([[last - 7, last - 3]], dtype=torch.int32, device=DEV)
    view = spd.KVView([2 * page], H * d, d, k_pool=pools[0], v_pool=pools[1], block_table=table, block_size=page, block_stride=page * H * d)
    ctx.spd_copy_pages(shape, [view], torch.tensor([[last, 3], [last, last - 3]], dtype=torch.int32, device=DEV))
    keep = torch.arange(page, 2 * page, dtype=torch.int32, device=DEV).repeat(2)
    ctx.spd_keep_tokens(shape, [view], [2 * page], keep, torch.tensor([page], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for t, w in zip(pools, want):
        for at in (3, last - 3, last - 7, last):
            assert torch.equal(t[at], w)
        assert not bool(t[last - 1].any()) and not bool(t[4].any())


def test_copies_recorded_on_another_stream(ctx):
    import paper_2409_19134_amd as spd
    H, d, page = 2, 64, 16
    shape = spd.make_shape(torch.float16, H, H, d, 1.0)
    pools = [[torch.randn((12, H, page, d), device=DEV).half() for _ in range(2)] for _ in range(9)]
    views = [spd.KVView([], d, page * d, k_pool=a, v_pool=b, block_size=page, block_stride=H * page * d) for a, b in pools]
    pairs, count = torch.zeros((3, 2), dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):      # (nothing has to run before it is recorded)
        ctx.spd_copy_pages(shape, views, pairs, count)
    for step in range(3):
        rng = np.random.default_rng(step)
        p, n = rng.permutation(12)[:6].reshape(3, 2).astype(np.int32), rng.integers(0, page + 1, 3).astype(np.int32)
        want = [[t.clone() for t in kv] for kv in pools]
        for kv in want:
            for t in kv:
                for (a, b), m in zip(p.tolist(), n.tolist()):
                    t[b, :, :m] = t[a, :, :m]
        pairs.copy_(torch.from_numpy(p))
        count.copy_(torch.from_numpy(n))
        graph.replay()
        torch.cuda.synchronize()
        for kv, w in zip(pools, want):
            assert all(torch.equal(x, y) for x, y in zip(kv, w))
