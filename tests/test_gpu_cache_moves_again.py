"""Moves within caches whose views are alike in all that they have to be, and in nothing else: against indexing on the CPU, bit for bit."""
import numpy as np
import pytest
import torch

import token_reference as ref
from test_gpu_cache_moves import _caches, _kept, _lists, ctx  # noqa: F401

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype,H,d", [(torch.bfloat16, 8, 128), (torch.float32, 2, 64)])
@pytest.mark.parametrize("layout", ["paged_hnd16", "paged_nhd16", "paged_hnd64"])
@pytest.mark.parametrize("n_last,past", [([26, 5, 0, 64], [100, 3, 40, 0]), ([300, 0, 33], [0, 9, 31]), ([700, 900], [16, 15]), ([9] * 70, [2])])
def test_kept_tokens_with_tables_of_other_widths(ctx, n_last, past, layout, dtype, H, d):  # noqa: F811
    """The layers' block tables have columns behind the pages that tokens lie in, another number in each, the first one's more and less than the others'."""
    import paper_2409_19134_amd as spd
    lens = [n + past[u % len(past)] for u, n in enumerate(n_last)]
    shape = spd.make_shape(dtype, H, H, d, 1.0)
    for wider in ([0, 5, 1], [7, 0, 64]):
        rows, caches = _caches(spd, lens, H, d, dtype, layout, len(wider), seed=len(n_last))
        views = []
        for c, w in zip(caches, wider):
            bad = np.setdiff1d(np.arange(c.k.shape[0]), np.concatenate([c.table[u, :-(-l // c.page)] for u, l in enumerate(lens)]))[0]      # (no token lies there)
            table = np.concatenate([c.table, np.full((len(lens), w), bad, np.int32)], 1)
            st = c.view.struct
            views.append(spd.KVView(lens, st.token_stride, st.head_stride, k_pool=c.k, v_pool=c.v, block_table=torch.from_numpy(table).to(DEV), block_size=c.page,
                                    block_stride=st.block_stride))
        keep, count = _lists(np.random.default_rng(4), n_last, "branch" if wider[0] else "any")
        want = []
        for c, (k, v) in zip(caches, rows):
            x = ref.Cache.__new__(ref.Cache)
            x.table, x.page, x.head_major, x.k, x.v = c.table, c.page, c.head_major, c.k.cpu(), c.v.cpu()
            for u, (a, b) in enumerate(zip(_kept(k, n_last, keep, count), _kept(v, n_last, keep, count))):
                x.put(u, 0, a, b)
            want.append(x)
        ctx.spd_keep_tokens(shape, views, n_last, torch.from_numpy(keep).to(DEV), torch.from_numpy(count).to(DEV))
        torch.cuda.synchronize()
        for c, x in zip(caches, want):
            assert all(torch.equal(a, b) for a, b in zip(c.bits(), x.bits()))


@pytest.mark.parametrize("dtype,H,d", [(torch.bfloat16, 4, 64), (torch.float32, 3, 128)])
@pytest.mark.parametrize("layout", ["k_v_side_by_side", "heads_outermost", "heads_outermost_flat"])
def test_pages_of_pools_in_other_orders(ctx, layout, dtype, H, d):  # noqa: F811
    """The last page is copied, and a number that no page has is left out, whatever the storage would hold there."""
    import paper_2409_19134_amd as spd
    page, pages = 16, 8
    shape = spd.make_shape(dtype, H, H, d, 1.0)
    gen = torch.Generator().manual_seed(9)
    if layout == "k_v_side_by_side":
        flat = torch.randn(pages * 2 * H * page * d, generator=gen).to(dtype).to("cuda:0")
        whole = [flat]
        pools, strides = (flat, flat[H * page * d:]), (d, page * d, 2 * H * page * d)
        by_page = [flat.view(pages, 2, H, page, d)[:, i] for i in range(2)]
    else:
        whole = [torch.randn((H, pages, page, d), generator=gen).to(dtype).to("cuda:0") for _ in range(2)]
        pools, strides = [t.view(-1) if layout.endswith("flat") else t for t in whole], (d, pages * page * d, page * d)
        by_page = [t.transpose(0, 1) for t in whole]
    view = spd.KVView([], strides[0], strides[1], k_pool=pools[0], v_pool=pools[1], block_size=page, block_stride=strides[2])
    assert view.pages(shape) == pages
    want = [t.clone() for t in by_page]
    given = [[7, 0], [2, 6], [8, 1], [3, 9], [4, 31], [1 << 20, 5]]
    for t in want:
        t[0], t[6] = t[7].clone(), t[2].clone()
    ctx.spd_copy_pages(shape, [view], torch.tensor(given, dtype=torch.int32, device="cuda:0"))
    torch.cuda.synchronize()
    for t, w in zip(by_page, want):
        assert torch.equal(t, w)
    assert all(bool(torch.isfinite(t).all()) for t in whole)
