"""How many pages Context.spd_copy_pages says that the pools have: what it passes to the library, without a GPU."""
import pytest
import torch

import paper_2409_19134_amd as spd
from paper_2409_19134_amd import binding as b
from test_tree_host import _Stream, _context, _here

H, PAGE, D = 4, 16, 64
ELEMENTS = H * PAGE * D      # of a page


class Lib:
    """The library, whose copies are only looked at."""

    def spd_copy_pages(self, ctx, shape, views, n_views, n_pages, n_pairs, *rest):
        self.n_pages = n_pages
        return spd.SPD_OK


def pages_of(monkeypatch, *views, heads=H):
    lib = Lib()
    monkeypatch.setattr(b, "lib", lib)
    _context().spd_copy_pages(spd.make_shape(torch.bfloat16, heads, heads, D, 1.0), views, _here(torch.zeros((1, 2), dtype=torch.int32)), stream=_Stream)
    return lib.n_pages


def view(k, v, token_stride, head_stride, block_stride, **kw):
    return spd.KVView([], token_stride, head_stride, k_pool=_here(k), v_pool=_here(v), block_size=PAGE, block_stride=block_stride, **kw)


def _pool(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def test_pools_of_their_own(monkeypatch):
    assert pages_of(monkeypatch, view(_pool(8, H, PAGE, D), _pool(8, H, PAGE, D), D, PAGE * D, ELEMENTS)) == 8
    assert pages_of(monkeypatch, view(_pool(8, PAGE, H, D), _pool(9, PAGE, H, D), H * D, D, ELEMENTS)) == 8
    assert pages_of(monkeypatch, view(_pool(8 * ELEMENTS), _pool(8 * ELEMENTS + 5), D, PAGE * D, ELEMENTS)) == 8
    padded = _pool(8, 2 * H * (PAGE + 1) * D)
    assert pages_of(monkeypatch, view(padded, padded.clone(), 2 * D, 2 * (PAGE + 1) * D, padded.shape[1])) == 8
    # some of a pool's pages: those that the tensor names
    assert pages_of(monkeypatch, view(_pool(8, H, PAGE, D)[2:5], _pool(8, H, PAGE, D)[2:5], D, PAGE * D, ELEMENTS)) == 3
    few, many = (view(_pool(n, H, PAGE, D), _pool(n, H, PAGE, D), D, PAGE * D, ELEMENTS) for n in (3, 8))
    assert pages_of(monkeypatch, many, few, many) == 3


def test_k_and_v_of_a_page_side_by_side(monkeypatch):
    """The last page's V ends with the storage, behind which no whole page's distance follows."""
    flat = _pool(8 * 2 * ELEMENTS)
    assert pages_of(monkeypatch, view(flat, flat[ELEMENTS:], D, PAGE * D, 2 * ELEMENTS)) == 8
    pairs = flat.view(8, 2, H, PAGE, D)
    assert pages_of(monkeypatch, view(pairs[:, 0], pairs[:, 1], D, PAGE * D, 2 * ELEMENTS)) == 8
    # token by token
    tokens = flat.view(8, PAGE, 2, H, D)
    assert pages_of(monkeypatch, view(tokens[:, :, 0], tokens[:, :, 1], 2 * H * D, D, 2 * ELEMENTS)) == 8
    assert pages_of(monkeypatch, view(flat, flat[H * D:], 2 * H * D, D, 2 * ELEMENTS)) == 8
    # halves of one tensor
    halves = flat.view(2, 8, H, PAGE, D)
    assert pages_of(monkeypatch, view(halves[0], halves[1], D, PAGE * D, ELEMENTS)) == 8


@pytest.mark.parametrize("pages", [8, 1])
def test_heads_or_tokens_outermost(monkeypatch, pages):
    """A page's number counts within a head (or a token's place): as many pages as heads times pages would lead out of the storage."""
    k, v = (_pool(H, pages, PAGE, D) for _ in range(2))
    assert pages_of(monkeypatch, view(k, v, D, pages * PAGE * D, PAGE * D)) == pages
    assert pages_of(monkeypatch, view(k.view(-1), v.view(-1), D, pages * PAGE * D, PAGE * D)) == pages
    both = _pool(2 * H * pages * PAGE * D)      # K's tensor reaches to the end of V
    assert pages_of(monkeypatch, view(both, both[both.numel() // 2:], D, pages * PAGE * D, PAGE * D)) == pages
    k, v = (_pool(PAGE, pages, H, D) for _ in range(2))
    assert pages_of(monkeypatch, view(k, v, pages * H * D, D, H * D)) == pages
    assert pages_of(monkeypatch, view(k.view(-1), k.view(-1), pages * H * D, D, H * D)) == pages


def test_one_head(monkeypatch):
    pool = _pool(8 * PAGE * D)
    assert pages_of(monkeypatch, view(pool, pool, D, 0, PAGE * D), heads=1) == 8
    assert pages_of(monkeypatch, view(pool, pool, D, 1 << 30, PAGE * D), heads=1) == 8      # (no second head)


def test_a_number_that_the_caller_gives(monkeypatch):
    pool = _pool(8, H, PAGE, D)
    for n in (0, 5, 8):
        assert pages_of(monkeypatch, view(pool, pool, D, PAGE * D, ELEMENTS, n_pages=n)) == n
    # pages of the storage behind the tensor
    assert pages_of(monkeypatch, view(pool[2], pool[2], D, PAGE * D, ELEMENTS, n_pages=6)) == 6
    for n, x in ((9, pool), (-1, pool), (7, pool[2])):
        with pytest.raises(AssertionError):
            pages_of(monkeypatch, view(x, x, D, PAGE * D, ELEMENTS, n_pages=n))
    small = _pool(ELEMENTS - 1)      # no page at all
    assert pages_of(monkeypatch, view(small, small, D, PAGE * D, ELEMENTS)) == 0
    with pytest.raises(AssertionError):
        pages_of(monkeypatch, view(small, small, D, PAGE * D, ELEMENTS, n_pages=1))


def test_pages_that_do_not_advance_are_refused():
    pool = _pool(8, H, PAGE, D)
    for stride in (0, -ELEMENTS):
        v, shape = view(pool, pool, D, PAGE * D, stride), spd.make_shape(torch.bfloat16, H, H, D, 1.0)
        assert b.lib.spd_validate_pages(b.C.byref(shape), b._view_array([v]), 1, v.pages(shape), 1, 0x10000, None) == spd.SPD_ERR_ALIGN
