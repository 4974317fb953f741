"""spd_rotate and spd_append_tokens against rotary positions in 64 bits and plain indexing.

Tolerance: the turns' fraction is rounded to 24 bits (half a turn at most: an angle off by pi 2^-24), a cosine or sine by 2 units (2^-22) and by the
angle's own 64-bit rounding 2 pi |turns| 2^-52; two products and a sum of 24 bits add 3 * 2^-24 of |x0| + |x1|: together under 2^-20 of it for positions to
2^30.  The result is then rounded once to its type."""
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


def _rope(spd, d, pairs, axes, adjacent, amplitude=1.0, base=10000.0):
    inv = torch.pow(base, -torch.arange(pairs, dtype=torch.float64) / pairs).float().to(DEV)
    axis = np.random.default_rng(pairs + axes).integers(0, axes, pairs).astype(np.uint8)
    return spd.Rope(inv, axes, axis, adjacent, amplitude), inv, axis


def _close(got, want, size, pairs, adjacent, amplitude=1.0):
    """size: |x0| + |x1| of every pair."""
    d = want.shape[-1]
    bound = torch.zeros_like(want)
    i, j = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if adjacent else (slice(0, pairs), slice(pairs, 2 * pairs))
    bound[..., i] = bound[..., j] = size * abs(amplitude) * 2.0 ** -20
    # (a rounding of a value that is itself off by `bound`; fp16's steps stop shrinking at 2^-24)
    bound[..., :2 * pairs] += ref.HALF_STEP[got.dtype] * (want + bound).abs()[..., :2 * pairs] * (1 + 2.0 ** -10) + 2.0 ** -25
    off = (got.double().cpu() - want).abs()
    assert bool((off <= bound).all()), float((off - bound).max())
    if 2 * pairs < d:
        assert torch.equal(got.double().cpu()[..., 2 * pairs:], want[..., 2 * pairs:])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,pairs,axes,adjacent", [(128, 64, 1, False), (128, 64, 3, True), (64, 32, 3, False), (64, 24, 2, True), (128, 8, 1, False),
                                                   (128, 40, 2, False), (64, 8, 3, True)])
@pytest.mark.parametrize("tokens,heads", [(1, 1), (3, 40), (2061, 5)])
def test_rotate(ctx, dtype, d, pairs, axes, adjacent, tokens, heads):
    import paper_2409_19134_amd as spd
    gen = torch.Generator().manual_seed(tokens + d)
    x = torch.randn((tokens, heads, d), generator=gen).to(ref.DTYPES[dtype])
    pos = torch.randint(-50000, 200000, (axes, tokens), generator=gen, dtype=torch.int32)
    rope, inv, axis = _rope(spd, d, pairs, axes, adjacent, 1.25)
    for transposed in (False, True):
        want, size = ref.turn(x, pos, inv, axis, adjacent, 1.25, transposed)
        got = ctx.spd_rotate(rope, x.to(DEV), pos.to(DEV), transposed=transposed)
        _close(got, want, size, pairs, adjacent, 1.25)


def test_rotate_in_place_and_inside_a_projections_rows(ctx):
    """Queries and keys side by side in a projection's result, turned where they are: nothing else changes; turned back they are what they were."""
    import paper_2409_19134_amd as spd
    gen = torch.Generator().manual_seed(5)
    T, H, d = 77, 12, 64
    qkv = torch.randn((T, H + 8, d), generator=gen).to(DEV)
    before = qkv.clone()
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    rope, inv, axis = _rope(spd, d, 32, 1, False)
    x = qkv[:, 4:4 + H]
    assert ctx.spd_rotate(rope, x, pos, x) is x
    want, size = ref.turn(before[:, 4:4 + H].contiguous(), pos[None], inv, axis, False)
    _close(x, want, size, 32, False)
    assert torch.equal(qkv[:, :4], before[:, :4]) and torch.equal(qkv[:, 4 + H:], before[:, 4 + H:])
    ctx.spd_rotate(rope, x, pos, x, transposed=True)
    assert float((x - before[:, 4:4 + H]).abs().max()) < 8 * 2.0 ** -20


def test_rotate_far_positions(ctx):
    import paper_2409_19134_amd as spd
    gen = torch.Generator().manual_seed(6)
    pos = torch.tensor([[0, 1, -1, 2 ** 24 + 1, 2 ** 30, -2 ** 30, 1000003]], dtype=torch.int32)
    x = torch.randn((7, 3, 128), generator=gen)
    rope, inv, axis = _rope(spd, 128, 64, 1, False)
    want, size = ref.turn(x, pos, inv, axis, False)
    _close(ctx.spd_rotate(rope, x.to(DEV), pos.to(DEV)), want, size, 64, False)


def test_transposed_map_is_the_gradient(ctx):
    """<g, R x'> - <g, R x> along each of a few directions is <R^T g, x' - x> (fp32: the map is linear)."""
    import paper_2409_19134_amd as spd
    gen = torch.Generator(device=DEV).manual_seed(7)
    x, g, e = (torch.randn((33, 6, 64), generator=gen, device=DEV) for _ in range(3))
    pos = torch.randint(0, 3071, (2, 33), generator=gen, device=DEV, dtype=torch.int32)
    rope, _, _ = _rope(spd, 64, 24, 2, True, 0.75)
    grad = ctx.spd_rotate(rope, g, pos, transposed=True)
    diff = (g.double() * (ctx.spd_rotate(rope, x + e, pos).double() - ctx.spd_rotate(rope, x, pos).double())).sum()
    want = (grad.double() * ((x + e).double() - x.double())).sum()
    # every product off by 2^-20 of its size at most
    assert abs(float(diff - want)) <= 2.0 ** -19 * float((g.abs().double() * (x.abs() + e.abs()).double()).sum())


APPEND = [("hnd", "bf16", (32, 8, 128), [1, 1, 1, 1], [0, 7, 300, 15]), ("nhd", "f16", (8, 8, 64), [5, 0, 33], [11, 4, 0]),
          ("exact", "f32", (8, 8, 64), [3, 1, 64], [0, 9, 1]), ("tables", "bf16", (14, 2, 64), [1, 9, 2], [3, 3, 50]),
          ("paged_hnd16", "bf16", (32, 8, 128), [17, 1, 0, 40], [3, 15, 5, 31]), ("paged_nhd64", "f16", (16, 1, 128), [100, 64], [63, 0]),
          ("paged_nhd16", "f32", (5, 5, 64), [1] * 60, list(range(60))), ("nhd", "bf16", (8, 8, 128), [1500, 1, 700], [1, 2, 3])]


@pytest.mark.parametrize("layout,dtype,heads,new,past", APPEND)
@pytest.mark.parametrize("turning", ["halves", "adjacent", "partly", "none"])
def test_append(ctx, layout, dtype, heads, new, past, turning):
    """New rows land at their places turned, queries beside them, and not one other byte of the cache (or of the query buffer behind the last token) changes."""
    import paper_2409_19134_amd as spd
    (Hq, H, d), dt = heads, ref.DTYPES[dtype]
    gen = torch.Generator().manual_seed(len(new) + d)
    held = [a + b for a, b in zip(new, past)]
    rows = [[torch.randn((l, H, d), generator=gen).to(dt) for l in held] for _ in range(2)]
    cache = ref.Cache(spd, *rows, layout, DEV, seed=3)
    T = sum(new)
    qkv = torch.randn((T, Hq + 2 * H, d), generator=gen).to(dt)
    pos = torch.randint(0, 5000, (3, T), generator=gen, dtype=torch.int32)
    rope = inv = None
    P = {"halves": d // 2, "adjacent": d // 2, "partly": 24, "none": 0}[turning]
    if P:
        rope, inv, axis = _rope(spd, d, P, 3, turning == "adjacent")
    before, dev = cache.bits(), qkv.to(DEV)
    q_out = torch.full((T + 2, Hq, d), 3.0, dtype=dt, device=DEV)
    shape = spd.make_shape(dt, Hq, H, d, 1.0)
    ctx.spd_append_tokens(shape, cache.view, new, dev[:, Hq:Hq + H], dev[:, Hq + H:], rope, pos.to(DEV) if P else None, dev[:, :Hq], q_out[:T])
    got = cache.bits()
    assert bool((q_out[T:] == 3.0).all())
    turned = qkv[:, :Hq + H].double()
    if P:
        turned, size = ref.turn(qkv[:, :Hq + H].contiguous(), pos, inv, axis, turning == "adjacent")
        _close(q_out[:T], turned[:, :Hq], size[:, :Hq], P, turning == "adjacent")
    else:
        assert torch.equal(q_out[:T].cpu(), qkv[:, :Hq])
    at, mine = 0, []
    for u, n in enumerate(new):       # read the rows back, then put the old ones in their place: the cache is what it was
        for t in range(held[u] - n, held[u]):
            mine.append(cache._place(cache.k, u, t).clone())
            assert torch.equal(cache._place(cache.v, u, t).cpu(), qkv[at, Hq + H:])
            at += 1
        cache.put(u, held[u] - n, rows[0][u][held[u] - n:], rows[1][u][held[u] - n:])
    if P:
        _close(torch.stack(mine), turned[:, Hq:], size[:, Hq:], P, turning == "adjacent")
    else:
        assert torch.equal(torch.stack(mine).cpu(), qkv[:, Hq:Hq + H])
    assert all(torch.equal(a, b) for a, b in zip(before, cache.bits())) and not all(torch.equal(a, b) for a, b in zip(before, got))


def test_append_far_into_a_long_cache(ctx):
    """A token's place beyond 2^32 bytes of its buffer."""
    import paper_2409_19134_amd as spd
    d, stride, n = 64, 1 << 21, 1200             # 4 MB from token to token in bf16
    k, v = (torch.empty(n * stride, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    view = spd.KVView([n], stride, d, k=[k], v=[v])
    shape = spd.make_shape(torch.bfloat16, 2, 2, d, 1.0)
    new = torch.randn((2, 2, 2, d), device=DEV).to(torch.bfloat16)
    ctx.spd_append_tokens(shape, view, [2], new[0].contiguous(), new[1].contiguous())
    for i in range(2):
        for store, rows in ((k, new[0]), (v, new[1])):
            at = (n - 2 + i) * stride
            assert torch.equal(store[at:at + 2 * d].view(2, d), rows[i])


def test_append_recorded_in_a_graph(ctx):
    """A call for many users (its table on the device) and one for few (its table with the arguments): refused in a recording before it has run once, then
    replayed with other contents."""
    import paper_2409_19134_amd as spd
    H, d = 2, 64
    for users in (3, 130):
        gen = torch.Generator(device=DEV).manual_seed(users)
        k, v = (torch.zeros((users, H, 40, d), device=DEV) for _ in range(2))
        view = spd.KVView([20 + u % 20 for u in range(users)], d, 40 * d, k=list(k), v=list(v))
        shape = spd.make_shape(torch.float32, 4, H, d, 1.0)
        new = [1] * users
        kn, vn, q, q_out = (torch.randn((users, h, d), generator=gen, device=DEV) for h in (H, H, 4, 4))
        pos = torch.arange(users, dtype=torch.int32, device=DEV)
        rope, _, _ = _rope(spd, d, 32, 1, False)
        call = lambda: ctx.spd_append_tokens(shape, view, new, kn, vn, rope, pos, q, q_out)  # noqa: E731
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream):
            if users > 48:
                torch.cuda.synchronize()
                refused = torch.cuda.CUDAGraph()
                with torch.cuda.graph(refused, stream=stream):
                    with pytest.raises(spd.SpdError) as e:
                        call()
                assert e.value.code == spd.SPD_ERR_HIP
            call()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                call()
        for _ in range(3):
            for t in (kn, vn, q):
                t.normal_()
            pos.add_(17)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (k, v, q_out)]
            for t in (k, v, q_out):
                t.zero_()
            call()
            torch.cuda.synchronize()
            assert torch.equal(got[2], q_out)
            for u in range(users):
                at = 19 + u % 20
                assert torch.equal(got[0][u, :, at], k[u, :, at]) and torch.equal(got[1][u, :, at], v[u, :, at])


def test_rotate_recorded_without_a_run_before(ctx):
    """A rotation needs nothing of the context: it can be recorded at once, and replays follow their inputs."""
    import paper_2409_19134_amd as spd
    x, y = torch.randn((37, 6, 128), device=DEV).bfloat16(), torch.zeros((37, 6, 128), device=DEV, dtype=torch.bfloat16)
    pos = torch.zeros((2, 37), dtype=torch.int32, device=DEV)
    rope = spd.Rope(torch.linspace(1.0, 0.001, 64, device=DEV), 2, [j % 2 for j in range(64)])
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        ctx.spd_rotate(rope, x, pos, y)
    for i in range(4):
        x.normal_()
        pos.random_(0, 1 << 20)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ctx.spd_rotate(rope, x, pos))
