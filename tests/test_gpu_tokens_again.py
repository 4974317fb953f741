"""Calls for several tokens per user that follow other calls of the same context, and what no single call shows, against 64 bits (the tolerances are
those of test_gpu_tokens.py, whose docstring derives them)."""
import pytest
import torch

import token_reference as ref
from test_gpu_tokens import Problem

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    import paper_2409_19134_amd as spd
    c = spd.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


@pytest.mark.parametrize("layout", ["nhd", "paged_hnd16"])
@pytest.mark.parametrize("window,prefix,new,lens,q_pos", [(32, 0, [1], [64, 104], [104, 104]), (50, 0, [3], [100, 160], [159, 160]),
                                                          (2, 0, [1], [10, 13], [12, 12]), (8, 5, [2], [40, 60], [60, 60])])
def test_keys_come_into_a_window_that_lay_behind_them(ctx, layout, window, prefix, new, lens, q_pos):
    """The other owner's cache is filled piece by piece under queries whose windows begin behind its end at first."""
    import paper_2409_19134_amd as spd
    p = Problem((8, 2, 64), "bf16", layout, new, [lens[1]], dict(window=window), "f32", elsewhere=True, seed=2)
    p.prefix = [prefix] if prefix else None
    p.store()
    full_k, full_v, c = p.k, p.v, p.cache
    for n, at in zip(lens, q_pos):
        p.held, p.q_pos, p.k, p.v = [n], [at], [full_k[0][:n]], [full_v[0][:n]]
        if c.page:
            table = torch.from_numpy(c.table).to(DEV)
            c.view = spd.KVView(p.held, 64, 16 * 64, k_pool=c.k, v_pool=c.v, block_table=table, block_size=16, block_stride=2 * 16 * 64)
        else:
            c.view = spd.KVView(p.held, 2 * 64, 64, k=list(c.k), v=list(c.v))
        p.score = spd.Score(window=window, prefix=p.prefix, q_pos=p.q_pos)
        p.check(*p.call(ctx))


def test_a_token_step_whose_tokens_move_into_the_prompt(ctx):
    """One TokenStep with a window: the last token of a conversation's turn joins the others in the public cache, whose windows lie behind the prompt; the turn is moved
    into the prompt's cache, and the next one begins."""
    import paper_2409_19134_amd as spd
    Hq, H, d, dt, window, turn = 8, 2, 64, torch.float32, 32, 40
    total = 64 + 2 * turn + 3
    gen = torch.Generator().manual_seed(41)
    q, k, v = (torch.randn((total, h, d), generator=gen) for h in (Hq, H, H))
    private, public = ([torch.zeros((n, H, d), device=DEV) for _ in range(2)] for n in (total, turn + 3))
    for store, rows in zip(private, (k, v)):
        store[:64] = rows[:64].to(DEV)
    for store, rows in zip(public, (k, v)):
        store[:turn - 1] = rows[64:64 + turn - 1].to(DEV)
    prompt = spd.KVView([64], H * d, d, k=[private[0]], v=[private[1]])
    view = spd.KVView([turn - 1], H * d, d, k=[public[0]], v=[public[1]])
    step = spd.TokenStep(ctx, dt, Hq, H, d, 0.125, view, [1], prompt=prompt, window=window)
    for at in range(64 + turn - 1, 64 + 2 * turn):
        if at == 64 + turn:      # the turn's tokens move
            for a, b in zip(private, public):
                a[64:64 + turn] = b[:turn]
            prompt.lens += turn
            view.lens -= turn
        view.lens += 1
        got, lse = step.run(*(t[at:at + 1].to(DEV) for t in (q, k, v)))
        torch.cuda.synchronize()
        a, want, b, most = ref.attend(q[at:at + 1], k[:at + 1], v[:at + 1], ref.visible(1, at + 1, at, 0, True, window), 0.125)
        # (d + 4) roundings of a score, twice for the two partials' weights, and the 24-bit sums
        delta = 2 ** -24 * (2 * (d + 4) * most + 256)
        assert bool(((got.double().cpu() - a).abs() <= (2 * delta + window * 2 ** -24) * b + 1e-6).all()), at
        assert bool(((lse.double().cpu() - want).abs() <= delta + window * 2 ** -24 + 8 * 2 ** -24 * want.abs()).all()), at


@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("f16", "same"), ("f32", "f32")])
@pytest.mark.parametrize("new", [[1], [7], [200]])
def test_far_values_that_are_not_finite_reach_the_queries_that_see_them(ctx, dtype, out, new):
    """Their weights vanish beside those of the near keys (distance biases over a long cache whose stretches are joined): what is not finite still makes its
    channel not finite, in the heads that read it, and no others."""
    p = Problem((8, 2, 64), dtype, "hnd", new, [4000], dict(slopes=True), out, seed=6)
    p.v[0][5, 0, 1], p.v[0][300, 0, 9], p.v[0][2000, 1, 7] = float("inf"), float("nan"), -float("inf")
    got, lse = p.store().call(ctx)
    want = torch.ones(got.shape, dtype=torch.bool)
    want[:, :4, 1] = want[:, :4, 9] = want[:, 4:, 7] = False
    assert torch.equal(torch.isfinite(got.cpu()), want) and bool(torch.isfinite(lse).all())


def test_rotation_and_append_of_more_tokens_than_a_launch_takes(ctx):
    """2^26 tokens and a few more: what a call for the tokens around the launches' borders and at the end computes, bit by bit, and every other token copied or
    turned as well."""
    import paper_2409_19134_amd as spd
    T, d = (1 << 26) + 5, 64
    x = torch.empty((T, 1, d), dtype=torch.bfloat16, device=DEV)
    for at in range(0, T, 1 << 23):
        x[at:at + (1 << 23)].normal_()
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    rope = spd.Rope(torch.linspace(1.0, 0.001, 32, device=DEV))
    y = ctx.spd_rotate(rope, x, pos)
    for at in range(0, T, 1 << 23):
        piece = slice(at, min(T, at + (1 << 23)))
        assert torch.equal(y[piece], ctx.spd_rotate(rope, x[piece], pos[piece])), at
    k = torch.zeros(((T + 9) * d,), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    view = spd.KVView([T + 2], d, d, k=[k], v=[v])
    ctx.spd_append_tokens(spd.make_shape(torch.bfloat16, 1, 1, d, 1.0), view, [T], x, y)
    for store, rows in ((k, x), (v, y)):
        store = store.view(T + 9, d)
        assert bool((store[:2] == 0).all()) and bool((store[T + 2:] == 0).all())
        for at in range(0, T, 1 << 23):
            piece = rows[at:at + (1 << 23), 0]
            assert torch.equal(store[2 + at:2 + at + piece.shape[0]], piece), at


@pytest.mark.parametrize("layout", ["nhd", "hnd", "tables", "paged_hnd16", "paged_nhd64"])
def test_append_tables_used_again(ctx, layout):
    """A call for forty users (its table on the device), some without new tokens, again and again: all lengths move on by one, by a page, then one user's alone.
    After every call the new rows are in their places and nothing else has changed."""
    import paper_2409_19134_amd as spd
    H, d, dt = 2, 64, torch.float16
    gen = torch.Generator().manual_seed(43)
    new = [(0, 1, 3, 1, 2)[u % 5] for u in range(40)]
    held = [n + u % 23 for u, n in enumerate(new)]
    most = [l + 130 for l in held]
    rows = [[torch.randn((l, H, d), generator=gen).to(dt) for l in most] for _ in range(2)]
    cache = ref.Cache(spd, *rows, layout, DEV, seed=4)
    want = [x.clone() for x in (cache.k, cache.v)]
    where = ref.Cache.__new__(ref.Cache)
    where.__dict__.update(cache.__dict__, k=want[0], v=want[1])
    shape, T = spd.make_shape(dt, H, H, d, 1.0), sum(new)
    for move in (0, 1, 1, 16, 64, None, 1):
        if move is None:
            held[7] += 5
        else:
            held = [l + move for l in held]
        cache.view.lens[:] = held
        k_new, v_new = (torch.randn((T, H, d), generator=gen).to(dt) for _ in range(2))
        ctx.spd_append_tokens(shape, cache.view, new, k_new.to(DEV), v_new.to(DEV))
        at = 0
        for u, n in enumerate(new):
            where.put(u, held[u] - n, k_new[at:at + n], v_new[at:at + n])
            at += n
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(cache.bits(), where.bits())), move
