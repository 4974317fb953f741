"""spd_partial_attn_tokens against attention in 64 bits from the masks' definition.

Tolerance, per element, from the inputs: a score's product of d terms rounds d times to 24 bits (off by at most d 2^-24 sum |q_c k_c|), its factor, cap
(tanh off by 2^-23 of 1, in the kernel for 16-bit results 2^-22) and bias once each, the exponential's argument and value by 2^-23 of what they are (arguments up to
64): together `delta`.  A row of L keys then has weights off by 2 delta relative to each other and sums of L terms (L 2^-24).  Probabilities enter the
second product in 24 (bf16), 22 (fp16) or 24 bits; for 16-bit results rounded once (half a step of sum p |v|).  The result is rounded to its type."""
import math

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


HEADS = [(8, 8, 64), (32, 8, 128), (14, 2, 64), (16, 1, 128), (5, 5, 64), (24, 3, 128)]
LAYOUTS = ["hnd", "nhd", "exact", "tables", "paged_hnd16", "paged_nhd16", "paged_hnd64", "paged_nhd256"]
NEW = [[1], [1, 1, 1, 1, 1], [2, 0, 5], [3, 1, 8, 2], [33, 1, 0, 4], [130], [64, 200, 1], [9, 17]]
PAST = [[0], [1, 31, 32, 33], [700, 5, 0, 90], [15, 16, 17, 64], [2500]]
SCORES = [dict(causal=False), dict(), dict(cap=5.0), dict(slopes=True), dict(window=1), dict(window=37), dict(prefix=True), dict(ranges=True),
          dict(prefix=True, window=20), dict(window=50, causal=False), dict(cap=30.0, slopes=True, window=300, prefix=True, ranges=True),
          dict(slopes=True, causal=False, ranges=True), dict(cap=50.0, causal=False, prefix=True)]


def _cases(n=120):
    """Every score with every list of new tokens, the other choices dealt out."""
    rng = np.random.default_rng(11)
    out = []
    for i, score in enumerate(SCORES):
        for j, new in enumerate(NEW):
            pick = lambda x: x[int(rng.integers(len(x)))]  # noqa: E731
            out.append((i, j, pick(HEADS), pick(["f32", "bf16", "f16"]), pick(LAYOUTS), pick(PAST), pick(["f32", "same"]), pick([False, False, True])))
    return out


class Problem:
    """One call: caches, queries, the score's parts, and the result in 64 bits."""

    def __init__(self, heads, dtype, layout, new, past, score, out, elsewhere=False, seed=1, scale=None, q_scale=2.0, fill=float("nan")):
        import paper_2409_19134_amd as spd
        self.spd, (self.Hq, self.H, self.d) = spd, heads
        self.dt = ref.DTYPES[dtype]
        self.out_dt = torch.float32 if out == "f32" else self.dt
        gen, rng, U = torch.Generator().manual_seed(seed), np.random.default_rng(seed), len(new)
        self.new = new
        past = [past[u % len(past)] for u in range(U)]
        self.held = [p if elsewhere else p + n for p, n in zip(past, new)]      # elsewhere: the tokens follow the view's keys, in another cache
        self.k, self.v = ([torch.randn((l, self.H, self.d), generator=gen).to(self.dt) for l in self.held] for _ in range(2))
        self.T = sum(new)
        self.q = (q_scale * torch.randn((self.T, self.Hq, self.d), generator=gen)).to(self.dt)
        self.scale = 1 / math.sqrt(self.d) if scale is None else scale
        self.causal, self.window, self.cap = score.get("causal", True), score.get("window", 0), score.get("cap", 0.0)
        self.k_pos = [int(x) for x in rng.integers(0, 50, U)] if seed % 2 else [0] * U
        self.q_pos = [kp + l + int(rng.integers(0, 9)) for kp, l in zip(self.k_pos, self.held)] if elsewhere else [kp + l - n for kp, l, n in
                                                                                                     zip(self.k_pos, self.held, new)]
        self.prefix = [int(x) for x in rng.integers(0, 2 + 2 * (max(self.held) // 3), U)] if score.get("prefix") else None
        self.slopes = torch.pow(2.0, -8.0 * (torch.arange(self.Hq) + 1) / self.Hq) if score.get("slopes") else None
        self.ranges = None
        if score.get("ranges"):
            parts = []
            for u, n in enumerate(new):
                lo = self.k_pos[u] + rng.integers(-5, self.held[u] + 5, n)
                size = rng.integers(-3, 60 + self.held[u], n)      # some empty, some that end before they begin
                parts.append(np.stack([lo, lo + size], 1))
            self.ranges = np.concatenate(parts).astype(np.int32).reshape(-1, 2)
        self.elsewhere, self.layout, self.fill, self.seed = elsewhere, layout, fill, seed
        self.shape = spd.make_shape(self.dt, *heads, self.scale)

    def store(self):
        self.cache = ref.Cache(self.spd, self.k, self.v, self.layout, DEV, seed=self.seed, fill=self.fill)
        self.score = self.spd.Score(cap=self.cap, slopes=None if self.slopes is None else self.slopes.float().to(DEV), causal=self.causal,
                                    window=self.window, prefix=self.prefix, ranges=None if self.ranges is None else torch.from_numpy(self.ranges).to(DEV),
                                    q_pos=self.q_pos if self.elsewhere else None, k_pos=self.k_pos if any(self.k_pos) else None)
        return self

    def call(self, ctx, stream=None):
        T, Hq, d = self.T, self.Hq, self.d
        out = torch.full((T + 3, Hq, d), 7.0, dtype=self.out_dt, device=DEV)
        lse = torch.full((T + 3, Hq), 7.0, device=DEV)
        wide = torch.full((T, Hq + 3, d), float("nan"), dtype=self.dt, device=DEV)      # the queries as a slice of wider rows
        wide[:, 1:1 + Hq] = self.q.to(DEV)
        ctx.spd_partial_attn_tokens(self.shape, wide[:, 1:1 + Hq], self.cache.view, self.new, self.score, out[:T], lse[:T], stream=stream)
        torch.cuda.synchronize()
        assert bool((out[T:] == 7.0).all()) and bool((lse[T:] == 7.0).all())
        return out[:T].clone(), lse[:T].clone()

    def exact(self):
        at, parts, self.most = 0, [], 0.0
        for u, n in enumerate(self.new):
            see = ref.visible(n, self.held[u], self.q_pos[u], self.k_pos[u], self.causal, self.window, None if self.prefix is None else self.prefix[u],
                              None if self.ranges is None else self.ranges[at:at + n])
            apart = torch.from_numpy(np.abs(self.q_pos[u] + np.arange(n)[:, None] - self.k_pos[u] - np.arange(self.held[u])[None])).double()
            a, lse, b, most = ref.attend(self.q[at:at + n], self.k[u], self.v[u], see, self.scale, self.cap,
                                         None if self.slopes is None else self.slopes.float().double(), apart)
            parts.append((a, lse, b, torch.from_numpy(see.any(1) if see.shape[1] else np.zeros(n, bool))))
            self.most = max(self.most, most)
            at += n
        return [torch.cat([p[i] for p in parts]) for i in range(4)]

    def check(self, out, lse):
        a, want_lse, b, any_key = self.exact()
        L = max(self.held + [1])
        eps = 2.0 ** -24
        delta = (self.d + 4) * eps * self.most + 2 * 64 * 2 * eps + (self.cap * (4 if self.out_dt == torch.float32 else 8) * eps)
        if self.slopes is not None:
            delta += 4 * eps * 64      # relative to the nearest key: terms beyond 64 vanish
        weights = 2 * delta + L * eps + {torch.float32: 2 * eps, torch.bfloat16: 2 * eps, torch.float16: 2.0 ** -21}[self.dt]
        if self.out_dt != torch.float32:
            weights += ref.HALF_STEP[self.dt]
        # a rounding of a value off by that much; fp16's steps stop shrinking at 2^-24
        bound = weights * b * 1.01 + ref.HALF_STEP[self.out_dt] * a.abs() * 1.01 + (2.0 ** -25 if self.out_dt == torch.float16 else 1e-12)
        off = (out.double().cpu() - a).abs()
        assert bool((off <= bound).all()), (float(off.max()), float((off - bound).max()))
        got = lse.double().cpu()
        assert bool((got[~any_key] == -np.inf).all()) and bool((out.cpu()[~any_key] == 0).all())
        g, w = got[any_key], want_lse[any_key]
        assert bool(((g - w).abs() <= delta + L * eps + 4 * eps * w.abs() + 2 * eps).all()), float((g - w).abs().max())


@pytest.mark.parametrize("case", _cases(), ids=lambda c: f"{c[0]}-{c[1]}-{'x'.join(map(str, c[2]))}-{c[3]}-{c[4]}-{c[5][0]}-{c[6]}-{int(c[7])}")
def test_attention_of_several_tokens(ctx, case):
    i, j, heads, dtype, layout, past, out, elsewhere = case
    p = Problem(heads, dtype, layout, NEW[j], past, SCORES[i], out, elsewhere, seed=100 + 13 * i + j).store()
    p.check(*p.call(ctx))


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "same"), ("f16", "f32"), ("f16", "same")])
@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 8, 64)])
@pytest.mark.parametrize("new", [[1], [3], [8, 5], [300]])
def test_every_kernel_and_type(ctx, heads, dtype, out, new):
    for k, score in enumerate((dict(), dict(cap=20.0, slopes=True))):
        for layout in ("hnd", "paged_nhd16"):
            p = Problem(heads, dtype, layout, new, [401, 77], score, out, seed=30 + k).store()
            p.check(*p.call(ctx))


@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0])
@pytest.mark.parametrize("new", [[1, 2], [60]])
def test_scales(ctx, scale, new):
    """No scale at all (every visible key alike), a negative one, one that makes rows nearly one-hot."""
    for dtype in ("bf16", "f32"):
        for score in (dict(), dict(cap=4.0)):
            p = Problem((8, 2, 64), dtype, "hnd", new, [90, 300], score, "f32", seed=9, scale=scale).store()
            p.check(*p.call(ctx))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [[3, 4], [7], [150]])
@pytest.mark.parametrize("kind", ["causal", "window", "ranges", "prefix"])
def test_what_a_query_does_not_see_does_not_reach_it(ctx, dtype, d, new, kind):
    """NaN and infinities in keys and values that some queries see and others do not: those that do not have the result without them; those
    that do have a value that is not finite in exactly those channels (values), and anything (keys)."""
    score = {"causal": dict(), "window": dict(window=9), "ranges": dict(ranges=True), "prefix": dict(prefix=True, window=5)}[kind]
    clean = Problem((8, 2, d), dtype, "hnd", new, [70, 40], score, "f32", seed=21)
    for part in ("v", "k"):
        dirty = Problem((8, 2, d), dtype, "hnd", new, [70, 40], score, "f32", seed=21)
        spots = []
        for u, l in enumerate(dirty.held):
            for x, (t, h, c) in enumerate(((l - 1, 0, 3), (l // 2, 1, 0), (2, 0, d - 1), (l - 2, 1, 5), (l - 2, 0, 5))):
                if part == "k" and x in (1, 2):      # (early keys: most rows see them, and one such key is all of a row's result)
                    continue
                getattr(dirty, part)[u][t, h, c] = (math.nan, math.inf, -math.inf, math.inf, -math.inf)[x]
                spots.append((u, t, h, c))
        a, _, _, _ = clean.exact()
        out, lse = dirty.store().call(ctx)
        base, base_lse = clean.store().call(ctx)
        touched, hit = torch.zeros((clean.T, 8, d), dtype=torch.bool), torch.zeros((clean.T, 8), dtype=torch.bool)
        for u, t, h, c in spots:
            at = sum(new[:u])
            see = ref.visible(new[u], clean.held[u], clean.q_pos[u], clean.k_pos[u], clean.causal, clean.window,
                              None if clean.prefix is None else clean.prefix[u], None if clean.ranges is None else clean.ranges[at:at + new[u]])
            rows = torch.from_numpy(np.nonzero(see[:, t])[0]) + at
            for g in range(4):
                hit[rows, 4 * h + g] = True
                touched[rows, 4 * h + g, c] = True
        if part == "v":
            assert torch.equal(lse.cpu(), base_lse.cpu())
            assert torch.equal(torch.isfinite(out.cpu()), ~touched)
            assert torch.equal(out.cpu()[~touched], base.cpu()[~touched])
        else:
            # rows that see none of it: the same sums; a tile's running maximum may differ by what other rows' keys no longer raise, so to rounding
            keep = ~hit
            assert bool(keep.any()) and bool(torch.isfinite(out.cpu()[keep]).all())
            assert bool(((out.cpu().double() - a)[keep].abs() <= (base.cpu().double() - a)[keep].abs().max() + 2.0 ** -20).all())


def test_values_that_are_not_finite_stay_in_their_channel(ctx):
    """... of the heads that read them, in steps that all rows see whole as well as in masked ones."""
    for new in ([1], [2], [140]):
        for dtype in ("bf16", "f32"):
            p = Problem((8, 2, 64), dtype, "nhd", new, [200], dict(), "f32", seed=3)
            p.v[0][5, 0, 1], p.v[0][40, 0, 2], p.v[0][41, 0, 2], p.v[0][80, 1, 7] = math.inf, math.inf, -math.inf, math.nan
            out, _ = p.store().call(ctx)
            want = torch.ones(out.shape, dtype=torch.bool)
            want[:, :4, 1:3] = want[:, 4:, 7] = False
            assert torch.equal(torch.isfinite(out.cpu()), want)


def test_rows_that_see_nothing(ctx):
    """Empty caches, empty ranges, queries before every key: A = 0, lse = -inf, beside rows that see something."""
    import paper_2409_19134_amd as spd
    for dtype in ("bf16", "f32"):
        for new in ([2, 3], [90, 70]):
            p = Problem((8, 2, 64), dtype, "hnd", new, [60, 0], dict(), "f32", elsewhere=True, seed=4).store()      # the second user's cache is empty
            out, lse = p.call(ctx)
            p.check(out, lse)
            assert bool((lse[new[0]:] == -math.inf).all())
            p.q_pos, p.k_pos, p.elsewhere = [10, 10], [11 + new[0] // 2, 900], True
            p.score = spd.Score(causal=True, q_pos=p.q_pos, k_pos=p.k_pos)
            p.check(*p.call(ctx))


def test_no_users_and_no_tokens(ctx):
    import paper_2409_19134_amd as spd
    shape = spd.make_shape(torch.bfloat16, 8, 2, 64, 1.0)
    q = torch.empty((0, 8, 64), dtype=torch.bfloat16, device=DEV)
    for lens in ([], [0, 5]):
        k = [torch.zeros((2, 8, 64), dtype=torch.bfloat16, device=DEV) for _ in lens]
        view = spd.KVView(lens, 64, 8 * 64, k=k, v=k)
        out, lse = ctx.spd_partial_attn_tokens(shape, q, view, [0] * len(lens))
        assert out.shape == (0, 8, 64) and lse.shape == (0, 8)
        ctx.spd_append_tokens(shape, view, [0] * len(lens), q[:, :2], q[:, :2])


def test_single_tokens_equal_the_decode_call(ctx):
    """One token per user and plain scores: what spd_partial_attn_private computes, to rounding."""
    p = Problem((32, 8, 128), "bf16", "paged_nhd16", [1] * 6, [3, 700, 2000, 64], dict(causal=False), "f32", seed=6).store()
    out, lse = p.call(ctx)
    a, l = ctx.spd_partial_attn_private(p.shape, p.q.to(DEV), p.cache.view)
    assert float((a - out).abs().max()) < 2e-4 and float((l - lse).abs().max()) < 1e-5


def test_the_same_call_twice_has_the_same_bits(ctx):
    for new in ([1, 1], [7], [200]):
        p = Problem((32, 8, 128), "bf16", "hnd", new, [3000, 900], dict(cap=20.0), "f32", seed=8).store()
        first, second = p.call(ctx), p.call(ctx)
        assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])


def test_a_growing_cache_is_served_by_its_schedule(ctx):
    """A decode loop: lengths grow by a token and step, and the queries with them; every step against 64 bits."""
    import paper_2409_19134_amd as spd
    for new, score in (([1, 1], dict()), ([2, 1], dict(window=50, prefix=True)), ([1, 1], dict(slopes=True))):
        p = Problem((8, 2, 64), "bf16", "paged_hnd16", new, [100, 230], score, "f32", seed=14)
        full_k, full_v = ([torch.randn((l + 80, 2, 64)).to(p.dt) for l in p.held] for _ in range(2))
        start, first_q = list(p.held), list(p.q_pos)
        p.k, p.v = full_k, full_v
        p.held = [l + 80 for l in start]
        p.store()
        for step in (0, 1, 2, 30, 64, 65, 80):
            p.held = [l + step for l in start]
            p.k, p.v = [x[:l] for x, l in zip(full_k, p.held)], [x[:l] for x, l in zip(full_v, p.held)]
            p.q_pos = [x + step for x in first_q]
            c = p.cache
            table = torch.from_numpy(c.table).to(DEV)
            c.view = spd.KVView(p.held, 64, 16 * 64, k_pool=c.k, v_pool=c.v, block_table=table, block_size=16, block_stride=2 * 16 * 64)
            p.check(*p.call(ctx))


def test_queries_move_on_over_a_cache_that_does_not_grow(ctx):
    """The prompt's owner in a decode loop: its keys stay, the queries' positions grow (windows and biases move)."""
    import paper_2409_19134_amd as spd
    p = Problem((8, 2, 64), "f16", "hnd", [1, 2], [300, 129], dict(window=120, slopes=True), "f32", elsewhere=True, seed=15).store()
    first = list(p.q_pos)
    for step in (0, 1, 5, 64, 66):
        p.q_pos = [x + step for x in first]
        p.score = spd.Score(causal=True, window=120, slopes=p.score.slopes, q_pos=p.q_pos, k_pos=p.k_pos)
        p.check(*p.call(ctx))


def test_far_into_a_long_cache(ctx):
    """Keys beyond 2^32 bytes of a buffer, for the kernels of few and of many rows."""
    import paper_2409_19134_amd as spd
    d, stride, n = 64, 1 << 21, 1200
    k, v = (torch.empty(n * stride, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    rows = torch.randn((2, n, d), device=DEV).to(torch.bfloat16)
    for store, r in ((k, rows[0]), (v, rows[1])):
        store.view(n, stride)[:, :d] = r
    view = spd.KVView([n], stride, d, k=[k], v=[v])
    shape = spd.make_shape(torch.bfloat16, 1, 1, d, 0.125)
    for tokens in (1, 40):
        q = torch.randn((tokens, 1, d), device=DEV).to(torch.bfloat16)
        out, _ = ctx.spd_partial_attn_tokens(shape, q, view, [tokens], spd.Score(causal=True))
        see = ref.visible(tokens, n, n - tokens, 0, True)
        a, _, b, most = ref.attend(q, rows[0][:, None], rows[1][:, None], see, 0.125)
        assert bool(((out.double().cpu() - a).abs() <= ((d + 4) * 2 ** -23 * most + n * 2 ** -24 + 2 ** -15) * b).all())


def test_two_contexts_on_two_streams(ctx):
    """Calls that overlap in time on contexts of their own."""
    import paper_2409_19134_amd as spd
    other = spd.Context(0)
    p = Problem((32, 8, 128), "bf16", "hnd", [4, 1, 1], [2000, 900], dict(), "f32", seed=16).store()
    r = Problem((32, 8, 128), "bf16", "nhd", [300], [500], dict(cap=9.0), "f32", seed=17).store()
    want = [x.call(ctx) for x in (p, r)]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    q = [x.q.to(DEV) for x in (p, r)]
    got = []
    torch.cuda.synchronize()
    for _ in range(5):
        for x, y, c, s in ((p, q[0], ctx, a), (r, q[1], other, b)):
            with torch.cuda.stream(s):
                got.append(c.spd_partial_attn_tokens(x.shape, y, x.cache.view, x.new, x.score))
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(got):
        assert torch.equal(out, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])
    other.close()


def test_a_schedule_built_on_one_stream_serves_another(ctx):
    """Calls on two streams, one behind the other: the second finds the first one's schedule."""
    p = Problem((8, 2, 64), "bf16", "hnd", [1, 3], [777, 52], dict(), "f32", seed=18).store()
    q = p.q.to(DEV)
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(first):
        ctx.spd_partial_attn_tokens(p.shape, q, p.cache.view, p.new, p.score)
    second.wait_stream(first)
    with torch.cuda.stream(second):
        out, lse = ctx.spd_partial_attn_tokens(p.shape, q, p.cache.view, p.new, p.score)
    torch.cuda.synchronize()
    p.check(out, lse)


def test_recorded_in_a_graph(ctx):
    """Refused before it has run once, then recorded; replays follow their inputs while other calls of the context come and go (more views than it
    remembers, scratch memory outgrown)."""
    import paper_2409_19134_amd as spd
    own = spd.Context(0)
    p = Problem((32, 8, 128), "bf16", "hnd", [1, 2, 1], [1500, 300, 40], dict(cap=20.0), "f32", seed=19).store()
    q = p.q.to(DEV)
    out, lse = torch.empty((p.T, 32, 128), device=DEV), torch.empty((p.T, 32), device=DEV)
    call = lambda c=own: c.spd_partial_attn_tokens(p.shape, q, p.cache.view, p.new, p.score, out, lse)  # noqa: E731
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        refused = torch.cuda.CUDAGraph()
        with torch.cuda.graph(refused, stream=stream):
            with pytest.raises(spd.SpdError) as e:
                call()
        assert e.value.code == spd.SPD_ERR_HIP
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
    for i in range(4):
        for j in range(40):      # other views of the same context
            k = [torch.zeros((2, 3071, 64), dtype=torch.bfloat16, device=DEV)]
            view = spd.KVView([1000 + 40 * i + 70 * j if j else 2900], 64, 64 * 3071, k=k, v=k)
            tokens = 1 if j else 1 + i
            own.spd_partial_attn_tokens(spd.make_shape(torch.bfloat16, 32, 2, 64, 1.0), torch.zeros((tokens, 32, 64), dtype=torch.bfloat16, device=DEV),
                                        view, [tokens])
        torch.cuda.synchronize()
        q.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        call(ctx)
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)
    own.close()


def test_many_views_come_and_go(ctx):
    """More views than the context remembers, each then again."""
    for _ in range(2):
        for n in range(150):
            p = Problem((2, 1, 64), "f32", "hnd", [1 + n % 5], [n], dict(), "f32", seed=40 + n).store()
            out, lse = p.call(ctx)
            if n % 29 == 0:
                p.check(out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("turned", [True, False])
def test_token_step(ctx, dtype, turned):
    """The operators together: a prompt goes into the private cache (turned on the way), then tokens that follow it - three at once, then one each, with capped
    scores - into the public one; their attention over both caches, merged, is attention over the whole sequence in 64 bits."""
    import paper_2409_19134_amd as spd
    Hq, H, d, dt = 8, 2, 64, ref.DTYPES[dtype]
    gen = torch.Generator().manual_seed(23)
    prompt, later = [70, 1, 133], [[3, 3, 3], [1, 1, 1]]
    total = [p + 4 for p in prompt]
    x = [[torch.randn((l, h, d), generator=gen).to(dt) for l in total] for h in (Hq, H, H)]
    inv = torch.pow(10000.0, -torch.arange(32, dtype=torch.float64) / 32).float().to(DEV)
    axis = np.arange(32) % 3
    pos = [torch.randint(0, 900, (3, l), generator=gen, dtype=torch.int32) for l in total]
    rope = spd.Rope(inv, 3, axis) if turned else None
    empty = [torch.zeros((0, H, d), dtype=dt)] * 3
    room = lambda n: [torch.zeros((l, H, d), dtype=dt) for l in n]  # noqa: E731
    private = ref.Cache(spd, room(prompt), room(prompt), "paged_nhd16", DEV)
    public = ref.Cache(spd, room([4] * 3), room([4] * 3), "nhd", DEV)
    # what the caches hold of a key: turned, and rounded to its type
    turn = lambda t, p: ref.turn(t, p, inv, axis, False)[0].to(dt) if turned else t  # noqa: E731
    done = [0, 0, 0]
    for n_new, view, begin in ((prompt, private.view, None), (later[0], None, private.view), (later[1], None, private.view)):
        if view is None:
            held = [dn - p + n for dn, p, n in zip(done, prompt, n_new)]
            view = spd.KVView(held, H * d, d, k=list(public.k), v=list(public.v))
        step = spd.TokenStep(ctx, dt, Hq, H, d, 0.125, view, n_new, rope, begin, cap=15.0, causal=True)
        rows = [torch.cat([t[u][done[u]:done[u] + n] for u, n in enumerate(n_new)]).to(DEV) for t in x]
        places = torch.cat([pos[u][:, done[u]:done[u] + n] for u, n in enumerate(n_new)], 1).contiguous().to(DEV) if turned else None
        got, lse = step.run(*rows, places)
        torch.cuda.synchronize()
        at = 0
        for u, n in enumerate(n_new):
            end = done[u] + n
            q = turn(x[0][u][done[u]:end], pos[u][:, done[u]:end])
            k = turn(x[1][u][:end], pos[u][:, :end])
            a, want, b, most = ref.attend(q, k, x[2][u][:end], ref.visible(n, end, done[u], 0, True), 0.125, 15.0)
            # q and k may round to the next value where the turned ones lie at a half step: one step of each product, and what the attention itself adds
            step_of = (4 * ref.HALF_STEP[dt] + (d + 4) * 2 ** -24) * most + 15 * 2 ** -21 if turned and dt != torch.float32 else 2 ** -19 * most + 2 ** -15
            assert bool(((got[at:at + n].double().cpu() - a).abs() <= (2 * step_of + 2 ** -12 * (dt == torch.float16) + 2 ** -15) * b + 1e-6).all())
            assert bool(((lse[at:at + n].double().cpu() - want).abs() <= step_of + 2 ** -14).all())
            at += n
            done[u] = end


def test_refusals_reach_no_kernel(ctx):
    """Errors of the checks come back as codes and leave the results alone."""
    import paper_2409_19134_amd as spd
    p = Problem((8, 2, 64), "bf16", "hnd", [1, 2], [30, 40], dict(), "f32", seed=2).store()
    q = p.q.to(DEV)
    out, lse = torch.full((3, 8, 64), 5.0, device=DEV), torch.full((3, 8), 5.0, device=DEV)
    for score, code in ((spd.Score(cap=-1.0), spd.SPD_ERR_SHAPE), (spd.Score(window=-1), spd.SPD_ERR_LEN), (spd.Score(prefix=[-1, 0]), spd.SPD_ERR_LEN),
                        (spd.Score(k_pos=[0, 1 << 30]), spd.SPD_ERR_LEN)):
        with pytest.raises(spd.SpdError) as e:
            ctx.spd_partial_attn_tokens(p.shape, q, p.cache.view, p.new, score, out, lse)
        assert e.value.code == code
    torch.cuda.synchronize()
    assert bool((out == 5.0).all()) and bool((lse == 5.0).all())


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "same"), ("f16", "same")])
@pytest.mark.parametrize("cap", [1e4, 1e6, 1e30])
@pytest.mark.parametrize("new", [[2, 1], [9], [300]])
@pytest.mark.parametrize("slopes", [False, True])
def test_a_cap_far_above_the_scores_changes_nothing(ctx, dtype, out, cap, new, slopes):
    """cap tanh(s / cap) = s (1 - (s / cap)^2 / 3 + ..): of scores below 64, a 24-bit rounding at most, so held to the bounds without a cap."""
    p = Problem((32, 8, 128), dtype, "hnd", new, [700], dict(slopes=slopes), out, seed=23).store()
    want = p.exact()
    assert 64.0 > p.most      # (a sum of magnitudes: the scores are smaller)
    p.score = p.spd.Score(cap=cap, slopes=None if p.slopes is None else p.slopes.float().to(DEV), causal=True, k_pos=p.k_pos)
    p.exact = lambda: want
    p.check(*p.call(ctx))


def test_caps_around_the_short_form(ctx):
    for cap in (0.01, 1.0, 63.0, 64.0, 65.0, 200.0):
        p = Problem((32, 8, 128), "bf16", "hnd", [200], [500], dict(cap=cap), "same", seed=24).store()
        p.check(*p.call(ctx))


def test_a_token_step_follows_its_view(ctx):
    """One TokenStep run again and again while the view's lengths (a host array that the caller owns) move on: the queries' positions over the prompt move with
    them, which a window shows."""
    import paper_2409_19134_amd as spd
    Hq, H, d, dt, prompt, steps, window = 8, 2, 64, torch.float32, [70, 1, 133], 6, 40
    gen = torch.Generator().manual_seed(29)
    q, k, v = ([torch.randn((p + steps, h, d), generator=gen) for p in prompt] for h in (Hq, H, H))
    private = ref.Cache(spd, [x[:p] for x, p in zip(k, prompt)], [x[:p] for x, p in zip(v, prompt)], "nhd", DEV)
    room = [torch.zeros((steps, H, d)) for _ in prompt]
    public = ref.Cache(spd, room, room, "nhd", DEV)
    view = spd.KVView([0] * 3, H * d, d, k=list(public.k), v=list(public.v))
    step = spd.TokenStep(ctx, dt, Hq, H, d, 0.125, view, [1] * 3, prompt=private.view, window=window)
    for i in range(steps):
        view.lens += 1
        rows = [torch.stack([t[u][p + i] for u, p in enumerate(prompt)]).to(DEV) for t in (q, k, v)]
        got, lse = step.run(*rows)
        torch.cuda.synchronize()
        for u, p in enumerate(prompt):
            end = p + i + 1
            a, want, b, most = ref.attend(q[u][end - 1:end], k[u][:end], v[u][:end], ref.visible(1, end, end - 1, 0, True, window), 0.125)
            # (d + 4) roundings of a score, twice for the two partials' weights, and the 24-bit sums
            delta = 2 ** -24 * (2 * (d + 4) * most + 256)
            assert bool(((got[u:u + 1].double().cpu() - a).abs() <= (2 * delta + end * 2 ** -24) * b + 1e-6).all()), i
            assert bool(((lse[u:u + 1].double().cpu() - want).abs() <= delta + end * 2 ** -24 + 8 * 2 ** -24 * want.abs()).all()), i


def test_tensors_elsewhere_are_refused(ctx):
    """Host tensors, whose addresses a kernel must not follow, do not get that far."""
    import paper_2409_19134_amd as spd
    p = Problem((8, 2, 64), "bf16", "hnd", [1, 2], [30, 40], dict(), "f32", seed=2).store()
    q = p.q.to(DEV)
    for args in ((p.q, spd.Score()), (q, spd.Score(slopes=torch.ones(8))), (q, spd.Score(ranges=torch.zeros((3, 2), dtype=torch.int32)))):
        with pytest.raises(AssertionError):
            ctx.spd_partial_attn_tokens(p.shape, args[0], p.cache.view, p.new, args[1])
    for out, lse in ((torch.empty((3, 8, 64)), None), (None, torch.empty((3, 8)))):
        with pytest.raises(AssertionError):
            ctx.spd_partial_attn_tokens(p.shape, q, p.cache.view, p.new, None, out, lse)
    inv, places = torch.ones(32), torch.zeros((1, 3), dtype=torch.int32)
    k = p.cache.view
    new = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    for rope, pos, x in ((spd.Rope(inv), places.to(DEV), q), (spd.Rope(inv.to(DEV)), places, q), (spd.Rope(inv.to(DEV)), places.to(DEV), p.q)):
        with pytest.raises(AssertionError):
            ctx.spd_rotate(rope, x, pos)
        with pytest.raises(AssertionError):
            ctx.spd_append_tokens(p.shape, k, p.new, new.to(DEV), new.to(DEV), rope, pos, x)
    for a, b in ((new, new.to(DEV)), (new.to(DEV), new)):
        with pytest.raises(AssertionError):
            ctx.spd_append_tokens(p.shape, k, p.new, a, b)


@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("f16", "same"), ("f32", "f32")])
@pytest.mark.parametrize("new", [[2, 1, 3, 1], [9, 20, 7, 12], [70, 200, 33, 129]])
@pytest.mark.parametrize("score", [dict(causal=True), dict(causal=False, slopes=True), dict(causal=False, window=60, slopes=True, cap=8.0),
                                   dict(causal=True, window=60, prefix=True, slopes=True)], ids=["causal", "slopes", "window", "prefix"])
def test_queries_before_among_and_after_the_keys(ctx, dtype, out, new, score):
    """Positions of the queries wherever the caller says: before every key of the view, among them, right behind them and far behind."""
    p = Problem((8, 2, 128), dtype, "nhd", new, [300, 150, 1, 420], score, out, elsewhere=True, seed=31)
    p.k_pos = [500, 90, 40, 0]
    p.q_pos = [3, 120, 41, 900]
    if p.prefix is not None:
        p.prefix = [600, 0, 41, 7]
    p.store()
    p.check(*p.call(ctx))


def test_a_thousand_users(ctx):
    """More users than a table's usual room, most with one token, some with none."""
    new = [u % 3 for u in range(1100)]
    p = Problem((4, 4, 64), "bf16", "hnd", new, [u % 7 for u in range(1100)], dict(cap=9.0), "f32", seed=33).store()
    got = p.call(ctx)
    p.check(*got)
    again = p.call(ctx)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_a_token_step_recorded_whole(ctx):
    """Append, attention over both owners' caches and the merge in one graph: replays follow the tokens, their positions and the caches, with eager calls of
    the same context in between."""
    import paper_2409_19134_amd as spd
    Hq, H, d, dt, prompt, new = 8, 2, 128, torch.bfloat16, [400, 3, 90], [4, 1, 30]
    gen = torch.Generator().manual_seed(37)
    rand = lambda l: torch.randn((l, H, d), generator=gen).to(dt)  # noqa: E731
    private = ref.Cache(spd, [rand(l) for l in prompt], [rand(l) for l in prompt], "paged_nhd16", DEV)
    public = ref.Cache(spd, [rand(l + 9) for l in new], [rand(l + 9) for l in new], "hnd", DEV)
    rope = spd.Rope(torch.linspace(1.0, 0.001, 64, device=DEV))
    T = sum(new)
    q, k, v = (torch.randn((T, h, d), device=DEV).to(dt) for h in (Hq, H, H))
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    step = spd.TokenStep(ctx, dt, Hq, H, d, 0.088, public.view, new, rope, private.view, cap=30.0, window=200)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step.run(q, k, v, pos)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            y, lse = step.run(q, k, v, pos)
    for i in range(4):
        for t in (q, k, v):
            t.normal_()
        pos.add_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), lse.clone()
        y.zero_()
        step.run(q, k, v, pos)
        torch.cuda.synchronize()
        assert torch.equal(got[0], y) and torch.equal(got[1], lse) and bool(torch.isfinite(lse).all())
