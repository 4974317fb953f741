"""spd_tree_plan and spd_partial_attn_tree against their definitions in 64 bits.

Tolerance of the attention, per element, from the inputs, as for the calls without a tree: a score's product of d terms rounds d times to 24 bits (off by at
most d 2^-24 sum |q_c k_c|), its factor, cap (tanh off by 2^-23 of 1, in the kernel for 16-bit results 2^-22) and bias once each, the exponential's argument and
value by 2^-23 of what they are (arguments up to 64): together `delta`.  Biases are taken relative to the query's own place: arguments lie up to slope times the
nearest seen key's distance lower, off by 2^-23 of that.  A row of L keys then has weights off by 2 delta relative to each other and sums of L
terms (L 2^-24).  Probabilities enter the second product in 24 (bf16), 22 (fp16) or 24 bits; for 16-bit results rounded once (half a step of sum p |v|).  The result is
rounded to its type."""
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


def branches(parents):
    """One user's branches [n, n] (bool) and depths, from parent to parent."""
    n = len(parents)
    see, depth = np.zeros((n, n), bool), np.zeros(n, np.int64)
    for i in range(n):
        j = i
        while True:
            see[i, j] = True
            p = parents[j]
            if not 0 <= p < j:
                break
            j = p
        depth[i] = see[i].sum() - 1
    return see, depth


def pack(see, words):
    """[n, n] bool -> int64 [n, words]."""
    n = see.shape[0]
    bits = np.zeros((n, 64 * words), bool)
    bits[:, :see.shape[1]] = see
    return np.packbits(bits, axis=1, bitorder="little").view(np.int64).reshape(n, words)


def random_parents(rng, n, kind):
    i = np.arange(n)
    if kind == "chain":
        return i - 1
    if kind == "roots":
        return np.full(n, -1)
    return np.array([rng.integers(max(-1, j // 3 - 2), j) if rng.random() < 0.8 else j - 1 for j in range(n)], np.int64)


@pytest.mark.parametrize("new,words", [([1], 1), ([13], 1), ([64, 0, 1, 33], 1), ([5, 64, 2], 3), ([65], 2), ([0, 130, 64, 1, 512], 8), ([1024, 3], 16),
                                       ([7] * 300, 1), ([70] * 150, 2)])
@pytest.mark.parametrize("kind", ["tree", "chain", "roots"])
def test_plan(ctx, new, words, kind):
    rng = np.random.default_rng(len(new) + words)
    lists = [random_parents(rng, n, kind) for n in new]
    first = rng.integers(0, 1 << 29, len(new)).astype(np.int32)
    parents = torch.from_numpy(np.concatenate(lists).astype(np.int32)).to(DEV)
    T = sum(new)
    import paper_2409_19134_amd as spd
    room = spd.Tree(T + 2, words)
    for t in (room.seen, room.depth, room.positions):
        t.fill_(-7)
    tree = spd.Tree.of(room.seen[:T], room.depth[:T], room.positions[:T])
    assert ctx.spd_tree_plan(parents, new, first=first, tree=tree) is tree
    torch.cuda.synchronize()
    for t in (room.seen, room.depth, room.positions):
        assert bool((t[T:] == -7).all())
    seen, depth, positions, at = tree.seen.cpu().numpy(), tree.depth.cpu().numpy(), tree.positions.cpu().numpy(), 0
    for u, n in enumerate(new):
        see, d = branches(lists[u])
        assert np.array_equal(seen[at:at + n], pack(see, words))
        assert np.array_equal(depth[at:at + n], d) and np.array_equal(positions[at:at + n], first[u] + d)
        at += n


def test_plan_of_parents_that_are_none(ctx):
    """Later tokens, the token itself, far numbers: a token without a parent."""
    for n in (40, 100):
        bad = [i if i % 3 == 0 else i + 5 if i % 3 == 1 else (1 << 31) - 1 if i % 2 else -(1 << 31) for i in range(n)]
        bad[n - 1] = n - 2
        tree = ctx.spd_tree_plan(torch.tensor(bad, dtype=torch.int32, device=DEV), [n])
        see, d = branches(bad)
        assert np.array_equal(tree.seen.cpu().numpy(), pack(see, tree.seen.shape[1])) and np.array_equal(tree.depth.cpu().numpy(), d)
        assert d[n - 1] == 1 and d[:n - 1].max() == 0


HEADS = [(8, 8, 64), (32, 8, 128), (14, 2, 64), (16, 1, 128), (5, 5, 64), (24, 3, 128)]
LAYOUTS = ["hnd", "nhd", "exact", "tables", "paged_hnd16", "paged_nhd16", "paged_hnd64", "paged_nhd256"]
NEW = [[1], [5, 1, 2], [8, 0, 5], [3, 1, 16, 2], [33, 1, 0, 4], [130], [64, 63, 65], [26] * 5]
PAST = [[0], [1, 31, 32, 33], [700, 5, 0, 90], [15, 16, 17, 64, 63], [2500]]
SCORES = [dict(causal=False), dict(), dict(cap=5.0), dict(slopes=True), dict(window=1), dict(window=3), dict(window=37), dict(prefix=True), dict(ranges=True),
          dict(prefix=True, window=20), dict(window=50, causal=False), dict(cap=30.0, slopes=True, window=300, prefix=True, ranges=True),
          dict(slopes=True, causal=False, ranges=True), dict(cap=50.0, slopes=True, window=2)]


class Problem:
    """One call: caches, queries, trees, the score's parts, and the result in 64 bits."""

    def __init__(self, heads, dtype, layout, new, past, score, out, elsewhere=False, seed=1, kind="tree", q_scale=2.0, fill=float("nan"), words=None):
        import paper_2409_19134_amd as spd
        self.spd, (self.Hq, self.H, self.d) = spd, heads
        self.dt = ref.DTYPES[dtype]
        self.out_dt = torch.float32 if out == "f32" else self.dt
        gen, rng, U = torch.Generator().manual_seed(seed), np.random.default_rng(seed), len(new)
        self.new, self.T = new, sum(new)
        past = [past[u % len(past)] for u in range(U)]
        self.held = [p if elsewhere else p + n for p, n in zip(past, new)]
        self.k, self.v = ([torch.randn((l, self.H, self.d), generator=gen).to(self.dt) for l in self.held] for _ in range(2))
        self.q = (q_scale * torch.randn((self.T, self.Hq, self.d), generator=gen)).to(self.dt)
        self.scale = 1 / math.sqrt(self.d)
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
                parts.append(np.stack([lo, lo + rng.integers(-3, 60 + self.held[u], n)], 1))
            self.ranges = np.concatenate(parts).astype(np.int32).reshape(-1, 2)
        words = words or max(1, -(-max(new) // 64)) + seed % 2
        sets, depths, self.see, self.depth = [], [], [], []
        for n in new:
            if kind == "sets":      # any sets at all, with depths that no tree of so many tokens has
                see, depth = rng.random((n, n)) < 0.4, rng.integers(-3, n + 4, n)
                see[n // 2:n // 2 + 1] = False
            else:
                see, depth = branches(random_parents(rng, n, kind))
            self.see.append(see)
            self.depth.append(np.clip(depth, 0, max(0, n - 1)))
            bits = np.concatenate([see, rng.random((n, 64 * words - n)) < 0.5], 1)      # (what lies behind the last token means nothing)
            sets.append(pack(bits, words))
            depths.append(depth)
        self.sets, self.depths = np.concatenate(sets), np.concatenate(depths).astype(np.int32)
        self.elsewhere, self.layout, self.fill, self.seed = elsewhere, layout, fill, seed
        self.shape = spd.make_shape(self.dt, *heads, self.scale)

    def store(self):
        self.cache = ref.Cache(self.spd, self.k, self.v, self.layout, DEV, seed=self.seed, fill=self.fill)
        self.score = self.spd.Score(cap=self.cap, slopes=None if self.slopes is None else self.slopes.float().to(DEV), causal=self.causal,
                                    window=self.window, prefix=self.prefix, ranges=None if self.ranges is None else torch.from_numpy(self.ranges).to(DEV),
                                    q_pos=self.q_pos if self.elsewhere else None, k_pos=self.k_pos if any(self.k_pos) else None)
        self.tree = self.spd.Tree.of(torch.from_numpy(self.sets).to(DEV), torch.from_numpy(self.depths).to(DEV))
        return self

    def call(self, ctx, stream=None):
        T, Hq, d = self.T, self.Hq, self.d
        out = torch.full((T + 3, Hq, d), 7.0, dtype=self.out_dt, device=DEV)
        lse = torch.full((T + 3, Hq), 7.0, device=DEV)
        wide = torch.full((T, Hq + 3, d), float("nan"), dtype=self.dt, device=DEV)      # the queries as a slice of wider rows
        wide[:, 1:1 + Hq] = self.q.to(DEV)
        ctx.spd_partial_attn_tree(self.shape, wide[:, 1:1 + Hq], self.cache.view, self.new, self.tree, self.score, out[:T], lse[:T], stream=stream)
        torch.cuda.synchronize()
        assert bool((out[T:] == 7.0).all()) and bool((lse[T:] == 7.0).all())
        return out[:T].clone(), lse[:T].clone()

    def exact(self):
        at, parts, self.most, self.away = 0, [], 0.0, 0.0
        for u, n in enumerate(self.new):
            l, base = self.held[u], self.held[u] - (0 if self.elsewhere else n)
            q = (self.q_pos[u] + self.depth[u])[:, None]
            pos = np.concatenate([self.k_pos[u] + np.arange(base), self.q_pos[u] + self.depth[u] if not self.elsewhere else np.zeros(0, np.int64)])[None]
            see = np.ones((n, l), bool)
            if self.causal:
                see[:, :base] &= pos[:, :base] <= q
            if not self.elsewhere:
                see[:, base:] = self.see[u]
            if self.window:
                see &= np.abs(q - pos) < self.window
            if self.prefix is not None:
                see[:, :base] |= pos[:, :base] < self.prefix[u]
            if self.ranges is not None:
                r = self.ranges[at:at + n]
                see &= (pos >= r[:, :1]) & (pos < r[:, 1:])
            apart = torch.from_numpy(np.abs(q - pos)).double()
            if self.slopes is not None and see.any():
                nearest = np.where(see, np.abs(q - pos), 1 << 40).min(1)
                self.away = max(self.away, float(self.slopes.max()) * float(nearest[see.any(1)].max()))
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
            delta += 4 * eps * (64 + self.away)
        weights = 2 * delta + L * eps + {torch.float32: 2 * eps, torch.bfloat16: 2 * eps, torch.float16: 2.0 ** -21}[self.dt]
        if self.out_dt != torch.float32:
            weights += ref.HALF_STEP[self.dt]
        bound = weights * b * 1.01 + ref.HALF_STEP[self.out_dt] * a.abs() * 1.01 + (2.0 ** -25 if self.out_dt == torch.float16 else 1e-12)
        off = (out.double().cpu() - a).abs()
        assert bool((off <= bound).all()), (float(off.max()), float((off - bound).max()))
        got = lse.double().cpu()
        assert bool((got[~any_key] == -np.inf).all()) and bool((out.cpu()[~any_key] == 0).all())
        g, w = got[any_key], want_lse[any_key]
        assert bool(((g - w).abs() <= delta + L * eps + 4 * eps * w.abs() + 2 * eps).all()), float((g - w).abs().max())


def _cases():
    """Every score with every list of new tokens, the other choices dealt out."""
    rng = np.random.default_rng(12)
    out = []
    for i in range(len(SCORES)):
        for j in range(len(NEW)):
            pick = lambda x: x[int(rng.integers(len(x)))]  # noqa: E731
            out.append((i, j, pick(HEADS), pick(["f32", "bf16", "f16"]), pick(LAYOUTS), pick(PAST), pick(["f32", "same"]), pick([False, False, False, True]),
                        pick(["tree", "tree", "sets", "chain"])))
    return out


@pytest.mark.parametrize("case", _cases(), ids=lambda c: f"{c[0]}-{c[1]}-{'x'.join(map(str, c[2]))}-{c[3]}-{c[4]}-{c[5][0]}-{c[6]}-{int(c[7])}-{c[8]}")
def test_attention_of_trees(ctx, case):
    i, j, heads, dtype, layout, past, out, elsewhere, kind = case
    p = Problem(heads, dtype, layout, NEW[j], past, SCORES[i], out, elsewhere, seed=200 + 13 * i + j, kind=kind).store()
    p.check(*p.call(ctx))


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "same"), ("f16", "f32"), ("f16", "same")])
@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 8, 64)])
@pytest.mark.parametrize("new", [[4], [8, 5], [16, 12], [300]])
def test_every_kernel_and_type(ctx, heads, dtype, out, new):
    for k, score in enumerate((dict(), dict(cap=20.0), dict(cap=20.0, slopes=True))):
        for layout in ("hnd", "paged_nhd16"):
            p = Problem(heads, dtype, layout, new, [401, 77], score, out, seed=40 + k).store()
            p.check(*p.call(ctx))


def test_the_largest_tree(ctx):
    p = Problem((4, 2, 64), "bf16", "paged_hnd16", [1024, 1000], [37, 500], dict(window=200, slopes=True), "f32", seed=5, words=16).store()
    p.check(*p.call(ctx))


@pytest.mark.parametrize("new", [[6], [40]])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_a_chain_is_the_call_without_a_tree(ctx, dtype, new):
    p = Problem((32, 8, 128), dtype, "paged_nhd16", new, [900], dict(cap=20.0, window=100), "f32", seed=4, kind="chain").store()
    p.check(*p.call(ctx))
    p.check(*ctx.spd_partial_attn_tokens(p.shape, p.q.to(DEV), p.cache.view, p.new, p.score))


@pytest.mark.parametrize("new", [[5, 2], [14], [50]])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_what_a_branch_does_not_see_does_not_reach_it(ctx, dtype, new):
    """Infinities and NaN in drafted tokens: in the results of the tokens that see them and in no others'."""
    for layout in ("hnd", "paged_nhd16"):
        p = Problem((8, 2, 64), dtype, layout, new, [70, 5], dict(), "f32", seed=6, kind="tree").store()
        clean, clean_lse = p.call(ctx)
        u, n = 0, new[0]
        bad = n // 2
        row = torch.zeros((1, p.H, p.d), dtype=p.dt)
        row[0, 0, 3], row[0, 0, 9], row[0, 1, 0] = float("inf"), float("nan"), float("-inf")
        p.cache.put(u, p.held[u] - n + bad, torch.full((1, p.H, p.d), 0.5, dtype=p.dt), row)
        p.k[u][p.held[u] - n + bad], p.v[u][p.held[u] - n + bad] = 0.5, 0.0
        out, lse = p.call(ctx)
        sees = torch.zeros(p.T, dtype=torch.bool)
        sees[:n] = torch.from_numpy(p.see[0][:, bad].copy())
        assert bool(sees.any()) and not bool(sees.all())
        assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse[~sees], clean_lse[~sees])
        hit = torch.zeros((p.Hq, p.d), dtype=torch.bool)
        hit[:4, 3] = hit[:4, 9] = hit[4:, 0] = True
        assert bool((~torch.isfinite(out[sees])[:, hit]).all()) and bool(torch.isfinite(out[sees][:, ~hit]).all())


def test_graphs_streams_and_growing_lengths(ctx):
    """Recorded after one eager call, replayed with other trees and queries in the same memory; a loop whose lengths and tree move on."""
    import paper_2409_19134_amd as spd
    for new in ([5, 8], [40, 12]):
        p = Problem((32, 8, 128), "bf16", "paged_nhd16", new, [300, 77], dict(), "f32", seed=8).store()
        want, want_lse = p.call(ctx)
        q = p.q.to(DEV)
        parents = torch.full((p.T,), -1, dtype=torch.int32, device=DEV)
        out, lse = torch.empty_like(want), torch.empty_like(want_lse)
        tree = spd.Tree(p.T, 1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            ctx.spd_tree_plan(parents, new, tree=tree)
            ctx.spd_partial_attn_tree(p.shape, q, p.cache.view, new, tree, p.score, out, lse)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ctx.spd_tree_plan(parents, new, tree=tree)
            ctx.spd_partial_attn_tree(p.shape, q, p.cache.view, new, tree, p.score, out, lse)
        for seed in range(3):
            r = Problem((32, 8, 128), "bf16", "paged_nhd16", new, [300, 77], dict(), "f32", seed=20 + 2 * seed)
            rng = np.random.default_rng(seed)
            lists = [random_parents(rng, n, "tree") for n in new]
            parents.copy_(torch.from_numpy(np.concatenate(lists).astype(np.int32)))
            q.copy_(r.q)
            graph.replay()
            torch.cuda.synchronize()
            p.q = r.q
            p.see, p.depth = zip(*[branches(x) for x in lists])
            p.check(out.clone(), lse.clone())
            other, other_lse = ctx.spd_partial_attn_tree(p.shape, q, p.cache.view, new, tree, p.score)
            assert torch.equal(other, out) and torch.equal(other_lse, lse)
    # lengths that move on, by as much for all users and by themselves
    p = Problem((32, 8, 128), "f16", "nhd", [7, 4], [200, 90], dict(window=64), "f32", seed=10)
    full = [(torch.randn((400, 8, 128)).half(), torch.randn((400, 8, 128)).half()) for _ in range(2)]
    store = [[t[i].to(DEV).contiguous() for t in full] for i in range(2)]
    for step in ([0, 0], [3, 3], [9, 9], [14, 10], [15, 40], [60, 85]):
        held = [207 + step[0], 94 + step[1]]
        p.held, p.k, p.v = held, [full[u][0][:held[u]] for u in range(2)], [full[u][1][:held[u]] for u in range(2)]
        p.k_pos, p.q_pos = [0, 0], [h - n for h, n in zip(held, p.new)]
        view = spd.KVView(held, 8 * 128, 128, k=store[0], v=store[1])
        tree = spd.Tree.of(torch.from_numpy(p.sets).to(DEV), torch.from_numpy(p.depths).to(DEV))
        out, lse = ctx.spd_partial_attn_tree(p.shape, p.q.to(DEV), view, p.new, tree, spd.Score(window=64))
        p.check(out, lse)


def test_another_stream(ctx):
    """All of it on a stream of its own, behind work of that stream that it has to wait for."""
    p = Problem((8, 2, 64), "bf16", "paged_hnd16", [9, 14], [200, 3], dict(slopes=True), "f32", seed=12).store()
    side = torch.cuda.Stream()
    q, out, lse = p.q.to(DEV), torch.empty((p.T, 8, 64), device=DEV), torch.empty((p.T, 8), device=DEV)
    parents = [random_parents(np.random.default_rng(3), n, "tree") for n in p.new]
    given = torch.from_numpy(np.concatenate(parents).astype(np.int32)).to(DEV)
    late = torch.empty_like(given)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late.copy_(given)
        tree = ctx.spd_tree_plan(late, p.new)
        ctx.spd_partial_attn_tree(p.shape, q, p.cache.view, p.new, tree, p.score, out, lse)
    side.synchronize()
    p.see, p.depth = zip(*[branches(x) for x in parents])
    p.check(out, lse)


def test_rows_that_see_nothing(ctx):
    """Empty sets over an empty past, and windows of one key without the token's own bit: zeros and -inf; the others as ever."""
    for new in ([3, 5], [60]):
        p = Problem((4, 1, 64), "f16", "nhd", new, [0], dict(window=1), "f32", seed=14, kind="sets")
        for u, n in enumerate(new):
            p.see[u][:] = np.eye(n, dtype=bool)
            p.see[u][::2] = False
        p.sets = np.concatenate([pack(x, p.sets.shape[1]) for x in p.see])
        out, lse = p.store().call(ctx)
        p.check(out, lse)
        assert bool(torch.isinf(lse).any()) and bool(torch.isfinite(lse).any())
