"""Biases by distance of tokens of a tree whose nearest seen key is far away: their range, or a set without their own bit, leaves nothing near.

The bound is the one of test_gpu_tree.py, row by row and without its allowance for far keys: biases are relative to the nearest key that a row sees, so the arguments of
exponentials that count lie within 64 of the largest however far all of them are (what lies lower has less than e^-64 of the weight), each off by 2^-24 for the slope's
conversion and for the sum.  The distances themselves are exact.  What the log-sum-exp gets back for the nearest key, slope times its distance, is rounded twice
(2^-23 of the result).  A row's sums have as many terms as its range has keys."""
import math

import numpy as np
import pytest
import torch

import token_reference as ref
from test_gpu_tree import Problem, ctx, pack  # noqa: F401

pytestmark = pytest.mark.gpu


class Far(Problem):
    def check(self, out, lse):
        a, want_lse, b, any_key = self.exact()
        terms = torch.from_numpy(np.concatenate([np.clip(np.diff(self.ranges[at:at + n], axis=1)[:, 0], 0, h) for at, n, h in
                                                 zip(np.cumsum([0] + self.new), self.new, self.held)])).double()[:, None]
        eps, rounded = 2.0 ** -24, ref.HALF_STEP[self.out_dt]
        delta = (self.d + 4) * eps * self.most + 256 * eps + self.cap * (4 if self.out_dt == torch.float32 else 8) * eps + 4 * eps * 64
        weights = 2 * delta + terms * eps + {torch.float32: 2 * eps, torch.bfloat16: 2 * eps, torch.float16: 2.0 ** -21}[self.dt]
        if self.out_dt != torch.float32:
            weights = weights + ref.HALF_STEP[self.dt]
        bound = weights[:, :, None] * b * 1.01 + rounded * a.abs() * 1.01 + (2.0 ** -25 if self.out_dt == torch.float16 else 1e-12)
        off = (out.double().cpu() - a).abs()
        assert bool((off <= bound).all()), (float(off.max()), float((off / bound).max()))
        got = lse.double().cpu()
        assert bool((got[~any_key] == -math.inf).all()) and bool((out.cpu()[~any_key] == 0).all())
        assert bool(((got - want_lse).abs() <= delta + terms * eps + 4 * eps * want_lse.abs() + 2 * eps)[any_key].all())

    def ranged(self, lists):
        """A range for every token, of positions from the user's first key on."""
        at = 0
        for u, n in enumerate(self.new):
            self.ranges[at:at + n] = np.array([lists(u, i) for i in range(n)]).reshape(n, 2) + self.k_pos[u]
            at += n
        return self.store()


TYPES = [("f32", "f32"), ("bf16", "f32"), ("f16", "f32"), ("bf16", "same"), ("f16", "same")]
# few rows in tiles of 16 and of 32, more rows in tiles of 64 and of 128
SIZES = [((8, 8, 64), [9, 4]), ((8, 2, 128), [7, 8]), ((8, 2, 64), [12, 16]), ((8, 2, 128), [30, 3]), ((8, 2, 64), [70, 1])]


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("heads,new", SIZES)
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_ranges_far_behind(ctx, heads, new, dtype, out, cap):  # noqa: F811
    """Documents at the front of a long past: short ones, and ones over many stretches; every fourth token sees everything, every seventh nothing."""
    for layout, seed in (("hnd", 31), ("paged_nhd16", 32)):
        p = Far(heads, dtype, layout, new, [20011, 9000], dict(slopes=True, ranges=True, cap=cap), out, seed=seed)
        rng = np.random.default_rng(seed)

        def of(u, i):
            lo, n = int(rng.integers(0, 300)), p.held[u]
            return [0, n + 100] if i % 4 == 3 else [50, 50] if i % 7 == 6 else [lo, lo + int(rng.integers(1, 400))] if i % 2 else [lo, lo + n // 2]

        p.ranged(of)
        p.check(*p.call(ctx))


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("heads,new", SIZES)
def test_sets_without_the_token_itself(ctx, heads, new, dtype, out):  # noqa: F811
    """Chains of drafted tokens, most of which do not see themselves: only the first tokens of the tree, or nothing of it and the front of the past."""
    p = Far(heads, dtype, "nhd", new, [12000, 60], dict(slopes=True, ranges=True), out, seed=33, kind="chain")
    rng = np.random.default_rng(33)
    sets = []
    for u, n in enumerate(new):
        see = rng.random((n, n)) < 0.3
        np.fill_diagonal(see, rng.random(n) < 0.2)
        see[:, n // 2:] &= rng.random((n, n - n // 2)) < 0.2
        see[n - 1] = False
        p.see[u] = see
        sets.append(pack(see, p.sets.shape[1]))
    p.sets = np.concatenate(sets)

    def of(u, i):
        base = p.held[u] - new[u]
        return ([0, 10], [0, base // 3], [base, base + 3], [base, base + new[u]], [0, base + new[u]], [base + 1, base + 1 + i // 2])[(i + u) % 6]

    p.ranged(of)
    p.check(*p.call(ctx))


def test_prefixes_far_behind(ctx):  # noqa: F811
    """A prefix and a short window over sets that leave all of the tree out: the window's keys are the nearest, or the range leaves only the prefix."""
    for new in ([3], [9, 2], [60], [130]):
        for dtype in ("f32", "bf16"):
            p = Far((4, 1, 64), dtype, "paged_hnd16", new, [15000, 700], dict(slopes=True, ranges=True, prefix=True, window=40), "f32", seed=35, kind="sets")
            p.prefix = [100] * len(new)
            for u, n in enumerate(new):
                p.see[u][:] = False
            p.sets = np.concatenate([pack(x, p.sets.shape[1]) for x in p.see])
            p.ranged(lambda u, i: [0, p.held[u] + 50] if i % 3 == 0 else [20, 90 + i] if i % 3 == 1 else [0, p.held[u] - new[u] - 10])
            p.check(*p.call(ctx))
