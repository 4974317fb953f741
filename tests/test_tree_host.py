"""The calls for trees of drafted tokens and for moves within caches without a GPU: what they refuse, what the Python side refuses before the library is
asked, and their tables."""
import ctypes as C
import itertools
import math
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2409_19134_amd as spd
from paper_2409_19134_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
P = 0x10000      # an address that is never followed
_caches = itertools.count(1)      # (no two views of one cache unless a test says so)
S, L, N, A = spd.SPD_ERR_SHAPE, spd.SPD_ERR_LEN, spd.SPD_ERR_NULL, spd.SPD_ERR_ALIGN


def _ints(x):
    return None if x is None else np.array(x, np.int32)


def _at(x):
    return None if x is None else x.ctypes.data


def _plan(n_new=(3, 5), parents=P, first=None, words=1, seen=P, depth=P, positions=None):
    n, f = _ints(n_new), _ints(first)
    return b.lib.spd_validate_tree_plan(len(n_new) if n_new is not None else 2, _at(n), parents, _at(f), words, seen, depth, positions)


def test_refusals_of_the_plan():
    assert _plan() == 0 and _plan(first=[0, 1 << 29], positions=P) == 0 and _plan(n_new=(64, 0)) == 0 and _plan(n_new=(1024,), words=16) == 0
    assert _plan(n_new=(65, 0)) == L and _plan(n_new=(-1, 3)) == L and _plan(n_new=(1025,), words=16) == L
    assert _plan(words=0) == S and _plan(words=17) == S and _plan(words=-1) == S
    assert _plan(n_new=None) == N and _plan(parents=None) == N and _plan(seen=None) == N and _plan(depth=None) == N
    assert _plan(first=[0, 0]) == N and _plan(positions=P) == N      # both or neither
    assert _plan(first=[-1, 0], positions=P) == L and _plan(first=[1 << 30, 0], positions=P) == L
    assert _plan(seen=P + 4) == A and _plan(parents=P + 2) == A and _plan(depth=P + 1) == A and _plan(first=[0, 0], positions=P + 2) == A
    assert _plan(n_new=(0, 0), parents=None, seen=None, depth=None) == 0 and _plan(n_new=()) == 0
    assert b.lib.spd_validate_tree_plan(-1, None, P, None, 1, P, P, None) == L
    n = _ints([1])
    assert b.lib.spd_tree_plan(None, 1, n.ctypes.data, P, None, 1, P, P, None, None) == N


def _shape(**kw):
    s = dict(dtype=spd.SPD_BF16, n_q_heads=8, n_kv_heads=2, head_dim=64, scale=0.125)
    s.update(kw)
    return spd.spd_shape(*s.values())


class View:
    """A view whose addresses are never followed."""

    def __init__(self, lens=(20, 30), page=0, **kw):
        self.lens = np.array(lens, np.int32)
        k, v = self.caches = [next(_caches) * P for _ in "kv"]
        self.ptrs = [(C.c_void_p * max(1, len(lens)))(*[x] * max(1, len(lens))) for x in (k, v)]
        st = spd.spd_kv_view()
        st.n_users, st.lens = len(lens), self.lens.ctypes.data_as(C.POINTER(C.c_int32))
        st.token_stride, st.head_stride = 64, 64 * 64
        if page:
            st.k_pool, st.v_pool, st.block_table = k, v, P
            st.block_size, st.max_blocks, st.block_stride = page, 100, 2 * 64 * page
        else:
            st.k_ptrs, st.v_ptrs = (C.cast(x, C.POINTER(C.c_void_p)) for x in self.ptrs)
        for k, v in kw.items():
            setattr(st, k, v)
        self.struct = st


def _tree(shape=None, view=None, n_new=(1, 2), tree=(1, P, P), score=None, q=P, q_stride=512, out=P, lse=P, out_dtype=0):
    view, n = view or View(), _ints(n_new)
    t = None if tree is None else C.byref(b.spd_tree(*tree))
    return b.lib.spd_validate_tree(C.byref(shape or _shape()), q, q_stride, C.byref(view.struct), n.ctypes.data, t,
                                   None if score is None else C.byref(score.struct), out, out_dtype, lse)


def test_refusals_of_the_trees_attention():
    assert _tree() == 0 and _tree(score=spd.Score(q_pos=[40, 50], window=3)) == 0 and _tree(tree=(16, P, P)) == 0
    assert _tree(tree=None) == N and _tree(tree=(1, None, P)) == N and _tree(tree=(1, P, None)) == N
    assert _tree(tree=(0, P, P)) == S and _tree(tree=(17, P, P)) == S
    assert _tree(tree=(1, P + 4, P)) == A and _tree(tree=(1, P, P + 2)) == A
    assert _tree(view=View(lens=(100, 30)), n_new=(65, 1)) == L and _tree(view=View(lens=(100, 30)), n_new=(65, 1), tree=(2, P, P)) == 0
    assert _tree(n_new=(21, 1)) == L and _tree(n_new=(21, 1), score=spd.Score(q_pos=[0, 0])) == 0
    assert _tree(n_new=(0, 0), tree=(1, None, None), q=None, out=None, lse=None) == 0
    # what the call without a tree refuses
    assert _tree(shape=_shape(head_dim=96)) == S and _tree(out_dtype=spd.SPD_F16) == S and _tree(q_stride=500) == A and _tree(lse=None) == N
    assert _tree(score=spd.Score(cap=math.inf)) == S and _tree(score=spd.Score(window=-1)) == L
    n, v, s, t = _ints([1, 1]), View(), _shape(), b.spd_tree(1, P, P)
    assert b.lib.spd_partial_attn_tree(None, C.byref(s), P, 512, C.byref(v.struct), n.ctypes.data, C.byref(t), None, P, 0, P, None) == N


def _keep(views=None, n_last=(3, 5), keep=P, n_keep=P, shape=None):
    views, n = [View()] if views is None else views, _ints(n_last)
    return b.lib.spd_validate_keep(C.byref(shape or _shape()), b._view_array(views), len(views), _at(n), keep, n_keep)


def test_refusals_of_kept_tokens():
    assert _keep() == 0 and _keep([View(), View()]) == 0 and _keep([View(page=16), View(page=16)]) == 0 and _keep([]) == 0
    assert _keep(n_last=(21, 0)) == L and _keep(n_last=(-1, 0)) == L and _keep(n_last=(20, 30)) == 0
    assert _keep(keep=None) == N and _keep(n_keep=None) == N and _keep(n_last=None) == N and _keep(keep=P + 2) == A and _keep(n_keep=P + 1) == A
    assert _keep(n_last=(0, 0), keep=None, n_keep=None) == 0
    # views that are not alike
    assert _keep([View(), View(lens=(20, 29))]) == S and _keep([View(), View(lens=(20, 30, 1))]) == S and _keep([View(), View(page=16)]) == S
    assert _keep([View(), View(token_stride=72)]) == S and _keep([View(), View(head_stride=128)]) == S and _keep([View(page=16), View(page=32)]) == S
    assert _keep([View(page=16), View(page=16, block_stride=4096)]) == S
    with_dev, more = View(k_ptrs_dev=P, v_ptrs_dev=2 * P), View(k_ptrs_dev=3 * P, v_ptrs_dev=4 * P)
    assert _keep([with_dev, more]) == 0 and _keep([View(), with_dev]) == S
    # a cache twice
    view, paged = View(), View(page=16)
    assert _keep([with_dev, more, with_dev]) == S and _keep([View(k_ptrs_dev=P, v_ptrs_dev=P)]) == S
    assert _keep([view, View(), view]) == S and _keep([View(k_ptrs=view.struct.v_ptrs), view]) == S and _keep([view, view], n_last=(0, 0)) == 0
    assert _keep([paged, paged]) == S and _keep([View(page=16, v_pool=paged.caches[0]), paged]) == S and _keep([paged, View(page=16, k_pool=paged.caches[0])]) == S
    assert _keep([paged, View(page=16, k_pool=paged.caches[0], v_pool=paged.caches[1], block_table=2 * P)]) == 0
    assert _keep([View(page=16) for _ in range(1024)]) == 0 and _keep([paged] + [View(page=16) for _ in range(1022)] + [paged]) == S
    a, c = (np.array(x, np.int64) for x in ([64, 128], [64, 64]))
    strided = [View(head_strides=x.ctypes.data_as(C.POINTER(C.c_int64))) for x in (a, a, c)]
    assert _keep(strided[:2]) == 0 and _keep(strided) == S and _keep([strided[0], View()]) == S
    assert _keep([View(token_stride=60)]) == A and _keep([View(page=24)]) == S and _keep(shape=_shape(dtype=9)) == S
    assert _keep([View(page=16, max_blocks=1)]) == L and _keep([View(page=16, block_table=None)]) == N
    assert b.lib.spd_validate_keep(C.byref(_shape()), None, 1, None, P, P) == N and b.lib.spd_validate_keep(C.byref(_shape()), None, 1025, None, P, P) == L
    assert b.lib.spd_keep_tokens(None, C.byref(_shape()), b._view_array([View()]), 1, _ints([1, 1]).ctypes.data, P, P, None) == N


def _pages(views=None, n_pages=10, n_pairs=3, pairs=P, n_tokens=None, shape=None):
    views = [View((), page=16)] if views is None else views
    return b.lib.spd_validate_pages(C.byref(shape or _shape()), b._view_array(views), len(views), n_pages, n_pairs, pairs, n_tokens)


def test_refusals_of_copied_pages():
    assert _pages() == 0 and _pages(n_tokens=P) == 0 and _pages([View((), page=16, block_table=None)] * 3) == 0 and _pages([]) == 0
    assert _pages(n_pages=-1) == L and _pages(n_pairs=-1) == L and _pages(n_pairs=0, pairs=None) == 0 and _pages(n_pages=0, pairs=None) == 0
    assert _pages(pairs=None) == N and _pages(pairs=P + 4) == A and _pages(n_tokens=P + 2) == A
    assert _pages([View(())]) == S and _pages([View((), page=48)]) == S
    assert _pages([View((), page=16), View((), page=32)]) == S and _pages([View((), page=16), View((), page=16, block_stride=4096)]) == S
    assert _pages([View((), page=16, k_pool=None)]) == N and _pages([View((), page=16, v_pool=P + 8)]) == A
    assert _pages([View((), page=16, token_stride=60)]) == A and _pages([View((), page=16, block_stride=0)]) == A and _pages([View((), page=16, head_stride=4)]) == A
    assert _pages(shape=_shape(head_dim=32)) == S
    assert b.lib.spd_copy_pages(None, C.byref(_shape()), b._view_array([View((), page=16)]), 1, 1, 1, P, None, None) == N


class Elsewhere:
    """A tensor's place in memory and nothing else of it."""

    def __init__(self, like, device):
        self.like, self.device_index = like, device

    def get_device(self):
        return self.device_index

    def __getattr__(self, name):
        return getattr(self.like, name)


class _Stream:
    cuda_stream = 0


def _context():
    """A context's checks without a device behind it.  (The library itself answers SPD_ERR_NULL: what is not refused gets there.)"""
    ctx = spd.Context.__new__(spd.Context)
    ctx.device, ctx.handle = 0, None
    return ctx


def _here(t, device=0):
    return Elsewhere(t, device)


def test_what_python_refuses():
    ctx, shape = _context(), spd.make_shape(torch.float32, 4, 2, 64, 0.125)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    k = [_here(torch.zeros((2, 30, 64))) for _ in range(2)]
    view = spd.KVView([30, 20], 64, 30 * 64, k=k, v=k)
    pool = _here(torch.zeros((4, 2, 16, 64)))
    paged = spd.KVView([30, 20], 64, 16 * 64, k_pool=pool, v_pool=pool, block_table=_here(ints(2, 2)), block_size=16, block_stride=2 * 16 * 64)
    assert paged.n_pages == 4
    away = spd.KVView([30, 20], 64, 30 * 64, k=[_here(t.like, 1) for t in k], v=k)
    keep, count = _here(ints(5)), _here(ints(2))

    def refused(error, call, *args, **kw):
        with pytest.raises(error):
            call(*args, stream=_Stream, **kw)

    refused(spd.SpdError, ctx.spd_keep_tokens, shape, [view], [2, 3], keep, count)
    refused(AssertionError, ctx.spd_keep_tokens, shape, [view, away], [2, 3], keep, count)
    refused(AssertionError, ctx.spd_keep_tokens, shape, [view], [2, 3], _here(ints(4)), count)
    refused(AssertionError, ctx.spd_keep_tokens, shape, [view], [2, 3], keep, _here(ints(3)))
    refused(AssertionError, ctx.spd_keep_tokens, shape, [view], [2, 3], _here(ints(5), 1), count)
    refused(AssertionError, ctx.spd_keep_tokens, shape, [view], [2, 3], _here(torch.zeros(5, dtype=torch.int64)), count)
    refused(spd.SpdError, ctx.spd_copy_pages, shape, [paged], _here(ints(3, 2)))
    refused(spd.SpdError, ctx.spd_copy_pages, shape, [paged], _here(ints(3, 2)), _here(ints(3)))
    refused(AssertionError, ctx.spd_copy_pages, shape, [view], _here(ints(3, 2)))
    refused(AssertionError, ctx.spd_copy_pages, shape, [paged], _here(ints(3, 2), 1))
    refused(AssertionError, ctx.spd_copy_pages, shape, [paged], _here(ints(3, 3)))
    refused(AssertionError, ctx.spd_copy_pages, shape, [paged], _here(ints(3, 2)), _here(ints(2)))
    assert ctx.spd_copy_pages(shape, [], ints(3, 2)) is None and ctx.spd_keep_tokens(shape, [], [], ints(0), ints(0)) is None

    def tree(T=3, words=1, device=0):
        t = spd.Tree(T, words, device="cpu")
        for name in ("seen", "depth", "positions"):
            setattr(t, name, _here(getattr(t, name), device))
        return t

    refused(spd.SpdError, ctx.spd_tree_plan, _here(ints(3)), [1, 2], tree=tree())
    refused(spd.SpdError, ctx.spd_tree_plan, _here(ints(3)), [1, 2], first=[4, 5], tree=tree())
    refused(AssertionError, ctx.spd_tree_plan, _here(ints(4)), [1, 2], tree=tree())
    refused(AssertionError, ctx.spd_tree_plan, _here(ints(3)), [1, 2], tree=tree(4))
    refused(AssertionError, ctx.spd_tree_plan, _here(ints(3)), [1, 2], first=[4], tree=tree())
    refused(AssertionError, ctx.spd_tree_plan, _here(ints(3)), [1, 2], tree=tree(device=1))
    refused(AssertionError, ctx.spd_tree_plan, _here(ints(3), 1), [1, 2], tree=tree())
    refused(AssertionError, ctx.spd_tree_plan, _here(ints(3)), [1, 2], words=2, tree=tree())
    q, out, lse = (_here(torch.zeros(x)) for x in ((3, 4, 64), (3, 4, 64), (3, 4)))
    refused(spd.SpdError, ctx.spd_partial_attn_tree, shape, q, view, [1, 2], tree(), None, out, lse)
    refused(AssertionError, ctx.spd_partial_attn_tree, shape, q, view, [1, 2], tree(2), None, out, lse)
    refused(AssertionError, ctx.spd_partial_attn_tree, shape, q, view, [1, 2], tree(device=1), None, out, lse)
    refused(AssertionError, ctx.spd_partial_attn_tree, shape, q, view, [1, 2], None, None, out, lse)
    refused(AssertionError, ctx.spd_partial_attn_tree, shape, q, away, [1, 2], tree(), None, out, lse)
    for bad in (dict(seen=torch.zeros((3, 1))), dict(depth=ints(2)), dict(positions=ints(4))):
        parts = dict(seen=torch.zeros((3, 1), dtype=torch.int64), depth=ints(3), positions=None) | bad
        with pytest.raises(AssertionError):
            spd.Tree.of(**parts)


def test_tables_under_asan_ubsan(tmp_path):
    """tests/host/tree_schedule_fuzz.cpp: every tile's keys in its stretches once, in order, and the masks key by key."""
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    exe = str(tmp_path / "tree_schedule_fuzz")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-x", "hip", "-Xarch_host", "-fsanitize=address,undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-o", exe, os.path.join(ROOT, "tests", "host", "tree_schedule_fuzz.cpp")]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("ok"), run.stdout[-3000:]
