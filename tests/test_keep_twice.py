"""Caches that are given to spd_keep_tokens twice are refused, whichever user's they are and however they are handed over.  (Host only: what the library says before
it launches anything.)"""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2409_19134_amd as spd
from paper_2409_19134_amd import binding as b
from test_tree_host import P, S, View, _keep

H, D, ROOM = 2, 64, 40


def _layers(n, users):
    """K and V of n layers, a buffer for every user."""
    return [[[torch.zeros((H, ROOM, D), dtype=torch.bfloat16) for _ in range(users)] for _ in range(2)] for _ in range(n)]


def _views(layers, lens, dev=False):
    return [spd.KVView(lens, D, ROOM * D, k=k, v=v, device_pointer_tables=dev) for k, v in layers]


def _answer(views, n_last):
    shape, n = spd.make_shape(torch.bfloat16, H, H, D, 1.0), np.array(n_last, np.int32)
    return b.lib.spd_validate_keep(C.byref(shape), b._view_array(views), len(views), n.ctypes.data, P, P)


@pytest.mark.parametrize("dev", [False, True])
@pytest.mark.parametrize("layers,users", [(1, 1), (1, 4), (2, 3), (5, 2), (33, 70), (1024, 2)])
def test_one_buffer_twice(dev, layers, users):
    rng = np.random.default_rng(layers + users)
    lens, n_last = [30] * users, [int(x) for x in rng.integers(1, 31, users)]
    if users > 2:
        n_last[1] = 0
    stores = _layers(1, users) * layers if layers > 100 else _layers(layers, users)
    if layers > 100:      # (addresses are all that is looked at)
        one = torch.zeros((2 * layers * users, H, ROOM, D), dtype=torch.bfloat16)
        stores = [[[one[(2 * i + kv) * users + u] for u in range(users)] for kv in range(2)] for i in range(layers)]
    assert _answer(_views(stores, lens, dev), n_last) == 0
    for u in {0, users - 1, users // 2}:
        for i, kv, j, other in ((0, 0, 0, 1), (0, 1, layers - 1, 0), (0, 0, layers - 1, 0), (layers // 2, 1, layers - 1, 1)):
            if (i, kv) == (j, other):
                continue
            given = [[list(x) for x in kv_] for kv_ in stores]
            given[j][other][u] = given[i][kv][u]
            want = S if n_last[u] else 0      # (a user without tokens has nothing that could move twice)
            assert _answer(_views(given, lens, dev), n_last) == want


def test_users_may_have_the_same_addresses_as_others():
    """What two users share is not looked at: a cache is a user's."""
    stores = _layers(2, 2)
    for kv in range(2):
        stores[1][kv][1] = stores[0][kv][0]
    assert _answer(_views(stores, [30, 30]), [3, 4]) == 0


def test_arrays_on_the_device():
    one, two = View(k_ptrs_dev=P, v_ptrs_dev=2 * P), View(k_ptrs_dev=3 * P, v_ptrs_dev=2 * P)
    assert _keep([one, two]) == S and _keep([one]) == 0
