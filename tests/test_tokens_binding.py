"""What the Python side of the calls for several tokens per user refuses before the library is asked (no GPU: the tensors lie elsewhere, as they are meant to)."""
import pytest
import torch

import paper_2409_19134_amd as spd


class Elsewhere:
    """A tensor's place in memory and nothing else of it."""

    def __init__(self, like, device):
        self.like, self.device_index = like, device

    def get_device(self):
        return self.device_index

    def __getattr__(self, name):
        return getattr(self.like, name)


def _context():
    """A context's checks without a device behind it."""
    ctx = spd.Context.__new__(spd.Context)
    ctx.device, ctx.handle = 0, None
    return ctx


def _views(device):
    k = [Elsewhere(torch.zeros((2, 30, 64)), device) for _ in range(2)]
    pool, table = Elsewhere(torch.zeros((4, 2, 16, 64)), device), Elsewhere(torch.zeros((2, 2), dtype=torch.int32), device)
    here = Elsewhere(torch.zeros((4, 2, 16, 64)), 0)
    yield spd.KVView([30, 20], 64, 30 * 64, k=k, v=[Elsewhere(t.like, 0) for t in k])
    yield spd.KVView([30, 20], 64, 30 * 64, k=[Elsewhere(t.like, 0) for t in k], v=k)
    yield spd.KVView([30, 20], 64, 16 * 64, k_pool=pool, v_pool=here, block_table=Elsewhere(table.like, 0), block_size=16, block_stride=2 * 16 * 64)
    yield spd.KVView([30, 20], 64, 16 * 64, k_pool=here, v_pool=pool, block_table=Elsewhere(table.like, 0), block_size=16, block_stride=2 * 16 * 64)
    yield spd.KVView([30, 20], 64, 16 * 64, k_pool=here, v_pool=here, block_table=table, block_size=16, block_stride=2 * 16 * 64)


@pytest.mark.parametrize("device", [-1, 1])
def test_caches_elsewhere_are_refused(device):
    """A cache or block table in host memory or on another card, whose addresses a kernel must not follow.  (Without a context the library itself answers
    SPD_ERR_NULL: what is not refused gets there.)"""
    ctx, shape = _context(), spd.make_shape(torch.float32, 4, 2, 64, 0.125)
    q, kv, out, lse = (Elsewhere(torch.zeros(s), 0) for s in ((3, 4, 64), (3, 2, 64), (3, 4, 64), (3, 4)))
    for where, refusal in ((device, AssertionError), (0, spd.SpdError)):
        for view in _views(where):
            with pytest.raises(refusal):
                ctx.spd_partial_attn_tokens(shape, q, view, [1, 2], None, out, lse, stream=_Stream)
            with pytest.raises(refusal):
                ctx.spd_append_tokens(shape, view, [1, 2], kv, kv, stream=_Stream)


def test_an_empty_cache_may_lie_anywhere():
    ctx, shape = _context(), spd.make_shape(torch.float32, 4, 2, 64, 0.125)
    view = spd.KVView([0], 64, 0, k=[torch.zeros((2, 0, 64))], v=[torch.zeros((2, 0, 64))])
    q, out, lse = (Elsewhere(torch.zeros(s), 0) for s in ((2, 4, 64), (2, 4, 64), (2, 4)))
    with pytest.raises(spd.SpdError):
        ctx.spd_partial_attn_tokens(shape, q, view, [2], spd.Score(q_pos=[0]), out, lse, stream=_Stream)


class _Stream:
    cuda_stream = 0
