"""One SPD decode step for one layer: private partial, public batched partial, merge (paper section 4, step 3).

Pure call sequencing over the C ABI; holds the output buffers so a step allocates nothing.
"""
from __future__ import annotations

import numpy as np
import torch

from .binding import Context, KVView, Rope, Score, make_shape


class DecodeStep:
    def __init__(self, ctx: Context, dtype, n_q_heads: int, n_kv_heads: int, head_dim: int, scale: float,
                 private: KVView, public: KVView, device="cuda:0"):
        self.ctx = ctx
        self.shape = make_shape(dtype, n_q_heads, n_kv_heads, head_dim, scale)
        self.private, self.public = private, public
        n = private.struct.n_users
        assert public.struct.n_users == n
        f32 = dict(device=device, dtype=torch.float32)
        self.a_in = torch.empty((n, n_q_heads, head_dim), **f32)
        self.a_out = torch.empty((n, n_q_heads, head_dim), **f32)
        self.y = torch.empty((n, n_q_heads, head_dim), **f32)
        self.lse_in = torch.empty((n, n_q_heads), **f32)
        self.lse_out = torch.empty((n, n_q_heads), **f32)
        self.lse = torch.empty((n, n_q_heads), **f32)
        self.w_in = torch.empty((n, n_q_heads), **f32)

    @classmethod
    def from_workload(cls, ctx: Context, wl, device_pointer_tables: bool = False) -> "DecodeStep":
        return cls(ctx, wl.dtype, wl.n_q_heads, wl.n_kv_heads, wl.head_dim, wl.scale,
                   KVView.from_side(wl.private, device_pointer_tables), KVView.from_side(wl.public, device_pointer_tables),
                   device=wl.q.device)

    def run(self, q: torch.Tensor, stream=None):
        """Enqueue the three calls on `stream` (default: torch's current stream).  No synchronisation."""
        c = self.ctx
        c.spd_partial_attn_private(self.shape, q, self.private, self.a_in, self.lse_in, stream)
        c.spd_partial_attn_public_batched(self.shape, q, self.public, self.a_out, self.lse_out, stream)
        c.spd_lse_merge(self.a_in, self.lse_in, self.a_out, self.lse_out, self.y, self.lse, self.w_in, stream)
        return self.y

    def run_two_parties(self, q: torch.Tensor, stream=None, k_new=None, v_new=None):
        """The deployment of the paper in two calls: the users' side (private partials) and the service's side
        (public partial, optional append, and the merge) - spd_public_attn_merge closes the step."""
        c = self.ctx
        c.spd_partial_attn_private(self.shape, q, self.private, self.a_in, self.lse_in, stream)
        return c.spd_public_attn_merge(self.shape, q, self.public, self.a_in, self.lse_in, self.a_out, self.lse_out,
                                       self.y, self.lse, self.w_in, stream, k_new, v_new)

    def run_fused(self, q: torch.Tensor, stream=None, k_new=None, v_new=None):
        """The same step through spd_decode_step: one launch for both owners, one closing kernel.  With k_new / v_new
        the new token is appended to the public cache in the same launch (the view's lengths already count it)."""
        return self.ctx.spd_decode_step(self.shape, q, self.private, self.public, self.a_in, self.lse_in, self.a_out,
                                        self.lse_out, self.y, self.lse, self.w_in, stream, k_new, v_new)

    def prepare(self, q: torch.Tensor, stream_ptr: int, k_new=None, v_new=None):
        """Marshal the three calls' arguments once; `run_prepared` then only makes the three C calls.
        For loops that reuse the same q buffer and stream (serving loops, benchmarks)."""
        import ctypes as C
        from .binding import lib
        n, Hq, d = self.private.struct.n_users, self.shape.n_q_heads, self.shape.head_dim
        assert q.is_contiguous() and tuple(q.shape) == (n, Hq, d)
        h, sp, st = self.ctx.handle, C.byref(self.shape), C.c_void_p(stream_ptr)
        self._keep_q = (q, k_new, v_new)
        self._calls = (
            (lib.spd_partial_attn_private, (h, sp, q.data_ptr(), C.byref(self.private.struct),
                                            self.a_in.data_ptr(), self.lse_in.data_ptr(), st)),
            (lib.spd_partial_attn_public_batched, (h, sp, q.data_ptr(), C.byref(self.public.struct),
                                                   self.a_out.data_ptr(), self.lse_out.data_ptr(), st)),
            (lib.spd_lse_merge, (h, n * Hq, d, self.a_in.data_ptr(), self.lse_in.data_ptr(), self.a_out.data_ptr(),
                                 self.lse_out.data_ptr(), self.y.data_ptr(), self.lse.data_ptr(),
                                 self.w_in.data_ptr(), st)),
        )

        self._fused = (lib.spd_decode_step, (h, sp, q.data_ptr(), C.byref(self.private.struct),
                                             C.byref(self.public.struct),
                                             None if k_new is None else k_new.data_ptr(),
                                             None if v_new is None else v_new.data_ptr(), self.a_in.data_ptr(),
                                             self.lse_in.data_ptr(), self.a_out.data_ptr(), self.lse_out.data_ptr(),
                                             self.y.data_ptr(), self.lse.data_ptr(), self.w_in.data_ptr(), st))

        self._two_parties = (
            self._calls[0],
            (lib.spd_public_attn_merge, (h, sp, q.data_ptr(), C.byref(self.public.struct),
                                         None if k_new is None else k_new.data_ptr(),
                                         None if v_new is None else v_new.data_ptr(), self.a_in.data_ptr(),
                                         self.lse_in.data_ptr(), self.a_out.data_ptr(), self.lse_out.data_ptr(),
                                         self.y.data_ptr(), self.lse.data_ptr(), self.w_in.data_ptr(), st)),
        )

    def run_prepared_two_parties(self):
        """The users' call (private partials) and the service's call (public partial and merge), arguments prepared."""
        for fn, args in self._two_parties:
            rc = fn(*args)
            if rc != 0:
                self.ctx._check(rc, fn.__name__)
        return self.y

    def run_prepared_fused(self):
        fn, args = self._fused
        rc = fn(*args)
        if rc != 0:
            self.ctx._check(rc, "spd_decode_step")
        return self.y

    def run_prepared(self, public_first: bool = False):
        """The three calls in sequence on the prepared stream; public_first swaps the two partial calls (the order
        in which the paper's service runs its own attention before it hears from the user processes)."""
        order = (1, 0, 2) if public_first else (0, 1, 2)
        for i in order:
            fn, args = self._calls[i]
            rc = fn(*args)
            if rc != 0:
                self.ctx._check(rc, fn.__name__)
        return self.y

    def run_streams(self, q: torch.Tensor, side: "torch.cuda.Stream"):
        """The two owners on two HIP streams of equal priority: the private call on torch's current stream, the public
        call on `side`, joined by events before the merge (the paper's "start the private computation as soon as Q
        exists" schedule, section 5, with streams standing in for processes).  No host synchronisation."""
        c = self.ctx
        main = torch.cuda.current_stream()
        fork = torch.cuda.Event()
        fork.record(main)          # everything already queued on main (the previous merge reads a_out) comes first
        side.wait_event(fork)
        c.spd_partial_attn_public_batched(self.shape, q, self.public, self.a_out, self.lse_out, side)
        join = torch.cuda.Event()
        join.record(side)
        c.spd_partial_attn_private(self.shape, q, self.private, self.a_in, self.lse_in, main)
        main.wait_event(join)
        c.spd_lse_merge(self.a_in, self.lse_in, self.a_out, self.lse_out, self.y, self.lse, self.w_in, main)
        return self.y


class TokenStep:
    """Several new tokens per user through one layer's caches: a prompt (or a chunk of one) into the cache that holds it, or tokens that follow a
    prompt in another owner's cache (one each, or several that are to be checked at once).

    `view` is the cache that takes the tokens: its lengths already count them, n_new[u] of user u.  With `prompt` (the other owner's view of
    the same users) the sequence begins there: the tokens attend to both caches, and the two partials are merged as in Theorem 1.  `rope`, and the
    keywords of Score that concern a sequence (cap, slopes, causal, window, prefix, ranges), are the model's.  Holds the result buffers, which are fp32.  The views'
    lengths are read at every run, so a loop may move them on."""

    def __init__(self, ctx: Context, dtype, n_q_heads: int, n_kv_heads: int, head_dim: int, scale: float, view: KVView, n_new,
                 rope: Rope = None, prompt: KVView = None, device="cuda:0", **score):
        self.ctx, self.view, self.prompt, self.rope = ctx, view, prompt, rope
        self.shape = make_shape(dtype, n_q_heads, n_kv_heads, head_dim, scale)
        self.n_new = np.ascontiguousarray(n_new, dtype=np.int32)
        T = int(self.n_new.sum())
        f32 = dict(device=device, dtype=torch.float32)
        self.q = torch.empty((T, n_q_heads, head_dim), device=device, dtype=dtype)
        self.a_out, self.lse_out = torch.empty((T, n_q_heads, head_dim), **f32), torch.empty((T, n_q_heads), **f32)
        begin = None if prompt is None else prompt.lens
        self.score_out = Score(k_pos=begin, **score)      # (the same array: what the caller makes of the lengths holds from the next run on)
        if prompt is not None:
            assert prompt.struct.n_users == view.struct.n_users
            self.a_in, self.y = (torch.empty((T, n_q_heads, head_dim), **f32) for _ in range(2))
            self.lse_in, self.lse, self.w_in = (torch.empty((T, n_q_heads), **f32) for _ in range(3))
            self.score_in = Score(q_pos=np.zeros_like(begin), **score)

    def run(self, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, positions: torch.Tensor = None, stream=None):
        """Enqueues the step; returns (attention, its log-sum-exp).  q, k_new, v_new: [T][heads][d] as the projection leaves them; positions
        (with a rope): int32 [axes][T]."""
        c = self.ctx
        turned = c.spd_append_tokens(self.shape, self.view, self.n_new, k_new, v_new, self.rope, positions,
                                     q if self.rope is not None else None, self.q if self.rope is not None else None, stream)
        q = q if self.rope is None else turned
        c.spd_partial_attn_tokens(self.shape, q, self.view, self.n_new, self.score_out, self.a_out, self.lse_out, stream=stream)
        if self.prompt is None:
            return self.a_out, self.lse_out
        np.add(self.prompt.lens, self.view.lens - self.n_new, out=self.score_in.per_user["q_pos"])
        c.spd_partial_attn_tokens(self.shape, q, self.prompt, self.n_new, self.score_in, self.a_in, self.lse_in, stream=stream)
        c.spd_lse_merge(self.a_in, self.lse_in, self.a_out, self.lse_out, self.y, self.lse, self.w_in, stream)
        return self.y, self.lse
