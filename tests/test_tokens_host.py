"""The calls for several tokens per user without a GPU: their argument checks, their tables and masks, and what the compiler makes of their kernels."""
import ctypes as C
import importlib.util
import math
import os
import re
import subprocess

import numpy as np
import pytest

import paper_2409_19134_amd as spd
from paper_2409_19134_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
P = 0x10000      # an address that is never followed


def test_tables_and_masks_under_asan_ubsan(tmp_path):
    """tests/host/tokens_schedule_fuzz.cpp: every row in one tile, every key that a row sees in exactly one of its tile's stretches."""
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    exe = str(tmp_path / "tokens_schedule_fuzz")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-x", "hip", "-Xarch_host", "-fsanitize=address,undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-o", exe, os.path.join(ROOT, "tests", "host", "tokens_schedule_fuzz.cpp")]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("ok 400"), run.stdout[-3000:]


@pytest.mark.parametrize("source", ["tokens_api.hip", "tokens_few.hip", "tokens_many.hip"])
def test_no_kernel_spills_registers(source, tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    spec = importlib.util.spec_from_file_location("spd_build", os.path.join(ROOT, "paper_2409_19134_amd", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    cmd = [HIPCC, *(f for f in build.HIPCC_FLAGS if f != "-shared"), "-Rpass-analysis=kernel-resource-usage", "-c", "-o", str(tmp_path / "x.o"),
           os.path.join(ROOT, "paper_2409_19134_amd", "csrc", source)]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-3000:]
    spills = [int(x) for x in re.findall(r"VGPRs Spill: (\d+)", res.stdout)]
    scratch = [int(x) for x in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", res.stdout)]
    assert len(spills) >= 20 and len(scratch) == len(spills) and max(spills) == 0 and max(scratch) == 0


def _shape(**kw):
    s = dict(dtype=spd.SPD_BF16, n_q_heads=8, n_kv_heads=2, head_dim=64, scale=0.125)
    s.update(kw)
    return spd.spd_shape(*s.values())


class View:
    """A contiguous view of two users whose addresses are never followed."""

    def __init__(self, lens=(20, 30), **kw):
        self.lens = np.array(lens, np.int32)
        self.ptrs = (C.c_void_p * len(lens))(*[P] * len(lens))
        st = spd.spd_kv_view()
        st.n_users, st.lens = len(lens), self.lens.ctypes.data_as(C.POINTER(C.c_int32))
        st.k_ptrs = st.v_ptrs = C.cast(self.ptrs, C.POINTER(C.c_void_p))
        st.token_stride, st.head_stride = 64, 64 * 64
        for k, v in kw.items():
            setattr(st, k, v)
        self.struct = st


def _counts(n):
    a = np.array(n, np.int32)
    return a, a.ctypes.data


def _tokens(shape=None, q=P, q_stride=8 * 64, view=None, n_new=(1, 2), score=None, out=P, out_dtype=spd.SPD_F32, lse=P):
    view = view or View()
    keep, n = _counts(n_new) if n_new is not None else (None, None)
    keep2 = score
    return b.lib.spd_validate_tokens(C.byref(shape or _shape()), q, q_stride, C.byref(view.struct), n, None if score is None else C.byref(score.struct), out,
                                     out_dtype, lse)


def test_refusals_of_the_attention():
    S, L, N, A = spd.SPD_ERR_SHAPE, spd.SPD_ERR_LEN, spd.SPD_ERR_NULL, spd.SPD_ERR_ALIGN
    score = spd.Score
    assert _tokens() == 0 and _tokens(score=score(cap=30.0, window=5, prefix=[0, 9], k_pos=[3, 4])) == 0
    assert _tokens(shape=_shape(head_dim=96)) == S and _tokens(shape=_shape(n_q_heads=9)) == S and _tokens(shape=_shape(scale=math.inf)) == S
    assert _tokens(shape=_shape(n_q_heads=34)) == S                        # 17 query heads to a KV head
    assert _tokens(out_dtype=spd.SPD_F16) == S and _tokens(out_dtype=spd.SPD_BF16) == 0
    assert _tokens(n_new=None) == N and _tokens(q=None) == N and _tokens(out=None) == N and _tokens(lse=None) == N
    assert _tokens(n_new=(0, 0), q=None, out=None, lse=None) == 0           # nothing to do
    assert _tokens(n_new=(21, 1)) == L and _tokens(n_new=(-1, 1)) == L       # more than the view holds
    assert _tokens(n_new=(21, 1), score=score(q_pos=[0, 5])) == 0           # ... which is for the caller to say
    assert _tokens(n_new=((1 << 30), 1), score=score(q_pos=[0, 5])) == L    # T * Hq
    assert _tokens(score=score(q_pos=[1 << 30, 0])) == L and _tokens(score=score(q_pos=[-1, 0])) == L
    assert _tokens(score=score(k_pos=[-1, 0])) == L and _tokens(score=score(k_pos=[0, (1 << 30) - 29])) == L
    assert _tokens(score=score(prefix=[0, -2])) == L and _tokens(score=score(window=-1)) == L and _tokens(score=score(window=1 << 30)) == 0
    for cap in (-1.0, math.inf, math.nan, 1e-45):
        assert _tokens(score=score(cap=cap)) == S, cap
    bad = score()
    bad.struct.causal = 2
    assert _tokens(score=bad) == S
    bad = score()
    bad.struct.slopes = P + 2
    assert _tokens(score=bad) == A
    bad = score()
    bad.struct.ranges = P + 4
    assert _tokens(score=bad) == A
    assert _tokens(q=P + 8) == A and _tokens(out=P + 4) == A and _tokens(lse=P + 2) == A
    assert _tokens(q_stride=8 * 64 - 8) == A and _tokens(q_stride=8 * 64 + 4) == A and _tokens(q_stride=8 * 64 + 8) == 0
    assert _tokens(view=View(lens=(20, -1))) == L and _tokens(view=View(token_stride=60)) == A and _tokens(view=View(block_size=24)) == S


def _append(shape=None, view=None, n_new=(1, 2), rope=None, positions=None, q=None, qs=8 * 64, q_out=None, k=P, ks=2 * 64, v=P, vs=2 * 64):
    view = view or View()
    keep, n = _counts(n_new)
    return b.lib.spd_validate_append(C.byref(shape or _shape()), C.byref(view.struct), n, None if rope is None else C.byref(rope), positions, q, qs, q_out,
                                     k, ks, v, vs)


def _rope(**kw):
    s = dict(n_axes=1, n_pairs=32, adjacent=0, pair_axis=None, inv_freq=P, amplitude=1.0)
    s.update(kw)
    return b.spd_rope(*s.values())


def test_refusals_of_the_append():
    S, L, N, A = spd.SPD_ERR_SHAPE, spd.SPD_ERR_LEN, spd.SPD_ERR_NULL, spd.SPD_ERR_ALIGN
    assert _append() == 0 and _append(rope=_rope(), positions=P) == 0 and _append(q=P, q_out=P) == 0
    assert _append(rope=_rope()) == N and _append(q=P) == N and _append(q_out=P) == N and _append(k=None) == N and _append(v=None) == N
    assert _append(n_new=(0, 0), k=None, v=None) == 0 and _append(n_new=(21, 0)) == L and _append(n_new=(0, -1)) == L
    assert _append(ks=2 * 64 - 8) == A and _append(vs=2 * 64 + 4) == A and _append(k=P + 2) == A and _append(v=P + 8) == A
    assert _append(q=P, q_out=P + 1) == A and _append(q=P, q_out=P, qs=9 * 64) == A and _append(q=P, q_out=P * 16, qs=9 * 64) == 0
    assert _append(rope=_rope(), positions=P + 1) == A
    for kw in (dict(n_axes=0), dict(n_axes=4), dict(n_pairs=0), dict(n_pairs=12), dict(n_pairs=40), dict(adjacent=2), dict(amplitude=math.nan)):
        assert _append(rope=_rope(**kw), positions=P) == S, kw
    assert _append(rope=_rope(inv_freq=None), positions=P) == N and _append(rope=_rope(inv_freq=P + 2), positions=P) == A
    axis = (C.c_uint8 * 32)(*[0] * 31 + [1])
    assert _append(rope=_rope(pair_axis=C.cast(axis, C.c_void_p)), positions=P) == S
    assert _append(rope=_rope(n_axes=2, pair_axis=C.cast(axis, C.c_void_p)), positions=P) == 0


def _rotate(dtype=spd.SPD_BF16, d=64, rope=None, n=5, pos=P, heads=8, x=P, xs=512, y=P, ys=512):
    rope = rope or _rope()
    return b.lib.spd_validate_rotate(dtype, d, C.byref(rope), n, pos, heads, x, xs, y, ys)


def test_refusals_of_the_rotation():
    S, L, N, A = spd.SPD_ERR_SHAPE, spd.SPD_ERR_LEN, spd.SPD_ERR_NULL, spd.SPD_ERR_ALIGN
    assert _rotate() == 0 and _rotate(y=P * 16, ys=1024) == 0
    assert _rotate(dtype=7) == S and _rotate(d=96) == S and _rotate(heads=0) == S and _rotate(heads=65536, xs=1 << 23, ys=1 << 23) == S
    assert _rotate(n=-1) == L and _rotate(n=0, pos=None, x=None, y=None) == 0
    assert _rotate(pos=None) == N and _rotate(x=None) == N and _rotate(y=None) == N
    assert _rotate(ys=1024) == A and _rotate(xs=504) == A and _rotate(x=P + 8) == A and _rotate(pos=P + 2) == A
    assert b.lib.spd_validate_rotate(spd.SPD_BF16, 64, None, 5, P, 8, P, 512, P, 512) == N


def test_calls_need_a_context():
    s, v, n, r = _shape(), View(), _counts((1, 2)), _rope()
    assert b.lib.spd_rotate(None, 1, 64, C.byref(r), 1, P, 8, P, 512, P, 512, 0, None) == spd.SPD_ERR_NULL
    assert b.lib.spd_append_tokens(None, C.byref(s), C.byref(v.struct), n[1], None, None, None, 0, None, P, 128, P, 128, None) == spd.SPD_ERR_NULL
    assert b.lib.spd_partial_attn_tokens(None, C.byref(s), P, 512, C.byref(v.struct), n[1], None, P, 0, P, None) == spd.SPD_ERR_NULL


def test_refusals_of_caps_and_strides():
    """Caps whose factors would not be finite or lose bits; strides whose products with a token's number the kernels cannot hold."""
    S, A = spd.SPD_ERR_SHAPE, spd.SPD_ERR_ALIGN
    for cap in (1.001e30, 3e38, 1e-39):      # (0.125 / 1e-39 four times is past the largest value)
        assert _tokens(score=spd.Score(cap=cap)) == S, cap
    assert _tokens(score=spd.Score(cap=1e30)) == 0 and _tokens(score=spd.Score(cap=1e-30)) == 0
    assert _tokens(shape=_shape(scale=1e-9), score=spd.Score(cap=1e30)) == S         # scale / cap below 2^-126
    assert _tokens(shape=_shape(scale=0.0), score=spd.Score(cap=1e30)) == 0
    most = (1 << 28) // 2                                                            # in 16-bit elements
    assert _tokens(view=View(token_stride=most, head_stride=64)) == 0 and _tokens(view=View(token_stride=most + 8, head_stride=64)) == A
