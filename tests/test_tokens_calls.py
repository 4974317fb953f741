"""The host side of the calls for several tokens per user without a GPU: what they launch and upload, recorded by a stand-in HIP runtime and gone through
key by key and byte by byte (see tests/host/tokens_calls.cpp)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    exe = str(tmp_path_factory.mktemp("tokens_calls") / "tokens_calls")
    cmd = [HIPCC, "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-no-hip-rt", "-rdynamic", "-x", "hip", "-o", exe,
           os.path.join(ROOT, "tests", "host", "tokens_calls.cpp"), "-ldl"]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-3000:]
    return exe


def _run(program, *args, **env):
    lib = os.path.join(ROOT, "paper_2409_19134_amd", "libspd_hip.so")
    run = subprocess.run([program, lib, *args], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300, env=dict(os.environ, **env))
    assert run.returncode == 0 and run.stdout.strip().endswith("ok"), run.stdout[-3000:]


def test_tables_used_again_hold_every_key(program):
    """Lengths and positions that move on from call to call, each by itself: every key that a query sees is in one of the launched stretches, windows that
    lay behind a cache's last key before it grew among them; a decode loop still builds its table once."""
    _run(program, "growth")


def test_append_tables_used_again(program):
    """Users' lengths that move on alike (the table is used again) or by themselves, in every kind of storage: every new token goes to its place."""
    _run(program, "append")


@pytest.mark.parametrize("told", [0, 1, 5, 300])
def test_as_many_views_as_the_context_was_told_to_remember(program, told):
    """SPD_SCHEDULE_CACHE_ENTRIES, which spd_create reads, holds for these calls too: so many views build their tables once, one more takes a place."""
    _run(program, "entries", str(told), **({"SPD_SCHEDULE_CACHE_ENTRIES": str(told)} if told else {}))


def test_calls_of_more_workgroups_than_a_launch_takes(program):
    """Tens of millions of tokens in one rotation or append, of (user, head) pairs in one attention: every one is taken once."""
    _run(program, "limits")
