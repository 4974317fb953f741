"""The host side of the moves within caches without a GPU: what they launch, recorded by a stand-in HIP runtime (see tests/host/cache_moves_calls.cpp)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    exe = str(tmp_path_factory.mktemp("cache_moves_calls") / "cache_moves_calls")
    cmd = [HIPCC, "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-no-hip-rt", "-rdynamic", "-x", "hip", "-o", exe,
           os.path.join(ROOT, "tests", "host", "cache_moves_calls.cpp"), "-ldl"]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-3000:]
    return exe


def _run(program, *args):
    lib = os.path.join(ROOT, "paper_2409_19134_amd", "libspd_hip.so")
    run = subprocess.run([program, lib, *args], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("ok"), run.stdout[-3000:]


def test_kept_tokens_of_block_tables_of_their_own_widths(program):
    """Layers whose block tables are not equally wide: each user's pages come from its own row of its layer's table."""
    _run(program, "tables")


def test_buffers_given_twice(program):
    """Refused before anything is launched, also by the call that remembers the pointers of calls before."""
    _run(program, "twice")
