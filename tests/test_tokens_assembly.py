"""The assembly of the kernel for many query rows: its loads into LDS take their place from M0, which the compiler has to write in front of each."""
import importlib.util
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """(assembly, what the compiler said)"""
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    spec = importlib.util.spec_from_file_location("spd_build", os.path.join(ROOT, "paper_2409_19134_amd", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    out = str(tmp_path_factory.mktemp("many") / "many.s")
    cmd = [HIPCC, *(f for f in build.HIPCC_FLAGS if f != "-shared"), "--cuda-device-only", "-S", "-o", out,
           os.path.join(ROOT, "paper_2409_19134_amd", "csrc", "tokens_many.hip")]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-3000:]
    with open(out) as f:
        return f.read(), res.stdout


def test_the_compiler_has_nothing_to_say_about_the_inline_assembly(compiled):
    """No reserved register on a list of changed ones, which it says may not be preserved."""
    assert "inline-asm" not in compiled[1] and "reserved register" not in compiled[1], compiled[1][:2000]


def test_every_load_into_lds_has_its_place_in_m0(compiled):
    """Between a load and the one before it, or its block's begin, M0 is written, once at least, then comes a wait state; nothing else names M0."""
    loads, written, waited = 0, False, False
    for line in compiled[0].splitlines():
        code = line.split(";")[0].strip()
        if re.match(r"[.\w$]+:", code):        # a label: M0 may come from several places
            written = False
        if not code or code.startswith("."):
            continue
        if code.startswith("global_load_lds"):
            assert written and waited, line
            loads, written = loads + 1, False
        elif re.match(r"s_\w+ m0, ", code):
            written = True
        else:
            assert not re.search(r"\bm0\b", code), line
        waited = code.startswith("s_nop")
    assert loads >= 24 * 8      # 24 instances, each with the loads of a first and of a following tile, whole and cut, four at least
