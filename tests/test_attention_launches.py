"""What the attention launches, seen without a GPU: the host side of its own files, compiled as it is and linked with a runtime of stubs
that notes every launch (tests/attention_launch_driver.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2403_04206_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if not os.path.exists(HIPCC) or shutil.which("g++") is None:
        pytest.skip("no compiler")
    at = tmp_path_factory.mktemp("launches")
    objects = []
    for src in [os.path.join(CSRC, n) for n in ("grawa_attention.cpp", "grawa_heads.hip", "grawa_attend.hip", "grawa_attend_back.hip")] + [os.path.join(ROOT, "tests", "attention_launch_driver.cpp")]:
        objects.append(str(at / (os.path.basename(src) + ".o")))
        res = subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-w", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src, "-o", objects[-1]],
                             capture_output=True, text=True)
        assert res.returncode == 0, res.stderr
    exe = str(at / "driver")
    # the device code, which is not there, is the only symbol that is left open
    res = subprocess.run(["g++", "-no-pie"] + objects + ["-Wl,--unresolved-symbols=ignore-in-object-files", "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return exe


@pytest.mark.parametrize("what", ["turns", "launches", "reached"])
def test_launches(driver, what):
    """turns: each block of each head is one workgroup's.  launches: grids, shared memory, room for what blocks share, at random numbers and
    at the limits.  reached: no form of a kernel is built that no call comes to."""
    res = subprocess.run([driver, what], capture_output=True, text=True, timeout=100)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr
