"""What the attention launches at the limits of its sizes, seen without a GPU (tests/attention_limits_driver.cpp, linked as in
test_attention_launches.py)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2403_04206_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


@pytest.mark.skipif(not os.path.exists(HIPCC) or shutil.which("g++") is None, reason="no compiler")
def test_launches_at_the_limits(tmp_path):
    objects = []
    for src in [os.path.join(CSRC, n) for n in ("grawa_attention.cpp", "grawa_heads.hip", "grawa_attend.hip", "grawa_attend_back.hip")] + [os.path.join(ROOT, "tests", "attention_limits_driver.cpp")]:
        objects.append(str(tmp_path / (os.path.basename(src) + ".o")))
        res = subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-w", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src, "-o", objects[-1]],
                             capture_output=True, text=True)
        assert res.returncode == 0, res.stderr
    exe = str(tmp_path / "driver")
    res = subprocess.run(["g++", "-no-pie"] + objects + ["-Wl,--unresolved-symbols=ignore-in-object-files", "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr
