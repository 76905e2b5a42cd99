"""Rows of heads far apart, without a GPU: the library's host side with its launchers replaced by stubs, under the sanitizers
(tests/attention_strides_driver.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM_INCLUDE = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g", "-O1"]


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(ROCM_INCLUDE), reason="no host compiler or HIP headers")
def test_rows_far_apart(tmp_path):
    csrc = os.path.join(ROOT, "paper_2403_04206_amd", "csrc")
    out = str(tmp_path / "driver")
    res = subprocess.run(["g++", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__"] + SAN + ["-I", ROCM_INCLUDE, "-I", os.path.join(ROOT, "include"), "-I", csrc,
                          os.path.join(ROOT, "tests", "attention_strides_driver.cpp"), os.path.join(csrc, "grawa_attention.cpp"), "-o", out],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([out], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr
