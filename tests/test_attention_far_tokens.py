"""Tokens that are far apart in memory: what a head does not have of a tile's row is not read, however long the rows are."""
import math
import os
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no compiler")
def test_offsets_of_pieces(tmp_path):
    """Every piece of every load of every tile is where its row has it, or beyond the largest descriptor (tests/attention_pieces_driver.cpp)."""
    exe = str(tmp_path / "driver")
    res = subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-w", "-I", os.path.join(ROOT, "include"), "-I",
                          os.path.join(ROOT, "paper_2403_04206_amd", "csrc"), os.path.join(ROOT, "tests", "attention_pieces_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr


@pytest.mark.gpu
@pytest.mark.parametrize("D", [72, 120, 128])
@pytest.mark.parametrize("token", [8600000, (1 << 24) - 16])
def test_values_far_apart(token, D):
    """256 tokens of values 8.6 and 16.8 MB apart with no numbers between them."""
    from test_gpu_attention import Case
    c = Case(1, 1, 300, 300, 2, 1, D, torch.bfloat16, seed=51)
    room = torch.full((299 * (token // 2) + D,), math.nan, device="cuda", dtype=torch.bfloat16)
    v = room.as_strided((1, 1, 300, 1, D), (room.numel(), room.numel(), token // 2, D, 1))
    v.copy_(c.v)
    c.v = v
    c.check()
