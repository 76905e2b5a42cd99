"""What the feed-forward sublayer launches, seen without a GPU: the host side of its own files, compiled as it is and linked with a runtime of
stubs that notes every launch (tests/sublayer_launch_driver.cpp)."""
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
    for src in [os.path.join(CSRC, n) for n in ("grawa_sublayer.cpp", "grawa_layernorm.hip", "grawa_dropout.hip", "grawa_ffn.hip")] + [os.path.join(ROOT, "tests", "sublayer_launch_driver.cpp")]:
        objects.append(str(at / (os.path.basename(src) + ".o")))
        res = subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-w", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src, "-o", objects[-1]],
                             capture_output=True, text=True)
        assert res.returncode == 0, res.stderr
    exe = str(at / "driver")
    # the device code, which is not there, is the only symbol that is left open
    res = subprocess.run(["g++", "-no-pie"] + objects + ["-Wl,--unresolved-symbols=ignore-in-object-files", "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return exe


def run(driver, what):
    res = subprocess.run([driver, what], capture_output=True, text=True, timeout=100)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr


def test_products_read_their_matrices_by_their_own_pitch(driver):
    """Every operand of every product, with each of x, dy, Wg, Wu and Wd on and off 16 bytes: the matrix that it points to has the pitch that the
    product walks it with, and the rows that the product reads are that matrix's."""
    run(driver, "operands")


def test_every_launch_fits_a_grid(driver):
    """Up to the limits that the calls take, and what a card's memory holds: fewer than 2^32 threads along x, at most 65535 blocks along y and z."""
    run(driver, "grids")


def test_every_kernel_is_launched_by_some_call(driver):
    """No form of a kernel is built that no call comes to."""
    run(driver, "reached")
