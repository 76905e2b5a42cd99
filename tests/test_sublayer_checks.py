"""Argument checks of the feed-forward sublayer without a GPU: the library's host side with its launchers replaced by stubs
(tests/sublayer_host_driver.cpp, under the sanitizers), and the Python binding's, on CPU tensors that stand in for device memory."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from paper_2403_04206_amd import grawa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM_INCLUDE = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g", "-O1"]


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(ROCM_INCLUDE), reason="no host compiler or HIP headers")
def test_host_side(tmp_path):
    csrc = os.path.join(ROOT, "paper_2403_04206_amd", "csrc")
    out = str(tmp_path / "driver")
    res = subprocess.run(["g++", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__"] + SAN + ["-I", ROCM_INCLUDE, "-I", os.path.join(ROOT, "include"), "-I", csrc,
                          os.path.join(ROOT, "tests", "sublayer_host_driver.cpp"), os.path.join(csrc, "grawa_sublayer.cpp"), "-o", out],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([out], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr


K, T, d, f = 3, 5, 8, 16


@pytest.fixture()
def plan(monkeypatch):
    monkeypatch.setattr(grawa, "_REQUIRE_DEVICE", False)

    class Reached:
        def __getattr__(self, name):
            if name == "grawa_sublayer_save_bytes":
                def size(h, T, n):
                    n._obj.value = 1000
                    return 0
                return size

            def fn(*args):
                raise AssertionError("%s was reached: validation let a bad argument through" % name)
            return fn
    monkeypatch.setattr(grawa, "lib", lambda: Reached())
    monkeypatch.setattr(grawa, "_stream", lambda s=None: 0)
    p = grawa.SublayerPlan.__new__(grawa.SublayerPlan)
    p.K, p.T, p.d, p.f, p.dtype = K, T, d, f, torch.bfloat16
    p._h = C.c_void_p(0)
    return p


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def short(*shape):
    """A view that says it has a shape whose memory it does not have."""
    t = zeros(*shape)
    t.untyped_storage().resize_(t.untyped_storage().nbytes() - 2)
    return t


BAD_TOKENS = [lambda: zeros(K, T, d, dtype=torch.float32), lambda: zeros(K, T, d + 1), lambda: zeros(K, T + 1, d), lambda: zeros(K + 1, T, d), lambda: zeros(K * T, d),
              lambda: zeros(K, T, 2 * d)[:, :, ::2], lambda: short(K, T, d), lambda: None]
BAD_VECTORS = [lambda: zeros(K, d, dtype=torch.float32), lambda: zeros(K, d + 1), lambda: zeros(K + 1, d), lambda: zeros(d), lambda: zeros(K, 2 * d)[:, ::2], lambda: short(K, d)]
BAD_MATRICES = [lambda: zeros(K, f, d, dtype=torch.float32), lambda: zeros(K, f, d + 1), lambda: zeros(K, d * f), lambda: zeros(K, f, 2 * d)[:, :, :d], lambda: zeros(K, d, f).transpose(1, 2),
                lambda: short(K, f, d), lambda: None]


def refused(fn):
    with pytest.raises((TypeError, ValueError)):
        fn()


def test_tokens_are_checked(plan):
    x, w, m, md = zeros(K, T, d), zeros(K, d), zeros(K, f, d), zeros(K, d, f)
    stats, save = zeros(K, T, 2, dtype=torch.float32), zeros(1000, dtype=torch.uint8)
    for make in BAD_TOKENS:
        b = make()
        refused(lambda: plan.layer_norm(b, w, w, x))
        refused(lambda: plan.layer_norm(x, w, w, b))
        refused(lambda: plan.layer_norm_backward(b, x, w, stats, x, w, w))
        refused(lambda: plan.layer_norm_backward(x, b, w, stats, x, w, w))
        refused(lambda: plan.layer_norm_backward(x, x, w, stats, b, w, w))
        refused(lambda: plan.ffn(b, m, m, md, x))
        refused(lambda: plan.ffn(x, m, m, md, b))
        refused(lambda: plan.ffn_backward(b, x, m, m, md, save, x, m, m, md))
        refused(lambda: plan.ffn_backward(x, b, m, m, md, save, x, m, m, md))
        refused(lambda: plan.ffn_backward(x, x, m, m, md, save, b, m, m, md))
        refused(lambda: grawa.dropout(x, b, 0.0, None))
        if b is not None:
            refused(lambda: plan.ffn(x, m, m, md, x, residual=b))
            refused(lambda: plan.layer_norm_backward(x, x, w, stats, x, w, w, add=b))
            refused(lambda: grawa.dropout(x, x, 0.0, None, residual=b))
    refused(lambda: grawa.dropout(None, x, 0.0, None))
    refused(lambda: grawa.dropout(x.half(), x, 0.0, None))
    refused(lambda: grawa.dropout(x[0], x, 0.0, None))


def test_parameters_are_checked(plan):
    x, w, m, md = zeros(K, T, d), zeros(K, d), zeros(K, f, d), zeros(K, d, f)
    stats, save = zeros(K, T, 2, dtype=torch.float32), zeros(1000, dtype=torch.uint8)
    for make in BAD_VECTORS:
        b = make()
        refused(lambda: plan.layer_norm(x, b, w, x))
        refused(lambda: plan.layer_norm(x, w, b, x))
        refused(lambda: plan.layer_norm_backward(x, x, b, stats, x, w, w))
        refused(lambda: plan.layer_norm_backward(x, x, w, stats, x, b, w))
        refused(lambda: plan.layer_norm_backward(x, x, w, stats, x, w, b))
    refused(lambda: plan.layer_norm(x, None, w, x))
    refused(lambda: plan.layer_norm_backward(x, x, w, stats, x, None, w))
    for make in BAD_MATRICES:
        b = make()
        refused(lambda: plan.ffn(x, b, m, md, x))
        refused(lambda: plan.ffn(x, m, b, md, x))
        refused(lambda: plan.ffn(x, m, m, b, x))
        for i in range(6):
            mats = [m, m, md, m, m, md]
            mats[i] = b
            refused(lambda: plan.ffn_backward(x, x, *mats[:3], save, x, *mats[3:]))


def test_other_buffers_are_checked(plan):
    x, w, m, md = zeros(K, T, d), zeros(K, d), zeros(K, f, d), zeros(K, d, f)
    for stats in (zeros(K, T, 2), zeros(K, T, 3, dtype=torch.float32), zeros(K, 2, T, dtype=torch.float32).transpose(1, 2)):
        refused(lambda: plan.layer_norm(x, w, w, x, stats_out=stats))
        refused(lambda: plan.layer_norm_backward(x, x, w, stats, x, w, w))
    refused(lambda: plan.layer_norm_backward(x, x, w, None, x, w, w))
    for save in (zeros(999, dtype=torch.uint8), zeros(2000), zeros(2000, dtype=torch.uint8)[::2], zeros(10, 100, dtype=torch.uint8)):
        refused(lambda: plan.ffn(x, m, m, md, x, save=save))
        refused(lambda: plan.ffn_backward(x, x, m, m, md, save, x, m, m, md))
    refused(lambda: plan.ffn_backward(x, x, m, m, md, None, x, m, m, md))
    for rng in (None, torch.zeros(2), torch.zeros(1, dtype=torch.int64), torch.zeros(4, dtype=torch.int64)[::2], torch.zeros((2, 1), dtype=torch.int64)):
        refused(lambda: grawa.dropout(x, x, 0.5, rng))
        refused(lambda: plan.ffn(x, m, m, md, x, p=0.5, rng=rng))
    rng = torch.zeros(2, dtype=torch.int64)
    for site in (-1, 1 << 32):
        refused(lambda: grawa.dropout(x, x, 0.5, rng, site=site))
        refused(lambda: plan.ffn(x, m, m, md, x, p=0.5, rng=rng, site=site))


def test_plans_are_checked(monkeypatch):
    refused(lambda: grawa.SublayerPlan(K, T, d, f, dtype=torch.float16))
    refused(lambda: grawa.SublayerPlan(K, T, d, f, activation="tanh"))
    x = zeros(K, T, d)
    with pytest.raises(TypeError):                # not on a device
        grawa.dropout(x, x, 0.0, None)
    for args in ((0, T, d, f), (K, -1, d, f), (K, T, 0, f), (K, T, d, -1)):
        with pytest.raises(grawa.GrawaError) as e:
            grawa.SublayerPlan(*args)
        assert e.value.status == grawa.ERR_INVALID_ARG
    for args in ((grawa.MAX_WORKERS + 1, T, d, f), (2, 1 << 30, d, f), (K, T, 1 << 20, f), (K, T, d, 1 << 20)):
        with pytest.raises(grawa.GrawaError) as e:
            grawa.SublayerPlan(*args)
        assert e.value.status == grawa.ERR_UNSUPPORTED


def test_checks_accept_what_is_in_order(monkeypatch):
    monkeypatch.setattr(grawa, "_REQUIRE_DEVICE", False)
    row = zeros(K, 3 + 2 * d * f)
    b = grawa._mats(row[:, 3:3 + d * f].view(K, f, d), (K, f, d), torch.bfloat16, "wg")._obj
    assert b.worker == 3 + 2 * d * f and b.data == row.data_ptr() + 6
    r = grawa._tokens(zeros(T, K, d).permute(1, 0, 2), K, T, d, torch.bfloat16, "x")._obj
    assert (r.worker, r.row) == (d, K * d)
    r = grawa._tokens(zeros(1, T, d).expand(K, T, d), K, T, d, torch.bfloat16, "x")._obj
    assert (r.worker, r.row) == (0, d)
    assert grawa._tokens(zeros(K, 0, d), K, 0, d, torch.bfloat16, "x") is not None
