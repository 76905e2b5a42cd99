"""Argument checks of the attention without a GPU: the library's host side with its launchers replaced by stubs
(tests/attention_host_driver.cpp, under the sanitizers), and the Python binding's, on CPU tensors that stand in for device memory; the
tables that the binding makes."""
import ctypes as C
import math
import os
import shutil
import subprocess

import pytest
import torch

from paper_2403_04206_amd import grawa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM_INCLUDE = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
# a type that is none of the enumeration's is passed on purpose
SAN = ["-fsanitize=address,undefined", "-fno-sanitize=enum", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g", "-O1"]


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(ROCM_INCLUDE), reason="no host compiler or HIP headers")
def test_host_side(tmp_path):
    csrc = os.path.join(ROOT, "paper_2403_04206_amd", "csrc")
    out = str(tmp_path / "driver")
    res = subprocess.run(["g++", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__"] + SAN + ["-I", ROCM_INCLUDE, "-I", os.path.join(ROOT, "include"), "-I", csrc,
                          os.path.join(ROOT, "tests", "attention_host_driver.cpp"), os.path.join(csrc, "grawa_attention.cpp"), "-o", out],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([out], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr


K, N, S, H, G, D, B = 2, 3, 4, 4, 2, 16, 5


def make_plan(buckets):
    p = grawa.AttentionPlan.__new__(grawa.AttentionPlan)
    p.K, p.N, p.S, p.H, p.G, p.D, p.dtype, p.buckets, p._device = K, N, S, H, G, D, torch.bfloat16, buckets, 0
    p._dims = (K, N, S, H, G, D, grawa.BF16, 0)
    p._h = C.c_void_p(0)
    return p


@pytest.fixture()
def reached(monkeypatch):
    """The names of the library's functions that calls come to."""
    names = []
    monkeypatch.setattr(grawa, "_REQUIRE_DEVICE", False)

    class Library:
        def __getattr__(self, name):
            return lambda *args: names.append(name) or 0
    monkeypatch.setattr(grawa, "lib", lambda: Library())
    monkeypatch.setattr(grawa.AttentionPlan, "_here", lambda self: 0)
    return names


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def short(*shape, dtype=torch.bfloat16):
    """A view that says it has a shape whose memory it does not have."""
    t = zeros(*shape, dtype=dtype)
    t.untyped_storage().resize_(t.untyped_storage().nbytes() - 2)
    return t


def bad_heads(h):
    return [zeros(K, N, S, h, D, dtype=torch.float32), zeros(K, N, S, h, D + 8), zeros(K, N, S, h + 1, D), zeros(K, N, S + 1, h, D), zeros(K, N + 1, S, h, D), zeros(K + 1, N, S, h, D),
            zeros(K, N * S, h, D), zeros(K, N, S, h, 2 * D)[..., ::2], short(K, N, S, h, D), None]


def everything(buckets):
    """The arguments of each call, in order, by name."""
    q, k, w, bias = zeros(K, N, S, H, D), zeros(K, N, S, G, D), zeros(K, D), zeros(K, H, B) if buckets else None
    places, lse = torch.zeros((K, N), dtype=torch.int32), torch.zeros((K, N, H, S))
    return {"head_norm": dict(q=q, k=k, qweight=w, kweight=w, q_out=q, k_out=k, starts=places),
            "head_norm_backward": dict(dq_out=q, dk_out=k, q=q, k=k, qweight=w, kweight=w, dq=q, dk=k, dqweight=w, dkweight=w, starts=places),
            "attention": dict(q=q, k=k, v=k, out=q, lse_out=lse, bias=bias, lengths=places, starts=places),
            "attention_backward": dict(dout=q, q=q, k=k, v=k, out=q, lse=lse, dq=q, dk=k, dv=k, bias=bias, dbias=bias, lengths=places, starts=places)}


@pytest.mark.parametrize("buckets", [0, B])
@pytest.mark.parametrize("call", ["head_norm", "head_norm_backward", "attention", "attention_backward"])
def test_every_argument_is_checked(call, buckets, reached):
    plan, good = make_plan(buckets), everything(buckets)[call]
    getattr(plan, call)(**good)
    assert reached == ["grawa_" + call]
    for name, value in good.items():
        if name in ("starts", "lengths"):
            bad = [torch.zeros((K, N)), torch.zeros((K, N), dtype=torch.int64), torch.zeros((K, N + 1), dtype=torch.int32), torch.zeros((K * N,), dtype=torch.int32),
                   torch.zeros((N, K), dtype=torch.int32).t(), short(K, N, dtype=torch.int32)]
        elif name in ("lse", "lse_out"):
            bad = [torch.zeros((K, N, S, H + 1)), torch.zeros((K, N, H, S), dtype=torch.float64), torch.zeros((K, N, H, S + 1)), torch.zeros((K, N, S, H)).transpose(2, 3), short(K, N, H, S, dtype=torch.float32)]
            bad += [None] if name == "lse" else []
        elif "weight" in name:
            bad = [zeros(K, D, dtype=torch.float32), zeros(K, D + 8), zeros(K + 1, D), zeros(D), zeros(K, 2 * D)[:, ::2], short(K, D), None]
        elif "bias" in name:
            bad = [zeros(K, H, B, dtype=torch.float32), zeros(K, H, B + 1), zeros(K, H * B), zeros(K, B, H).transpose(1, 2), short(K, H, B), None] if buckets else [zeros(K, H, B)]
        else:
            bad = bad_heads(value.shape[3])
        for b in bad:
            del reached[:]
            with pytest.raises((TypeError, ValueError)):
                getattr(plan, call)(**{**good, name: b})
            assert not reached, (call, name)
    for name in ("starts", "lengths", "lse_out"):                # these may be left out
        if name in good:
            getattr(plan, call)(**{**good, name: None})
            assert reached == ["grawa_" + call]
            del reached[:]


def test_more_than_the_plan_takes(reached):
    plan = make_plan(0)
    for n, s in ((N + 1, S), (N, S + 1)):
        q, k, w = zeros(K, n, s, H, D), zeros(K, n, s, G, D), zeros(K, D)
        for fn in (lambda: plan.head_norm(q, k, w, w, q, k), lambda: plan.attention(q, k, k, q)):
            with pytest.raises(ValueError):
                fn()
    assert not reached
    q, k = zeros(K, 2, 1, H, D), zeros(K, 2, 3, G, D)            # fewer sequences, fewer new tokens than keys
    plan.attention(q, k, k, q)
    assert reached == ["grawa_attention"]


def test_plans_refuse_what_does_not_go_together():
    for bad in (dict(dtype=torch.float16), dict(buckets=3), dict(bucket_of=[0, 1]), dict(buckets=2, bucket_of=[[0], [1]]), dict(frequencies=[[1.0]])):
        with pytest.raises((TypeError, ValueError)):
            grawa.AttentionPlan(1, 1, 8, 2, 1, 64, **bad)


def test_frequencies():
    f = grawa.rotary_frequencies(8, 16.0)
    assert f == [1.0, 0.5, 0.25, 0.125] and grawa.rotary_frequencies(0) == []
    for bad in ((3,), (-2,), (8, 0.0)):
        with pytest.raises(ValueError):
            grawa.rotary_frequencies(*bad)


@pytest.mark.parametrize("buckets,far", [(2, 2), (2, 100), (3, 2), (8, 20), (19, 77), (32, 128), (64, 464), (256, 1000)])
def test_buckets_of_distances(buckets, far):
    """Half a bucket for each distance, then the floor of a logarithm; whole numbers to the rest, so away from borders both agree."""
    of = grawa.log_buckets(buckets, far)
    half = buckets // 2
    assert of[:half] == list(range(half)) and of[-1] == buckets - 1 and of[-2] < buckets - 1 and all(0 <= b - a <= buckets for a, b in zip(of, of[1:]))
    assert len(of) <= far + 1
    for n in range(half, len(of)):
        x = (buckets - half) * math.log(n / half) / math.log(far / half)
        if abs(x - round(x)) > 1e-9:
            assert of[n] == min(half + int(x), buckets - 1), n
    for bad in ((1, 10), (8, 4), (8, 2)):
        with pytest.raises(ValueError):
            grawa.log_buckets(*bad)
