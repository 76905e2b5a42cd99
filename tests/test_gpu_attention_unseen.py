"""Gradients beside keys that no query sees because the queries end before the keys do: whatever those keys hold reaches nothing."""
import math

import pytest
import torch

import attention_reference as ref
from paper_2403_04206_amd import grawa
from test_gpu_attention import Case

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
NAN, INF = math.nan, math.inf
# queries, keys, position of the first query: the last query stands before the last key, in the same tile of keys and in others
PLACES = [(100, 128, 0), (100, 128, 17), (1, 40, 3), (70, 300, 20), (600, 640, 0), (600, 1200, 30)]


def odd_keys(case, what, value, last):
    """The keys behind position `last`, all of them or one, are `value`."""
    for t in [case.k, case.v] if what == "both" else [getattr(case, what)]:
        t[:, :, last + 1:, :, 3] = value
        t[:, :, last + 1] = value


def check_gradients(case, want, names):
    case.forward()
    case.backward()
    torch.cuda.synchronize()
    for name in ("o", "lse") + names:
        ref.check(getattr(case, name), *want[name], name)
    case.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("what,value", [("k", NAN), ("v", NAN), ("k", INF), ("both", -INF)])
@pytest.mark.parametrize("Sq,Sk,start", PLACES)
def test_gradients_of_queries_and_bias(Sq, Sk, start, what, value, D, dtype):
    c = Case(1, 2, Sq, Sk, 2, 1, D, dtype, seed=31, starts=[start] * 2, buckets=8, far=30, window=0 if start else 90, sinks=2)
    want = c.want()
    odd_keys(c, what, value, start + Sq - 1)
    check_gradients(c, want, ("dq", "dbias"))


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_of_rows_that_see_nothing(dtype):
    """Every distance of head 0 hidden by the bias, gradients of its outputs no numbers: its dq and dbias are 0, head 1's as without."""
    c = Case(1, 1, 150, 150, 2, 1, 64, dtype, seed=32, buckets=4, far=20)
    c.bias[:, 0] = -INF
    want = c.want()
    for name in ("dq", "dbias"):                                                 # dS of hidden pairs is 0 x do . v = 0 in the formulas too
        assert not bool(want[name][0].select(3 if name == "dq" else 1, 0).any())
    c.do[:, :, :, 0] = NAN
    check_gradients(c, want, ("dq", "dbias"))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("what,value", [("k", NAN), ("v", NAN), ("k", INF), ("both", -INF)])
@pytest.mark.parametrize("Sq,Sk,start", PLACES)
def test_gradients_of_keys_and_values(Sq, Sk, start, what, value, biased, D, dtype):
    c = Case(1, 2, Sq, Sk, 4, 2, D, dtype, seed=33, starts=[start] * 2, window=0 if start else 90, sinks=2, **(dict(buckets=8, far=30) if biased else {}))
    want = c.want()
    odd_keys(c, what, value, start + Sq - 1)
    check_gradients(c, want, ("dq", "dk", "dv"))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_bias_of_distances_that_no_pair_has(value, dtype):
    """100 tokens have distances up to 99; the bucket from 100 on is not finite."""
    c = Case(1, 2, 100, 100, 2, 1, 64, dtype, seed=34, buckets=2, far=3)
    c.plan.destroy()
    c.bucket_of = [0] * 100 + [1]
    c.plan = grawa.AttentionPlan(1, 2, 100, 2, 1, 64, dtype=dtype, buckets=2, bucket_of=c.bucket_of)
    want = c.want()
    assert not bool(want["dbias"][0][:, :, 1].any())
    c.bias[:, :, 1] = value
    check_gradients(c, want, ("dq", "dk", "dv", "dbias"))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [0, 40])
def test_gradients_of_keys_of_rows_that_see_nothing(window, dtype):
    """Every distance of head 0 hidden by the bias, gradients of its outputs no numbers: the keys that it shares with head 1 have head 1's gradients
    alone."""
    c = Case(1, 1, 150, 150, 2, 1, 64, dtype, seed=35, buckets=4, far=20, window=window)
    c.bias[:, 0] = -INF
    want = c.want()
    c.forward()
    torch.cuda.synchronize()
    for name in ("o", "lse"):
        ref.check(getattr(c, name), *want[name], name)
    c.do[:, :, :, 0] = NAN
    c.backward()
    torch.cuda.synchronize()
    for name in ("dq", "dk", "dv", "dbias"):
        ref.check(getattr(c, name), *want[name], name)
    c.plan.destroy()
