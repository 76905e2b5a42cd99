"""A bias that hides keys: minus infinity, the type's lowest number and everything below -2^100 alike; a bias above it hides nothing."""
import math

import pytest
import torch

import attention_reference as ref
from test_gpu_attention import Case

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
INF = math.inf
# queries, keys: a block's, a wave's of a few, shared by blocks
FORMS = [(100, 100), (600, 600), (1, 90), (1, 5000), (70, 4000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq,Sk", FORMS)
@pytest.mark.parametrize("hidden", ["infinity", "lowest", "below"])
def test_rows_whose_keys_are_all_hidden_are_0(hidden, Sq, Sk, dtype):
    value = {"infinity": -INF, "lowest": torch.finfo(dtype).min, "below": -1.5 * 2.0 ** 100}[hidden]
    c = Case(1, 2, Sq, Sk, 2, 1, 64, dtype, seed=61, buckets=4, far=20)
    c.bias[:, 0] = -INF
    want = c.want()
    c.bias[:, 0] = value
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    assert not bool(c.o[:, :, :, 0].any()) and bool((c.lse[:, :, 0] == -INF).all())
    assert not bool(c.dq[:, :, :, 0].any()) and not bool(c.dbias[:, 0].any())
    for name, (exact, off) in want.items():
        ref.check(getattr(c, name), exact, off, name)
    c.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq,Sk", FORMS)
@pytest.mark.parametrize("value", [-2.0 ** 100, -2.0 ** 99])
def test_a_bias_of_minus_two_to_the_hundred_hides_nothing(value, Sq, Sk, dtype):
    """Beside it float32 has nothing left of q . k: all keys are equal.  Their weights are 1 before the sum, (Sk / 16 + 64) E off with it."""
    c = Case(1, 1, Sq, Sk, 2, 1, 64, dtype, seed=62, buckets=4, far=20)
    c.bias[:, 0] = value
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    seen = ref.visible(Sk - Sq, Sk, Sq, Sk, 0, 0, "cuda")[0].double()
    P, V = seen / seen.sum(1, keepdim=True), c.v[0, 0, :, 0].double()
    o = P @ V
    ref.check(c.o[0, 0, :, 0], o, (P @ V.abs()) * (Sk / 16 + 64) * ref.E + ref.half_step(dtype) * o.abs() + 1e-38, "o")
    assert bool(((c.lse[0, 0, 0].double() - value).abs() <= 8 * ref.E * abs(value)).all())
    for t in (c.dq, c.dk, c.dv, c.dbias):
        assert bool(t.isfinite().all())
    c.plan.destroy()
