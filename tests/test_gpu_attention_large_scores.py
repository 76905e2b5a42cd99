"""Scores that are large and equal, or large and a little apart: the weights of keys do not depend on which block or wave has them.

All scores here are exact: queries and keys have one or two elements that are not 0, whose products and sums are whole multiples of a
power of two below 2^24 of them.  Keys of equal scores then have equal weights, exactly; keys a number of units apart have weights
exp(units) with an exponent that takes three roundings of a number below 4 (the unit's, the product's, the exponential's), 16 E is
taken.  Sums as in attention_reference: (Sk / 16 + 64) E, and with bfloat16 half a step for each exponential that is not a power of two
and for the result."""
import math

import pytest
import torch

import attention_reference as ref
from paper_2403_04206_amd import grawa
from test_gpu_attention import Case, generator

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


class Keys:
    """Queries and keys whose score is `base` + unit[j]."""

    def __init__(self, Sq, Sk, length, H, G, D, dtype, base, units, scale, seed, window=0, sinks=0, bias=None):
        gen = generator(seed)
        self.dims, self.dtype, self.kinds = (Sq, Sk, length, H, G, D), dtype, dict(window=window, sinks=sinks)
        self.q, self.k = torch.zeros((1, 1, Sq, H, D), device="cuda", dtype=dtype), torch.zeros((1, 1, Sk, G, D), device="cuda", dtype=dtype)
        root = 2.0 ** (math.log2(base / scale) // 2) if base else 0.0
        self.q[..., 0], self.k[..., 0] = root, base / scale / root if base else 0.0
        self.q[..., 1], self.k[..., 1] = 1.0 / scale, units.to(dtype)[:, None] if torch.is_tensor(units) else units
        self.units = units.double() if torch.is_tensor(units) else torch.full((Sk,), float(units), device="cuda", dtype=torch.float64)
        self.base = base
        self.v = ref.make((1, 1, Sk, G, D), dtype, gen)
        self.o, self.lse = torch.full_like(self.q, 7.0), torch.full((1, 1, H, Sq), 7.0, device="cuda")
        self.bias, more = None, {}
        if bias is not None:
            self.bias, self.base = torch.full((1, H, 2), bias, device="cuda", dtype=dtype), base + bias
            more = dict(buckets=2, bucket_of=[0, 1])
        self.plan = grawa.AttentionPlan(1, 1, Sk, H, G, D, dtype=dtype, scale=scale, **self.kinds, **more)

    def check(self, equal):
        Sq, Sk, length, H, G, D = self.dims
        places = {n: torch.full((1, 1), x, dtype=torch.int32, device="cuda") for n, x in (("lengths", length), ("starts", length - Sq))}
        self.plan.attention(self.q, self.k, self.v, self.o, lse_out=self.lse, bias=self.bias, **places)
        torch.cuda.synchronize()
        seen = ref.visible(length - Sq, length, Sq, Sk, self.kinds["window"], self.kinds["sinks"], "cuda")[0]
        P = torch.where(seen, torch.exp(self.units), 0.0)
        total = P.sum(1, keepdim=True)
        P = P / total
        U = ref.half_step(self.dtype)
        near = (Sk / 16 + 64) * ref.E + (0.0 if equal else 16 * ref.E + (U if self.dtype is torch.bfloat16 else 0.0))
        for h in range(H):
            V = self.v[0, 0, :, h // (H // G)].double()
            o = P @ V
            ref.check(self.o[0, 0, :, h], o, (P @ V.abs()) * near + U * o.abs() + 1e-38, "o")
            lse = self.base + torch.log(total[:, 0])
            ref.check(self.lse[0, 0, h], lse, near + 8 * ref.E * lse.abs(), "lse")    # scaled, its logarithm added, in another unit and back
        self.plan.destroy()


# by keys: a token or a few; by queries: more rows than that.  Lengths whose tiles no number of blocks divides, and room that blocks share
# without a key for most of them; the last two of each: one block has all keys
FORMS = [(1, 5000, 5000, 1, 1, 64), (3, 5000, 4500, 4, 2, 128), (1, 5000, 300, 2, 1, 64), (1, 250, 250, 1, 1, 64), (5, 255, 249, 6, 2, 128),
         (70, 5000, 4200, 1, 1, 64), (70, 5000, 4200, 2, 1, 128), (130, 5000, 3333, 1, 1, 72), (70, 190, 190, 1, 1, 64), (70, 200, 170, 1, 1, 128)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq,Sk,length,H,G,D", FORMS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (2900, 3)])
@pytest.mark.parametrize("base", [2.0 ** 8, 2.0 ** 20, 2.0 ** 25, 2.0 ** 30, -2.0 ** 29])
def test_equal_scores(base, window, sinks, Sq, Sk, length, H, G, D, dtype):
    c = Keys(Sq, Sk, length, H, G, D, dtype, abs(base), 0.0, 2.0 ** -3, 41, window=window, sinks=sinks)
    if base < 0:
        c.k, c.base = -c.k, base
    c.check(True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq,Sk,length,H,G,D", FORMS)
@pytest.mark.parametrize("bias", [2.0 ** 20, -2.0 ** 26, 2.0 ** 30])
def test_equal_scores_by_a_large_bias(bias, Sq, Sk, length, H, G, D, dtype):
    Keys(Sq, Sk, length, H, G, D, dtype, 0.0, 0.0, 2.0 ** -3, 42, bias=bias).check(True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq,Sk,length,H,G,D", FORMS)
@pytest.mark.parametrize("where", ["mixed", "first", "last"])
@pytest.mark.parametrize("base", [0.0, 2.0 ** 15, 2.0 ** 19, 2.0 ** 21, 2.0 ** 23])
def test_scores_a_little_apart(base, where, Sq, Sk, length, H, G, D, dtype):
    """Keys of 0, 1 and 2 units; the largest ones everywhere, in the first keys alone or in the last ones of the sequence alone."""
    gen = generator(43)
    units = torch.randint(0, 3, (Sk,), device="cuda", generator=gen).float()
    if where != "mixed":
        j = torch.arange(Sk, device="cuda")
        units = torch.where(j < 40 if where == "first" else j >= length - 40, 2.0, units.clamp(max=1.0))
    Keys(Sq, Sk, length, H, G, D, dtype, base, units, 2.0 ** -7, 44).check(False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("S,D,window", [(200, 64, 1), (200, 128, 0), (700, 64, 0), (700, 128, 300), (33, 64, 0)])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("size", [2.0 ** 24, 2.0 ** 30])
def test_gradients_beside_large_scores(size, biased, S, D, window, dtype):
    """Scores of `size` leave the gradients no digits, but exponentials stay about 1 at most and what is formed of them is no more than that
    gives: |dv| <= sum |do|, |dS| <= |dP| + |delta|, and |delta| <= sum |dP| or |do||o|.  Exponents are taken above lse where that is beyond
    2^20 in units of log2; for the rows of smaller scores lse is off by the roundings of the maximum, of the logarithm added, to
    natural logarithms and back, and by the constants' product, 0.2 of one: 4.2 E 2^20 = 0.27, a factor of 2^0.27.  Other roundings: a few
    of the type's half steps, and of the sums (S + 2 D) E."""
    c = Case(1, 1, S, S, 2, 1, D, dtype, seed=45, window=window, **(dict(buckets=2, far=3) if biased else {}))
    c.q.mul_(size)
    if biased:
        c.q.mul_(2.0 ** -30)
        c.bias.mul_(size)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    q, k, v, do, o = (t[0, 0].double() for t in (c.q, c.k, c.v, c.do, c.o))
    seen = ref.visible(0, S, S, S, window, 0, "cuda")[0]
    more = 2.0 ** 0.27 * (1 + 4 * ref.half_step(dtype) + (S + 2 * D) * ref.E)
    dv, dk = torch.zeros_like(v[:, 0]), torch.zeros_like(v[:, 0])
    for h in range(2):
        dP = torch.where(seen, do[:, h].abs() @ v[:, 0].abs().T, 0.0)
        delta = torch.maximum(dP.sum(1, keepdim=True), (do[:, h] * o[:, h]).abs().sum(1, keepdim=True))
        dS = torch.where(seen, dP + delta, 0.0)
        dv += seen.double().T @ do[:, h].abs()
        dk += dS.T @ q[:, h].abs() * D ** -0.5
        assert bool((c.dq[0, 0, :, h].double().abs() <= more * (dS @ k[:, 0].abs()) * D ** -0.5).all()), "dq"
        if biased:
            assert bool((c.dbias[0, h].double().abs() <= more * dS.sum()).all()), "dbias"
    assert bool((c.dv[0, 0, :, 0].double().abs() <= more * dv).all()), "dv"
    assert bool((c.dk[0, 0, :, 0].double().abs() <= more * dk).all()), "dk"
    c.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("base", [2.0 ** 21, -2.0 ** 23])
def test_gradients_where_scores_and_bias_cancel(base, D, dtype):
    """Queries and keys of a large score and a bias that takes all but 0, 1 or 2 units of it away again: sums and exponentials are ordinary,
    and dv = P^T do has its digits.  lse is below 16 then, and the 4.2 roundings of it in units of log2 (23) and of the exponent are 128 E."""
    gen = generator(46)
    S = 190
    c = Keys(S, S, S, 2, 1, D, dtype, abs(base), torch.randint(0, 3, (S,), device="cuda", generator=gen).float(), 2.0 ** -7, 47, bias=-base)
    if base < 0:
        c.k[..., 0].neg_()
    do, dq, dk, dv = ref.make(c.q.shape, dtype, gen), torch.empty_like(c.q), torch.empty_like(c.k), torch.empty_like(c.v)
    dbias = torch.empty_like(c.bias)
    c.plan.attention(c.q, c.k, c.v, c.o, lse_out=c.lse, bias=c.bias)
    c.plan.attention_backward(do, c.q, c.k, c.v, c.o, c.lse, dq, dk, dv, bias=c.bias, dbias=dbias)
    torch.cuda.synchronize()
    assert bool((c.lse.abs() < 16).all())
    seen = ref.visible(0, S, S, S, 0, 0, "cuda")[0]
    P = torch.where(seen, torch.exp(c.units), 0.0)
    P = P / P.sum(1, keepdim=True)
    U, near = ref.half_step(dtype), (S / 8 + 64 + 128) * ref.E + (ref.half_step(dtype) if dtype is torch.bfloat16 else 0.0)
    want = sum(P.T @ do[0, 0, :, h].double() for h in range(2))
    ref.check(dv[0, 0, :, 0], want, near * sum(P.T @ do[0, 0, :, h].double().abs() for h in range(2)) + U * want.abs() + 1e-38, "dv")
    c.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq", [1, 5, 700])
@pytest.mark.parametrize("size", [2.0 ** -80, 2.0 ** 87])
def test_values_of_any_size(size, Sq, dtype):
    """Values of up to 2^90 beside scores that grow by a few from token to token: sums before the division hold them."""
    c = Case(1, 1, Sq, 700, 2, 1, 64, dtype, seed=48)
    c.k[..., 0] = (torch.arange(700, device="cuda", dtype=torch.float32) / 16)[:, None].to(dtype)
    c.q[..., 0] = 24.0
    c.v.mul_(size)
    want = c.want(False)
    c.forward()
    torch.cuda.synchronize()
    assert bool(c.o.isfinite().all())
    for name, (value, off) in want.items():
        ref.check(getattr(c, name), value, off, name)
    c.plan.destroy()
