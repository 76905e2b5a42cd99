"""Gradients of the bias beside many keys: sums of dS over pairs that nearly cancel, since dS of a row add up to 0."""
import pytest
import torch

import attention_reference as ref
from paper_2403_04206_amd import grawa
from test_gpu_attention import Case, generator

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mean", [0.0, 8.0])
@pytest.mark.parametrize("S,buckets,far,window,sinks", [(700, 2, 3, 0, 0), (877, 2, 3, 0, 1), (1500, 8, 100, 0, 0), (1500, 19, 77, 900, 70), (1300, 64, 900, 0, 0), (2100, 2, 402, 1000, 4)])
def test_only_the_result_is_rounded(S, buckets, far, window, sinks, mean, D):
    """bfloat16.  The outputs that the gradients start from are rounded, by 2^-8 of themselves at most, the same for all of a row's dS, and do not
    cancel in their sums: beside values with a mean of 8 they would be off by a multiple of 8 x 2^-9 = 1.6 %.  The result's own rounding is at most half
    a step for each element, 2^-8 of the root of the sum of squares.  Roundings to float32, of scores and exponentials, 2^-24 of numbers below 2^4 that
    differ from pair to pair and add up as roots of squares, as dS do, are 2^-20 of them, times 8 with such a mean: 2^-12 is allowed."""
    c = Case(2, 1, S, S, 4, 2, D, torch.bfloat16, seed=81, buckets=buckets, far=far, window=window, sinks=sinks)
    c.v.copy_(ref.make(c.v.shape, torch.bfloat16, generator(82), mean=mean))
    want = c.want()["dbias"][0]
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    off = float((c.dbias.double() - want).norm() / want.norm())
    print("[case]", off, flush=True)
    assert off <= 2.0 ** -8 + 2.0 ** -12
    c.plan.destroy()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("last,low", [(700, 0.0), (690, -20.0), (300, -20.0), (5, -30.0), (600, 0.0)])
def test_distances_of_no_pair_or_of_small_weight(last, low, D):
    """The last bucket begins at a distance that no pair has, a few pairs have, or whose bias leaves them little: 0, or what little they have."""
    c = Case(1, 2, 700, 700, 2, 1, D, torch.bfloat16, seed=83, buckets=2, far=3)
    c.plan.destroy()
    c.bucket_of = [0] * last + [1]
    c.plan = grawa.AttentionPlan(1, 2, 700, 2, 1, D, dtype=torch.bfloat16, buckets=2, bucket_of=c.bucket_of)
    c.bias[:, :, 1] += low
    want = c.want()
    assert last < 700 or not bool(want["dbias"][0][:, :, 1].any())
    c.check()
