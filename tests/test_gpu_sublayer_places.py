"""The gated feed-forward block where its matrices do not stand alike: each of Wg, Wu and Wd by itself off 16 bytes, by its place or by the
distance between the workers, at widths whose copies have another pitch than the matrices."""
import pytest
import torch

import sublayer_reference as ref
from paper_2403_04206_amd import grawa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def normal(seed, *shape, scale=1.0):
    return torch.randn(shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).mul_(scale)


def matrix(seed, K, rows, columns, scale, first, gap):
    """K matrices, `first` elements from an allocation's start and `gap` elements apart; NaN around them."""
    n = rows * columns
    room = torch.full((first + K * (n + gap),), float("nan"), device=DEV, dtype=BF)
    m = torch.as_strided(room, (K, rows, columns), (n + gap, columns, 1), first)
    m.copy_(normal(seed, K, rows, columns, scale=scale))
    return m


@pytest.mark.parametrize("K,T,d,f", [(1, 40, 72, 136), (1, 300, 1000, 264), (3, 40, 72, 136), (2, 70, 1000, 200), (2, 33, 72, 90), (3, 5, 1000, 72)])
@pytest.mark.parametrize("odd", ["wg", "wu", "wd", "wg wd"])
@pytest.mark.parametrize("how", ["place", "stride"])
def test_one_matrix_off_16_bytes(K, T, d, f, odd, how):
    print("[case]", K, T, d, f, odd, how, flush=True)
    at = {n: ((3, 8) if how == "place" else (8, 5)) if n in odd.split() else (8, 16) for n in ("wg", "wu", "wd")}
    wg, wu = matrix(1, K, f, d, d ** -0.5, *at["wg"]), matrix(2, K, f, d, d ** -0.5, *at["wu"])
    wd = matrix(3, K, d, f, f ** -0.5, *at["wd"])
    x, dy = normal(4, K, T, d).to(BF), normal(5, K, T, d).to(BF)
    y, dx, eval_y = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    grads = [torch.full((K,) + tuple(w.shape[1:]), 7.0, device=DEV, dtype=BF) for w in (wg, wu, wd)]
    with grawa.SublayerPlan(K, T, d, f, dtype=BF) as plan:
        save = torch.full((plan.save_bytes(T),), 0xff, dtype=torch.uint8, device=DEV)
        plan.ffn(x, wg, wu, wd, y, save=save)
        plan.ffn_backward(dy, x, wg, wu, wd, save, dx, *grads)
        plan.ffn(x, wg, wu, wd, eval_y)
        torch.cuda.synchronize()
    assert torch.equal(y, eval_y)
    for k in range(K):
        out, low = ref.ffn(x[k].double(), wg[k].double(), wu[k].double(), wd[k].double(), dy[k].double(), "silu", BF)
        for n, got in (("y", y), ("dx", dx), ("dwg", grads[0]), ("dwu", grads[1]), ("dwd", grads[2])):
            ref.assert_within(got[k], out[n], low[n], "worker %d %s" % (k, n), BF)
