"""The gated feed-forward block at the ends of its numbers: gates that are infinite or far out, values whose bits are all in use, infinities."""
import pytest
import torch

from paper_2403_04206_amd import grawa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32


def tensor(values, dtype):
    return torch.tensor(values, device=DEV, dtype=torch.float64).to(dtype)


def forward_and_back(x, wg, wu, wd, dy, act):
    """One worker's y, dx, dWg, dWu, dWd: x, dy [T, d], wg, wu [f, d], wd [d, f]."""
    (T, d), f, dtype = x.shape, wg.shape[0], x.dtype
    x, wg, wu, wd, dy = (t.unsqueeze(0).contiguous() for t in (x, wg, wu, wd, dy))
    y, dx, dwg, dwu, dwd = (torch.full_like(t, 7.0) for t in (x, x, wg, wu, wd))
    with grawa.SublayerPlan(1, T, d, f, dtype=dtype, activation=act) as plan:
        save = torch.empty(plan.save_bytes(), dtype=torch.uint8, device=DEV)
        plan.ffn(x, wg, wu, wd, y, save=save)
        plan.ffn_backward(dy, x, wg, wu, wd, save, dx, dwg, dwu, dwd)
        torch.cuda.synchronize()
    return tuple(t[0].double() for t in (y, dx, dwg, dwu, dwd))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T", [3, 40, 140])
def test_relu_closes_a_gate_whatever_stands_beside_it(dtype, T):
    print("[case] relu", dtype, T, flush=True)
    big = 2.0 ** 70                                    # its square is no float32
    x, one = tensor([[big]] * T, dtype), tensor([[1.0]], dtype)
    # a gate of -infinity: relu gives 0, and so do the block and its gradients
    y, dx, dwg, dwu, dwd = forward_and_back(x, -one * big, one / big, one, torch.ones_like(x), "relu")
    for t in (y, dx, dwg, dwu, dwd):
        assert (t == 0).all()
    # gates of -1: what comes back through them is 0 beside an infinite up, and under an infinite gradient
    y, dx, dwg, dwu, dwd = forward_and_back(x, -one / big, one * big, one, torch.ones_like(x), "relu")
    assert (dwg == 0).all()
    y, dx, dwg, dwu, dwd = forward_and_back(x, -one / big, one / big, one * big, x, "relu")
    assert (y == 0).all() and (dwg == 0).all()
    # a gate that is no number is none afterwards, an infinite one stays
    nan = x.clone()
    nan[T - 1, 0] = float("nan")
    y = forward_and_back(nan, one / big, one / big, one, torch.ones_like(x), "relu")[0]
    assert torch.isnan(y[T - 1]).all() and (y[:T - 1] == 1).all()
    y = forward_and_back(x, one * big, one / big, one, torch.ones_like(x), "relu")[0]
    if dtype is BF or T <= 64:
        assert (y == float("inf")).all()
    else:                                              # terms of a float32 that are 0 make a NaN of it
        assert not torch.isfinite(y).any()


@pytest.mark.parametrize("T", [3, 200])
def test_float32_products_of_numbers_with_all_their_bits(T):
    """One product after the other, (x wg) (x wu) wd with positive numbers, against 64 bits.  Each of the three products may lack 2^-24 of
    itself, and its terms are added with an error of 2^-23, whichever way a sum is rounded; the gate times the up and the result are rounded
    once more, 2^-24 each: 3 * 3 + 2 times 2^-24, and one for what is of second order."""
    print("[case] bits", T, flush=True)
    g = torch.Generator().manual_seed(3)
    worst = [1 + 2.0 ** -7 - 2.0 ** -23, 1 + 2.0 ** -8 - 2.0 ** -23, 1 + 2.0 ** -7 + 2.0 ** -15 - 2.0 ** -23, 2 - 2.0 ** -23]
    for weights in [[w] * 3 for w in worst] + (1 + torch.rand((20, 3), generator=g)).tolist():
        x = (1 + torch.rand((T, 1), generator=g)).to(DEV)
        x[0, 0], x[-1, 0] = weights[0], worst[0]
        wg, wu, wd = (tensor([[w]], F) for w in weights)
        y, dx, dwg, dwu, dwd = forward_and_back(x, wg, wu, wd, torch.ones_like(x), "relu")
        x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
        want = (x * wg) * (x * wu) * wd
        off = ((y - want) / want).abs().max().item() * 2.0 ** 24
        assert off <= 12, (weights, off)
        # dx = 2 x wg wu wd: three products one after the other in each of two that are added, a rounding more
        off = ((dx - 2 * x * wg * wu * wd) / (2 * x * wg * wu * wd)).abs().max().item() * 2.0 ** 24
        assert off <= 14, (weights, off)


@pytest.mark.parametrize("T", [3, 40, 140])
def test_gate_and_up_go_to_the_backward_pass_rounded_to_nearest(T):
    """bfloat16.  An up (a gate) a little above the middle between two bfloat16 numbers, by less than one part in 2^15: dG (dU) is the up (the gate) rounded
    to bfloat16 here, the upper of the two."""
    print("[case] kept", T, flush=True)
    x, dy = torch.zeros((T, 3), device=DEV, dtype=BF), torch.zeros((T, 3), device=DEV, dtype=BF)
    x[T - 1] = 1
    dy[T - 1, 0] = 1
    one, wd = tensor([[1.0, 0.0, 0.0]], BF), tensor([[1.0], [0.0], [0.0]], BF)
    for sign, at in ((1, 0), (-1, 0), (1, 1)):
        odd = tensor([[1.0, 2.0 ** -8, 29 * 2.0 ** -20]], BF) * sign
        y, dx, dwg, dwu, dwd = forward_and_back(x, odd if at else one, one if at else odd, wd, dy, "relu")
        got = dwu if at else dwg
        assert (got == sign * (1 + 2.0 ** -7)).all(), (sign, at, got)


@pytest.mark.parametrize("T", [30, 481])
@pytest.mark.parametrize("act,low", [("gelu", -12.5), ("silu", -80.0)])
def test_activations_far_out(act, low, T):
    """bfloat16.  The activation of x and its derivative, which the block gives as they are with an up of 1 and matrices of 0 and 1, against 64 bits: one
    rounding to bfloat16, 2^-8, and 2^-11 for the function; the derivative's two terms may cancel, with 2^-18 of them left."""
    print("[case] tails", act, T, flush=True)
    z = torch.linspace(low, 12.5, T, device=DEV, dtype=torch.float64).to(BF)
    x = torch.stack((z, torch.ones_like(z)), 1)
    dy = torch.zeros_like(x)
    dy[:, 0] = 1
    y, dx, _, _, _ = forward_and_back(x, tensor([[1.0, 0.0]], BF), tensor([[0.0, 1.0]], BF), tensor([[1.0], [0.0]], BF), dy, act)
    z = z.double()
    if act == "gelu":
        first, second = 0.5 * torch.erfc(-z / 2 ** 0.5), z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    else:
        first = torch.sigmoid(z)
        second = z * first * torch.sigmoid(-z)
    for what, got, want, slack in (("value", y[:, 0], z * first, 0), ("derivative", dx[:, 0], first + second, 2.0 ** -18 * (first + second.abs()))):
        over = (got - want).abs() - (2.0 ** -8 + 2.0 ** -11) * want.abs() - slack
        i = over.argmax().item()
        assert over[i] <= 0, (what, z[i].item(), got[i].item(), want[i].item())


@pytest.mark.parametrize("T", [30, 481])
@pytest.mark.parametrize("act,low", [("gelu", -12.5), ("silu", -80.0)])
def test_activations_far_out_in_float32(act, low, T):
    """The same in float32, with numbers that are exact in one term: 2^-19 for the functions and the sums, and what roundings of the functions' arguments, 2^-24
    each, come to: z^2 2^-23 (silu: |z| 2^-23) of each term."""
    print("[case] tails in float32", act, T, flush=True)
    z = torch.linspace(low, 12.5, T, device=DEV, dtype=torch.float64).to(BF).to(F)
    x = torch.stack((z, torch.ones_like(z)), 1)
    dy = torch.zeros_like(x)
    dy[:, 0] = 1
    y, dx, _, _, _ = forward_and_back(x, tensor([[1.0, 0.0]], F), tensor([[0.0, 1.0]], F), tensor([[1.0], [0.0]], F), dy, act)
    z = z.double()
    if act == "gelu":
        first, second = 0.5 * torch.erfc(-z / 2 ** 0.5), z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
        share = 2.0 ** -19 + z * z * 2.0 ** -23
    else:
        first = torch.sigmoid(z)
        second = z * first * torch.sigmoid(-z)
        share = 2.0 ** -19 + z.abs() * 2.0 ** -23
    for what, got, want, size in (("value", y[:, 0], z * first, (z * first).abs()), ("derivative", dx[:, 0], first + second, first + second.abs())):
        over = (got - want).abs() - share * size
        i = over.argmax().item()
        assert over[i] <= 0, (what, z[i].item(), got[i].item(), want[i].item())
