"""The layer norm of more rows than one launch may have threads for, against the same formula in float32 by torch."""
import pytest
import torch

from paper_2403_04206_amd import grawa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def norm_of_rows(K, T, d, dtype, seed, check, backward):
    """Calls the layer norm and compares the rows of `check`, ranges of rows, with 64 bits."""
    print("[case] norm", K, T, d, dtype, flush=True)
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.empty((K, T, d), device=DEV, dtype=dtype).normal_(generator=g)
    w, b = torch.rand((K, d), device=DEV, generator=g).to(dtype), torch.rand((K, d), device=DEV, generator=g).to(dtype)
    y, stats = torch.full_like(x, float("nan")), torch.full((K, T, 2), float("nan"), device=DEV)
    with grawa.SublayerPlan(K, T, d, dtype=dtype) as plan:
        plan.layer_norm(x, w, b, y, stats_out=stats)
        if backward:
            dy, dx = torch.empty_like(x).normal_(generator=g), torch.full_like(x, float("nan"))
            plan.layer_norm_backward(dy, x, w, stats, dx, torch.empty_like(w), torch.empty_like(b))
        torch.cuda.synchronize()
    assert not torch.isnan(stats).any() and not torch.isnan(y).any()
    for first, last in check:
        xs = x[:, first:last].double()
        var, mean = torch.var_mean(xs, 2, correction=0, keepdim=True)
        rstd = (var + 1e-5) ** -0.5
        h = (xs - mean) * rstd
        want = h * w[:, None].double() + b[:, None].double()
        # one rounding, 2^-8 of a value with bfloat16, and the float32 steps, which take 2^-18 of numbers of the row's size at the very most
        size, u = 1 + rstd * xs.abs().amax(2, keepdim=True), torch.finfo(dtype).eps / 2
        assert ((y[:, first:last].double() - want).abs() <= u * want.abs() + 2.0 ** -18 * size).all(), (first, last)
        if backward:
            dys = dy[:, first:last].double()
            a = dys * w[:, None].double()
            want = rstd * (a - a.mean(2, keepdim=True) - h * (a * h).mean(2, keepdim=True))
            bound = 2.0 ** -18 * rstd * size * size * (1 + dys.abs().amax(2, keepdim=True))
            assert ((dx[:, first:last].double() - want).abs() <= u * want.abs() + bound).all(), (first, last)
    if backward:
        assert not torch.isnan(dx).any()


@pytest.fixture(autouse=True)
def memory_back():
    yield
    torch.cuda.empty_cache()


def test_rows_of_a_wave():
    most = (1 << 31) // 64                       # rows of a launch, a wave each
    norm_of_rows(1, 2 * most + 301, 8, torch.bfloat16, 1, [(0, 500), (most - 200, most + 200), (2 * most - 200, 2 * most + 301)], True)


def test_rows_of_a_block():
    most = (1 << 31) // 1024                     # a block of 1024 threads each; these are the shortest rows of that kind
    norm_of_rows(1, most + 3, 8200, torch.bfloat16, 2, [(0, 40), (most - 20, most + 3)], False)
