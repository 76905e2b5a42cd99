"""Norms of heads whose squares float32 does not hold: rows of any size that the type has, ordinary ones beside them."""
import pytest
import torch

import attention_reference as ref
from paper_2403_04206_amd import grawa

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,R,interleaved", [(64, 64, False), (128, 40, True), (72, 20, False)])
@pytest.mark.parametrize("eps", [1e-6, 0.0, 1e-36])
@pytest.mark.parametrize("size", [1e-37, 1e-30, 1e-21, 1e-17, 1.0, 1e17, 1e19, 1e21, 1e30, 6e37])
def test_rows_of_any_size(size, eps, D, R, interleaved, dtype):
    """Every third row is of `size`, the others of size one.  The bounds are those of ordinary rows: factors of two are exact, and gradients
    below 1e-38 are 0."""
    gen = torch.Generator(device="cuda").manual_seed(71)
    K, N, S, H, G = 2, 1, 41, 3, 1
    x = [ref.make((K, N, S, h, D), torch.float32, gen) for h in (H, G)]
    for t in x:
        t[:, :, ::3] *= size
    x, dy = [t.to(dtype) for t in x], [ref.make((K, N, S, h, D), dtype, gen) for h in (H, G)]
    w = [ref.make((K, D), dtype, gen, 0.2, 1.0) for _ in range(2)]
    y, dx, dw = [torch.full_like(t, 7.0) for t in x], [torch.full_like(t, 7.0) for t in x], [torch.full_like(t, 7.0) for t in w]
    frequencies = grawa.rotary_frequencies(R)
    with grawa.AttentionPlan(K, N, S, H, G, D, dtype=dtype, frequencies=frequencies, interleaved=interleaved) as plan:
        plan.head_norm(*x, *w, *y, eps=eps)
        plan.head_norm_backward(*dy, *x, *w, *dx, *dw, eps=eps)
        over, back, dw2 = [t.clone() for t in x], [t.clone() for t in dy], [torch.full_like(t, 7.0) for t in w]
        plan.head_norm_backward(*back, *x, *w, *back, *dw2, eps=eps)                # in place
        plan.head_norm(*over, *w, *over, eps=eps)
        torch.cuda.synchronize()
    for a, b in zip(y + dx + dw, over + back + dw2):
        assert torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0))
    angle = ref.angles(torch.zeros((K, N), device="cuda"), S, frequencies)
    limit = torch.finfo(dtype).max
    for i in range(2):
        ref.check(y[i], *ref.head_norm(x[i], w[i], eps, angle, interleaved, dtype), "y")
        want, dweight, off, dweight_off = ref.head_norm_backward(dy[i], x[i], w[i], eps, angle, interleaved, dtype)
        held = want.abs() + off < limit                                          # dy / x may be more than the type holds
        ref.check(dx[i][held], want[held], off[held], "dx")
        ref.check(dw[i], dweight, dweight_off, "dw")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("value", [0.0, float("inf"), float("nan")])
def test_rows_without_a_norm(value, dtype):
    """Zeros beside an eps of 0, infinities and no numbers: what 0 / 0 and infinity / infinity are; rows beside them are as without."""
    gen = torch.Generator(device="cuda").manual_seed(72)
    x = [ref.make((1, 1, 20, h, 64), dtype, gen) for h in (2, 1)]
    w = [ref.make((1, 64), dtype, gen, 0.2, 1.0) for _ in range(2)]
    y = [torch.full_like(t, 7.0) for t in x]
    want = [ref.head_norm(t, v, 0.0, ref.angles(torch.zeros((1, 1), device="cuda"), 20, []), False, dtype) for t, v in zip(x, w)]
    for t in x:
        t[:, :, 5] = value
    with grawa.AttentionPlan(1, 1, 20, 2, 1, 64, dtype=dtype) as plan:
        plan.head_norm(*x, *w, *y, eps=0.0)
        torch.cuda.synchronize()
    other = torch.arange(20, device="cuda") != 5
    for t, (n, off) in zip(y, want):
        assert bool(t[:, :, 5].isnan().all())
        ref.check(t[:, :, other], n[:, :, other], off[:, :, other], "y")
