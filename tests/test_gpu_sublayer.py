"""Layer norm, gated feed-forward block and dropout of K workers against the same formulas in 64 bits: widths and token counts
around the tile edges, parameters at odd places of the flat rows, strided and shared activations, gradients added to what is
there, gaps that hold NaN, no tokens, other streams, captured graphs."""
import numpy as np
import pytest
import torch

import sublayer_reference as ref
from paper_2403_04206_amd import grawa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
NAN = float("nan")


def say(*a):
    print("[case]", *a, flush=True)


def rows_in(values, layout):
    """The [K, T, d] values inside an array whose other elements are NaN."""
    K, T, d = values.shape
    if layout == "plain":
        return values.clone()
    if layout == "padded":          # gaps between rows and workers, rows at odd elements
        room = torch.full((K, T + 1, d + 3), NAN, device=DEV, dtype=values.dtype)
        v = room[:, :T, 1:1 + d]
    elif layout == "padded16":      # gaps of whole 16 bytes
        room = torch.full((K, T + 1, d + 16), NAN, device=DEV, dtype=values.dtype)
        v = room[:, :T, 8:8 + d]
    elif layout == "tokens_first":
        room = torch.full((T, K, d), NAN, device=DEV, dtype=values.dtype)
        v = room.permute(1, 0, 2)
    v.copy_(values)
    return v


class Params:
    """Vectors and matrices of K workers in flat rows that are NaN elsewhere."""

    def __init__(self, K, d, f, dtype, shift, fill=None):
        self.shapes = {"weight": (d,), "bias": (d,), "wg": (f, d), "wu": (f, d), "wd": (d, f)}
        P = shift + 2 * d + 3 * d * f + 5
        self.rows = torch.full((K, P), NAN, device=DEV, dtype=dtype)
        self.used = torch.zeros((K, P), device=DEV, dtype=torch.bool)
        self.v, at = {}, shift
        for n, s in self.shapes.items():
            c = int(np.prod(s))
            if c:
                self.v[n] = self.rows[:, at:at + c].view((K,) + s)
                self.used[:, at:at + c] = True
                if fill is not None:
                    self.v[n].fill_(fill)
            at += c

    def __getitem__(self, n):
        return self.v[n]

    def untouched(self):
        return torch.isnan(self.rows[~self.used]).all().item()


def make(seed, *shape, dtype=F, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, device=DEV, generator=g) * scale).to(dtype)


def fill_params(p, seed, d, f):
    for i, n in enumerate(p.v):
        s = {"weight": 0.3, "bias": 0.3, "wg": d ** -0.5, "wu": d ** -0.5, "wd": max(f, 1) ** -0.5}[n]
        p[n].copy_(make(seed + i, *p[n].shape, scale=s).to(p.rows.dtype) + (1 if n == "weight" else 0))


# -- the gated feed-forward block ---------------------------------------------------

def run_ffn(seed, K, T, d, f, dtype, act="silu", shift=0, layout="plain", accumulate=False, plan_T=None, shared=False):
    say("ffn", K, T, d, f, dtype, act, "shift", shift, layout, "accumulate", accumulate)
    p, gr = Params(K, d, f, dtype, shift), Params(K, d, f, dtype, shift)
    fill_params(p, seed, d, f)
    before = {}
    if accumulate:
        for i, n in enumerate(gr.v):
            gr[n].copy_(make(seed + 40 + i, *gr[n].shape, scale=0.5).to(dtype))
            before[n] = gr[n].double()
    x = make(seed + 20, K, T, d, dtype=dtype)
    if shared:
        x = x[:1].expand(K, T, d)
        xv = x
    else:
        xv = rows_in(x, layout)
    dyv = rows_in(make(seed + 21, K, T, d, dtype=dtype), layout)
    y, dx = rows_in(torch.zeros((K, T, d), device=DEV, dtype=dtype), layout), rows_in(torch.zeros((K, T, d), device=DEV, dtype=dtype), layout)
    eval_y = torch.empty_like(y)
    with grawa.SublayerPlan(K, plan_T or T, d, f, dtype=dtype, activation=act) as plan:
        save = torch.full((plan.save_bytes(T),), 0xff, dtype=torch.uint8, device=DEV)
        plan.ffn(xv, p["wg"], p["wu"], p["wd"], y, save=save)
        plan.ffn_backward(dyv, xv, p["wg"], p["wu"], p["wd"], save, dx, gr["wg"], gr["wu"], gr["wd"], accumulate=accumulate)
        plan.ffn(xv, p["wg"], p["wu"], p["wd"], eval_y)
        torch.cuda.synchronize()
    assert gr.untouched()
    for k in range(K):
        out, low = ref.ffn(xv[k].double(), p["wg"][k].double(), p["wu"][k].double(), p["wd"][k].double(), dyv[k].double(), act, dtype)
        got = {"y": y[k], "dx": dx[k], "dwg": gr["wg"][k], "dwu": gr["wu"][k], "dwd": gr["wd"][k]}
        for n in got:
            want, bound = out[n], low[n]
            if accumulate and n in ("dwg", "dwu", "dwd"):
                old = before[n[1:]][k]
                want, bound = want + old, bound + ref.U[dtype] * (want + old).abs() + 2.0 ** -23 * old.abs()
            ref.assert_within(got[n], want, bound, "worker %d %s" % (k, n), dtype)
        ref.assert_within(eval_y[k], out["y"], low["y"], "worker %d y without a backward pass" % k, dtype)
    return y, dx, gr


SIZES = [(1, 1, 1, 1), (2, 1, 8, 8), (3, 5, 7, 9), (2, 64, 64, 64), (2, 65, 72, 136), (1, 129, 257, 130), (3, 16, 200, 72), (2, 17, 1000, 96),
         (4, 300, 96, 200), (1, 33, 1030, 515), (1, 48, 2048, 80), (2, 130, 136, 1032)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("size", SIZES)
def test_ffn_sizes(size, dtype):
    run_ffn(100, *size, dtype)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_ffn_activations(act, dtype):
    run_ffn(200, 2, 140, 80, 144, dtype, act=act, shift=3)
    run_ffn(210, 2, 3, 80, 144, dtype, act=act)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("layout,shift", [("padded", 1), ("padded16", 8), ("padded16", 5), ("tokens_first", 0), ("plain", 7)])
def test_ffn_layouts(layout, shift, dtype):
    run_ffn(300, 3, 70, 72, 80, dtype, shift=shift, layout=layout)
    run_ffn(310, 3, 6, 72, 80, dtype, shift=shift, layout=layout)


@pytest.mark.parametrize("dtype", [BF, F])
def test_ffn_accumulates(dtype):
    run_ffn(400, 2, 150, 72, 100, dtype, accumulate=True)
    run_ffn(410, 2, 150, 72, 104, dtype, accumulate=True, shift=8)


def test_ffn_shared_batch_and_larger_plan():
    run_ffn(500, 3, 70, 64, 72, BF, shared=True, plan_T=200)


def test_ffn_large_tiles():
    run_ffn(600, 32, 530, 520, 530, BF, shift=8)


@pytest.mark.parametrize("K,T,d,f,dtype", [(1, 40, 6704, 6712, BF),      # matrices that no cache holds, more tiles than CUs
                                           (17, 70, 1000, 1032, BF), (1, 70, 4104, 4099, F)])
def test_ffn_large_matrices(K, T, d, f, dtype):
    run_ffn(700, K, T, d, f, dtype)
    torch.cuda.empty_cache()
    run_ffn(610, 16, 600, 264, 1056, F, act="gelu")


def test_ffn_no_tokens():
    K, d, f = 2, 24, 40
    for dtype in (BF, F):
        p, gr = Params(K, d, f, dtype, 0), Params(K, d, f, dtype, 0, fill=2.0)
        fill_params(p, 1, d, f)
        none = torch.empty((K, 0, d), device=DEV, dtype=dtype)
        save = torch.empty(0, dtype=torch.uint8, device=DEV)
        with grawa.SublayerPlan(K, 4, d, f, dtype=dtype) as plan:
            args = (none, none, p["wg"], p["wu"], p["wd"], save, none, gr["wg"], gr["wu"], gr["wd"])
            plan.ffn(none, p["wg"], p["wu"], p["wd"], none, save=save)
            plan.ffn_backward(*args, accumulate=True)
            torch.cuda.synchronize()
            assert all((gr[n] == 2).all().item() for n in ("wg", "wu", "wd"))
            plan.ffn_backward(*args)
            torch.cuda.synchronize()
            assert all((gr[n] == 0).all().item() for n in ("wg", "wu", "wd")) and (gr["weight"] == 2).all().item()
            assert gr.untouched()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T", [3, 140])
def test_ffn_nan_stays_in_its_row(dtype, T):
    K, d, f = 2, 72, 136
    p = Params(K, d, f, dtype, 0)
    fill_params(p, 7, d, f)
    x = make(8, K, T, d, dtype=dtype)
    y0, y1 = torch.empty_like(x), torch.empty_like(x)
    with grawa.SublayerPlan(K, T, d, f, dtype=dtype) as plan:
        plan.ffn(x, p["wg"], p["wu"], p["wd"], y0)
        x[1, T - 1, 5] = NAN
        plan.ffn(x, p["wg"], p["wu"], p["wd"], y1)
        torch.cuda.synchronize()
    assert torch.isnan(y1[1, T - 1]).all()
    assert torch.equal(y0[0], y1[0]) and torch.equal(y0[1, :T - 1], y1[1, :T - 1])


@pytest.mark.parametrize("dtype", [BF, F])
def test_ffn_same_bits_twice_and_on_another_stream(dtype):
    a = run_ffn(700, 2, 200, 136, 264, dtype)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        b = run_ffn(700, 2, 200, 136, 264, dtype)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert all(torch.equal(a[2][n], b[2][n]) for n in ("wg", "wu", "wd"))


def test_ffn_gradient_against_differences():
    """The gradients against central differences of the 64-bit forward formula's loss sum(y dy), along random directions."""
    K, T, d, f = 1, 40, 48, 72
    for act in ("silu", "gelu"):
        p = Params(K, d, f, F, 0)
        fill_params(p, 31, d, f)
        y, dx, gr = run_ffn(31, K, T, d, f, F, act=act)
        x, dy = make(51, K, T, d)[0].double(), make(52, K, T, d)[0].double()
        at = {"x": x, "wg": p["wg"][0].double(), "wu": p["wu"][0].double(), "wd": p["wd"][0].double()}
        grad = {"x": dx[0].double(), "wg": gr["wg"][0].double(), "wu": gr["wu"][0].double(), "wd": gr["wd"][0].double()}

        def loss(v):
            return (ref.ffn(v["x"], v["wg"], v["wu"], v["wd"], None, act, F)[0]["y"] * dy).sum()

        for i, n in enumerate(at):
            way = make(900 + i, *at[n].shape).double()
            h = 1e-5
            diff = (loss({**at, n: at[n] + h * way}) - loss({**at, n: at[n] - h * way})) / (2 * h)
            got = (grad[n] * way).sum()
            # float32 gradients: 2^-19 of their sums; differences: h^2 of a third derivative, 1e-16 / h of the loss
            size = (grad[n].abs() * way.abs()).sum()
            assert abs(diff - got) <= 1e-5 * size, (act, n, diff.item(), got.item())


# -- dropout ------------------------------------------------------------------------

def rng_of(seed, step):
    s = seed - (1 << 64) if seed >= 1 << 63 else seed
    return torch.tensor([s, step], dtype=torch.int64, device=DEV)


def dropped(x, p, seed, step, site):
    K, T, d = x.shape
    w = ref.words(K * T, d, seed, step, site).view(K, T, d).to(DEV)
    p = float(np.float32(p))
    return torch.where(w >= int(p * 2.0 ** 32), x.double() / (1 - p), torch.zeros((), device=DEV, dtype=torch.float64))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("K,T,d", [(1, 1, 1), (2, 3, 8), (3, 5, 7), (2, 4, 64), (1, 2, 1003), (2, 33, 12), (4, 1, 256)])
def test_dropout(K, T, d, dtype):
    for layout in ("plain", "padded", "padded16", "tokens_first"):
        for p, seed, step, site in ((0.1, 1, 0, 0), (0.5, (1 << 64) - 12345, (7 << 32) + 9, 5), (0.9999999, 3, 1, (1 << 32) - 1), (0.0, 4, 1, 1)):
            say("dropout", K, T, d, dtype, layout, p)
            x, r = rows_in(make(1, K, T, d, dtype=dtype), layout), rows_in(make(2, K, T, d, dtype=dtype), layout)
            y = rows_in(torch.zeros((K, T, d), device=DEV, dtype=dtype), layout)
            want = dropped(x, p, seed, step, site)
            grawa.dropout(x, y, p, rng_of(seed, step), site=site)
            ref.assert_within(y, want, (ref.U[dtype] + 2.0 ** -23) * want.abs(), "dropout", dtype)
            assert torch.equal(y == 0, want == 0)
            grawa.dropout(x, y, p, rng_of(seed, step), site=site, residual=r)
            total = want + r.double()
            ref.assert_within(y, total, (ref.U[dtype] + 2.0 ** -23) * total.abs() + 2.0 ** -22 * want.abs(), "dropout and residual", dtype)
            grawa.dropout(x, x, p, rng_of(seed, step), site=site, residual=r)
            assert torch.equal(x, y)


def test_dropout_of_infinities_and_nan():
    K, T, d, p = 1, 8, 64, 0.5
    keep = dropped(torch.ones((K, T, d), device=DEV), p, 11, 2, 3) != 0
    for bad in (float("inf"), NAN):
        x = torch.where(keep, torch.ones((K, T, d), device=DEV), torch.full((K, T, d), bad, device=DEV))
        y = torch.empty_like(x)
        grawa.dropout(x, y, p, rng_of(11, 2), site=3)
        assert torch.equal(y, torch.where(keep, torch.full_like(x, 2.0), torch.zeros_like(x)))


def test_dropout_keeps_as_many_as_it_should():
    x = torch.ones((4, 256, 1024), device=DEV)
    y = torch.empty_like(x)
    for p in (0.1, 0.5, 0.8):
        grawa.dropout(x, y, p, rng_of(77, 5))
        n, kept = x.numel(), (y != 0).sum().item()
        assert abs(kept - n * (1 - p)) < 6 * (n * p * (1 - p)) ** 0.5        # six standard deviations


def test_dropout_of_more_rows_than_a_grid_has():
    T, d = 65535 * 256 + 300, 8                       # a thread a row: blocks walk on
    x, res = make(31, 1, T, d, dtype=BF), make(32, 1, T, d, dtype=BF)
    y, tail = torch.empty_like(x), torch.empty((1, T, d), device=DEV, dtype=BF)
    grawa.dropout(x, y, 0.0, rng_of(6, 2), residual=res)
    grawa.dropout(x, tail, 0.5, rng_of(6, 2), site=1)
    torch.cuda.synchronize()
    assert torch.equal(y, (x.float() + res.float()).to(BF))
    assert torch.logical_or(tail == 0, tail == 2 * x).all()
    assert abs((tail[0, -300:] != 0).double().mean().item() - 0.5) < 0.1
    del x, res, y, tail
    torch.cuda.empty_cache()


def test_ffn_with_dropout_and_residual_equals_the_two_calls():
    for dtype, T in ((BF, 140), (F, 140), (BF, 5), (F, 5), (BF, 40)):
        K, d, f = 2, 72, 136
        p = Params(K, d, f, dtype, 0)
        fill_params(p, 3, d, f)
        x = make(4, K, T, d, dtype=dtype)
        y, z = torch.empty_like(x), torch.empty_like(x)
        rng = rng_of(9, 4)
        with grawa.SublayerPlan(K, T, d, f, dtype=dtype) as plan:
            plan.ffn(x, p["wg"], p["wu"], p["wd"], y, residual=x, p=0.3, rng=rng, site=2)
            plan.ffn(x, p["wg"], p["wu"], p["wd"], z)
            torch.cuda.synchronize()
            for k in range(K):
                out, low = ref.ffn(x[k].double(), p["wg"][k].double(), p["wu"][k].double(), p["wd"][k].double(), None, "silu", dtype)
                keep = dropped(torch.ones_like(x), 0.3, 9, 4, 2)[k]
                want = x[k].double() + keep * out["y"]
                ref.assert_within(y[k], want, ref.U[dtype] * want.abs() + 2 * low["y"] * keep, "T %d" % T, dtype)
                assert torch.equal(y[k][keep == 0], x[k][keep == 0])
            inplace = x.clone()
            plan.ffn(x, p["wg"], p["wu"], p["wd"], inplace, residual=inplace, p=0.3, rng=rng, site=2)
            torch.cuda.synchronize()
            assert torch.equal(inplace, y)


# -- layer norm ---------------------------------------------------------------------

def run_norm(seed, K, T, d, dtype, shift=0, layout="plain", eps=1e-5, mean=0.0, bias=True, add=False, accumulate=False, alias=None):
    say("norm", K, T, d, dtype, "shift", shift, layout, eps, bias, add, accumulate, alias)
    p, gr = Params(K, d, 0, dtype, shift), Params(K, d, 0, dtype, shift, fill=0.5)
    fill_params(p, seed, d, 0)
    x = rows_in((make(seed + 20, K, T, d) + mean).to(dtype), layout)
    dy, more = rows_in(make(seed + 21, K, T, d, dtype=dtype), layout), rows_in(make(seed + 22, K, T, d, dtype=dtype), layout)
    y, dx = rows_in(torch.zeros((K, T, d), device=DEV, dtype=dtype), layout), rows_in(torch.zeros((K, T, d), device=DEV, dtype=dtype), layout)
    x0, dy0 = x.double(), dy.double()
    stats = torch.full((K, T, 2), NAN, device=DEV)
    with grawa.SublayerPlan(K, T, d, dtype=dtype) as plan:
        plan.layer_norm(x, p["weight"], p["bias"] if bias else None, y, eps=eps, stats_out=stats)
        if alias == "dx is dy":
            dx = dy
        plan.layer_norm_backward(dy, x, p["weight"], stats, dx, gr["weight"], gr["bias"] if bias else None, add=more if add else None, accumulate=accumulate)
        if alias == "y is x":
            plan.layer_norm(x, p["weight"], p["bias"] if bias else None, x, eps=eps)
            torch.cuda.synchronize()
            assert torch.equal(x, y)
        torch.cuda.synchronize()
    assert gr.untouched() and p.untouched()
    for k in range(K):
        out, low = ref.norm(x0[k], p["weight"][k].double(), p["bias"][k].double() if bias else None, eps, dtype, dy0[k], more[k].double() if add else None)
        got = {"y": y[k], "dx": dx[k], "dweight": gr["weight"][k], "dbias": gr["bias"][k]}
        for n in got:
            if n == "dbias" and not bias:
                assert (got[n] == 0.5).all()
                continue
            want, bound = out[n], low[n]
            if accumulate and n in ("dweight", "dbias"):
                want, bound = want + 0.5, bound + ref.U[dtype] * (want + 0.5).abs() + 2.0 ** -23
            ref.assert_within(got[n], want, bound, "worker %d %s" % (k, n), dtype)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [1, 2, 7, 64, 100, 512, 513, 1003, 1024, 1025, 1032, 4096, 4100, 5000, 8192, 9000, 16384, 16390, 20000])
def test_norm_widths(d, dtype):
    for K, T in ((1, 1), (3, 5), (2, 70)):
        run_norm(100, K, T, d, dtype, eps=1e-3 if d == 1 else 1e-5)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("layout,shift", [("padded", 1), ("padded16", 8), ("padded16", 3), ("tokens_first", 0), ("plain", 5)])
def test_norm_layouts(layout, shift, dtype):
    for d in (64, 72, 1000, 2056):
        run_norm(200, 3, 9, d, dtype, shift=shift, layout=layout, add=True, accumulate=True)
        run_norm(210, 2, 3, d, dtype, shift=shift, layout=layout, bias=False)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [96, 3001, 20001])
def test_norm_in_place(d, dtype):
    run_norm(300, 2, 7, d, dtype, alias="y is x")
    run_norm(310, 2, 7, d, dtype, alias="dx is dy", add=True)


def test_norm_many_workers_and_tokens():
    run_norm(400, 130, 11, 40, F)
    run_norm(410, 1024, 2, 8, BF)
    run_norm(420, 2, 4097, 200, BF, accumulate=True)
    run_norm(430, 1, 2500, 1500, F, add=True)


def test_norm_far_from_zero_and_constant_rows():
    run_norm(500, 2, 40, 300, F, mean=1000.0)
    K, T, d = 1, 3, 80
    x = torch.full((K, T, d), 3.25, device=DEV)
    w, b = torch.full((K, d), 2.0, device=DEV), torch.full((K, d), -1.0, device=DEV)
    y = torch.empty_like(x)
    with grawa.SublayerPlan(K, T, d, dtype=F) as plan:
        plan.layer_norm(x, w, b, y)
        torch.cuda.synchronize()
        assert (y == -1).all()
        x[0, 1, 3] = NAN
        plan.layer_norm(x, w, b, y)
        torch.cuda.synchronize()
        assert torch.isnan(y[0, 1]).all() and (y[0, 0] == -1).all() and (y[0, 2] == -1).all()


def test_norm_no_tokens():
    for dtype in (BF, F):
        none = torch.empty((2, 0, 24), device=DEV, dtype=dtype)
        p, gr = Params(2, 24, 0, dtype, 0, fill=1.0), Params(2, 24, 0, dtype, 0, fill=2.0)
        stats = torch.empty((2, 0, 2), device=DEV)
        with grawa.SublayerPlan(2, 4, 24, dtype=dtype) as plan:
            plan.layer_norm(none, p["weight"], p["bias"], none, stats_out=stats)
            plan.layer_norm_backward(none, none, p["weight"], stats, none, gr["weight"], gr["bias"], accumulate=True)
            torch.cuda.synchronize()
            assert (gr["weight"] == 2).all() and (gr["bias"] == 2).all()
            plan.layer_norm_backward(none, none, p["weight"], stats, none, gr["weight"], gr["bias"])
            torch.cuda.synchronize()
            assert (gr["weight"] == 0).all() and (gr["bias"] == 0).all() and gr.untouched()


# -- together -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F])
def test_captured_step_replays(dtype):
    """A sublayer's training step recorded into a graph: each replay uses the inputs and the step number as they then are."""
    K, T, d, f = 2, 96, 64, 136
    p, gr = Params(K, d, f, dtype, 0), Params(K, d, f, dtype, 0, fill=0.0)
    fill_params(p, 5, d, f)
    x, dy = make(6, K, T, d, dtype=dtype), make(7, K, T, d, dtype=dtype)
    n, y, dz, dx = (torch.empty_like(x) for _ in range(4))
    stats, rng = torch.empty((K, T, 2), device=DEV), rng_of(123, 0)
    with grawa.SublayerPlan(K, T, d, f, dtype=dtype) as plan:
        save = torch.empty(plan.save_bytes(), dtype=torch.uint8, device=DEV)
        w3, g3 = (p["wg"], p["wu"], p["wd"]), (gr["wg"], gr["wu"], gr["wd"])

        def step():
            plan.layer_norm(x, p["weight"], p["bias"], n, stats_out=stats)
            plan.ffn(n, *w3, y, save=save, residual=x, p=0.25, rng=rng, site=1)
            grawa.dropout(dy, dz, 0.25, rng, site=1)
            plan.ffn_backward(dz, n, *w3, save, dx, *g3)
            plan.layer_norm_backward(dx, x, p["weight"], stats, dx, gr["weight"], gr["bias"], add=dy)

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        seen = []
        for i in range(4):
            rng[1] = i
            x.copy_(make(60 + i, K, T, d, dtype=dtype))
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (y, dx, gr.rows)]
            step()
            torch.cuda.synchronize()
            for a, b in zip(got, (y, dx, gr.rows)):
                assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))
            seen.append(got[0])
        assert not torch.equal(seen[0], seen[1])
        graph.reset()
