"""Attention and head norm where numbers are not ordinary: no number and infinities in places that a row does not see, scores that
overflow or vanish, rows whose bias hides everything, layouts and sizes at the edges, gradients against differences."""
import math

import pytest
import torch

import attention_reference as ref
from paper_2403_04206_amd import grawa
from test_gpu_attention import Case, generator

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
NAN, INF = math.nan, math.inf


def results(c, train=True):
    c.forward(lse=train)
    if train:
        c.backward()
    torch.cuda.synchronize()
    names = ["o", "dq", "dk", "dv"] if train else ["o"]
    return {n: getattr(c, n).double() for n in names}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("what", ["q", "k", "v", "do"])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_what_a_row_does_not_see_does_not_reach_it(what, value, D, dtype):
    """One odd element in token 100 of 200, window 20: rows that do not see it, and keys that no row sees together with it, are as without it."""
    S, W, j = 200, 20, 100
    c = Case(1, 1, S, S, 2, 1, D, dtype, seed=3, window=W)
    want = c.want()
    getattr(c, what)[0, 0, j, 0, 3] = value
    got = results(c)
    i = torch.arange(S, device="cuda")
    row = i == j
    rows = (i >= j) & (i < j + W) if what in "kv" else row                     # queries that have to do with it
    keys = (i > j - W) & (i < j + W) if what in "kv" else (i > j - W) & (i <= j)
    touched = {"o": rows if what != "do" else i < 0, "dq": rows, "dk": keys, "dv": keys if what != "v" else i < 0}
    for name, (value64, off) in want.items():
        if name == "lse":
            continue
        heads = slice(0, 1) if what in ("q", "do") and name in ("o", "dq") else slice(None)
        other = got[name][:, :, ~touched[name]]
        ref.check(other, value64[:, :, ~touched[name]], off[:, :, ~touched[name]], "%s beside" % name)
        if what == "v" and name == "o":                                          # the element's own column of the rows that see it
            assert not bool(got["o"][0, 0, rows, :, 3].isfinite().any())
            keep = [e for e in range(D) if e != 3]
            ref.check(got["o"][..., keep], value64[..., keep], off[..., keep], "o's other elements")
        elif bool(touched[name].any()) and value is NAN:
            sel = got[name][0, 0, row][:, heads]
            assert not bool(sel.isfinite().all()), name
    c.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq", [1, 100])
def test_a_cache_holds_anything_outside_of_what_is_seen(Sq, dtype):
    """Tokens behind the length and tokens that left the window are no numbers."""
    Sk, W, sinks = 400, 50, 3
    lengths = [300, Sq, 129]
    c = Case(1, 3, Sq, Sk, 4, 2, 64, dtype, seed=4, lengths=lengths, starts=[n - Sq for n in lengths], window=W, sinks=sinks)
    want = c.want(False)
    for n, length in enumerate(lengths):
        for t in (c.k, c.v):
            t[0, n, length:] = NAN
            t[0, n, sinks:max(sinks, length - Sq - W + 1)] = INF
    c.forward(lse=False)
    torch.cuda.synchronize()
    ref.check(c.o, *want["o"], "o")
    c.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
def test_padding_holds_anything(dtype):
    lengths = [150, 64, 0, 97]
    c = Case(2, 2, 150, 150, 2, 1, 72, dtype, seed=5, lengths=lengths, starts=[0] * 4, buckets=8, far=30)
    want = c.want()
    for n, length in enumerate(lengths):
        for t in (c.q, c.k, c.v, c.do):
            t[n // 2, n % 2, length:] = NAN
    c.forward()
    for n, length in enumerate(lengths):
        assert not bool(c.o[n // 2, n % 2, length:].any()) and bool((c.lse[n // 2, n % 2, :, length:] == -INF).all())
        c.o[n // 2, n % 2, length:] = NAN
    c.backward()
    torch.cuda.synchronize()
    for name in ("dq", "dk", "dv", "dbias"):
        ref.check(getattr(c, name), *want[name], name)
    c.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [1e-30, 1e3, 1e17])
def test_scores_of_any_size(size, dtype):
    """One key far above the others; exponentials of all others vanish, the sums neither overflow nor lose the rest."""
    c = Case(1, 1, 130, 130, 1, 1, 64, dtype, seed=6, scale=0.1)
    c.q.fill_(size)
    c.k.zero_()
    c.k[0, 0, 40] = 1.0                                                         # score 6.4 size for key 40, 0 for the others
    c.k[0, 0, 90] = -1.0
    want = c.want(False)["o"][0]
    c.forward(lse=False)
    torch.cuda.synchronize()
    # products of equal numbers are exact up to one rounding of the score, 6.4 size 2^-24, where it matters (size 1e-30: none)
    off = 4 * ref.half_step(dtype) * c.v.double().abs().amax() + 70 * ref.E
    assert bool(c.o.isfinite().all()) and bool(((c.o.double() - want).abs() <= off).all())
    c.plan.destroy()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 3)])
def test_values_with_a_mean_beside_few_keys(window, sinks, D):
    """What all values have in common cancels in dS, which the rounding of o would hide: 8 in all values are 2^-8 8 sqrt(2 / 3) / 2 = 1.3 % of dP.
    Two roundings to bfloat16, of dS and of the result, are off by 2^-8 / sqrt(3) at most in the mean of squares, and together by
    sqrt(2) of that, 0.0032; keys and queries are independent of each other, so that their sums keep the ratio."""
    c = Case(1, 1, 200, 200, 2, 1, D, torch.bfloat16, seed=21, window=window, sinks=sinks)
    c.v.copy_(ref.make(c.v.shape, torch.bfloat16, generator(22), mean=8.0))
    want = c.want()
    got = results(c)
    for name in ("dq", "dk"):
        exact = want[name][0]
        assert float((got[name] - exact).norm() / exact.norm()) < 0.0035, name
    c.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
def test_growing_scores_move_the_maximum(dtype):
    """Each token's score is above all before it by a few: the running maximum moves in most tiles."""
    c = Case(1, 1, 600, 600, 2, 2, 64, dtype, seed=7)
    ramp = torch.arange(600, device="cuda", dtype=torch.float32) / 8
    c.k[..., 0] = ramp[:, None].to(dtype)
    c.q[..., 0] = 24.0
    c.check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Sq,length,window,sinks", [(1, 5000, 0, 0), (3, 5000, 0, 0), (1, 90, 0, 0), (1, 4999, 700, 3), (70, 5000, 0, 0), (70, 70, 0, 0), (129, 4321, 0, 0), (5, 3, 0, 0)])
def test_many_blocks_share_the_keys(Sq, length, window, sinks, D, dtype):
    """Few rows over many keys: most blocks' shares, some of them, or all but one are empty; what is behind the length is no number."""
    Sk = 5000
    c = Case(1, 1, Sq, Sk, 3, 1, D, dtype, seed=23, lengths=[length], starts=[length - Sq], window=window, sinks=sinks)
    want = c.want(False)
    for t in (c.k, c.v):
        t[0, 0, length:] = NAN
    c.forward()
    torch.cuda.synchronize()
    ref.check(c.o, *want["o"], "o")
    ref.check(c.lse, *want["lse"], "lse")
    c.v[0, 0, 0] = NAN                                                             # a share that is no number beside others that are
    c.forward()
    torch.cuda.synchronize()
    seen = ref.visible(length - Sq, length, Sq, Sk, window, sinks, "cuda")[0][:, 0]
    assert bool(c.o[0, 0, seen].isnan().all())
    ref.check(c.o[:, :, ~seen], want["o"][0][:, :, ~seen], want["o"][1][:, :, ~seen], "o of those that do not see it")
    c.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hidden", [-INF, "lowest"])
def test_a_bias_that_hides(hidden, dtype):
    """Every distance hidden by minus infinity gives rows of 0; by the type's lowest number, an average of what is equally low."""
    value = -INF if hidden == -INF else torch.finfo(dtype).min
    c = Case(1, 1, 100, 100, 2, 1, 64, dtype, seed=8, buckets=4, far=20)
    c.bias[:, 0] = value                                                         # head 0: all hidden
    c.bias[:, 1, 1:] = value                                                     # head 1: all but the first distance
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    alone = c.v[:, :, :, :1].double()                                            # head 1 sees itself alone
    assert bool(((c.o[:, :, :, 1:].double() - alone).abs() <= 2 * ref.half_step(dtype) * alone.abs() + 1e-6).all())
    if hidden == -INF:
        assert not bool(c.o[:, :, :, 0].any()) and bool((c.lse[:, :, 0] == -INF).all())
        assert not bool(c.dq[:, :, :, 0].any()) and not bool(c.dbias[:, 0].any())
    else:
        assert bool(c.o.isfinite().all())
    for t in (c.dq, c.dk, c.dv, c.dbias):
        assert bool(t.isfinite().all())
    c.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
def test_layouts(dtype):
    """Heads before tokens, a cache with room between its rows, keys shared by workers and sequences, outputs between other data."""
    K, N, S, H, G, D = 2, 3, 70, 4, 2, 64
    c = Case(K, N, S, S, H, G, D, dtype, seed=9, window=30)
    gen = generator(10)
    big = ref.make((K, N, H, S, 2 * D), dtype, gen)
    c.q = big[..., :D].transpose(2, 3)
    c.k = ref.make((1, 1, G, S, D), dtype, gen).transpose(2, 3).expand(K, N, S, G, D)
    c.v = ref.make((N, S, K, G, D + 8), dtype, gen)[..., :D].permute(2, 0, 1, 3, 4)
    room = torch.full((K, N, S, H, 2 * D), 5.0, device="cuda", dtype=dtype)
    c.o = room[..., D:]
    c.dq = torch.full((H, S, K, N, D), 7.0, device="cuda", dtype=dtype).permute(2, 3, 1, 0, 4)
    c.check()
    assert bool((room[..., :D] == 5.0).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradient_of_the_bias_is_added(dtype):
    c = Case(2, 2, 90, 90, 2, 1, 64, dtype, seed=11, buckets=9, far=50)
    c.forward()
    c.backward()
    once = c.dbias.double()
    c.backward(accumulate=True)
    torch.cuda.synchronize()
    assert bool(((c.dbias.double() - 2 * once).abs() <= 2 * ref.half_step(dtype) * once.abs() + 2 * ref.E * once.abs().amax()).all())
    beside = c.rows[1].clone()
    beside[:, 3:3 + 18] = 0
    assert not bool(beside.any())
    c.plan.destroy()


def test_same_results_every_time():
    for dtype in DTYPES:
        c = Case(1, 2, 700, 700, 4, 2, 64, dtype, seed=12, window=90, sinks=5, buckets=8, far=40)
        c.forward()
        c.backward()
        first = [getattr(c, n).clone() for n in ("o", "lse", "dq", "dk", "dv", "dbias")]
        for _ in range(5):
            c.forward()
            c.backward()
        for a, n in zip(first, ("o", "lse", "dq", "dk", "dv", "dbias")):
            assert torch.equal(a, getattr(c, n)), n
        c.plan.destroy()


def test_no_tokens_and_no_sequences():
    c = Case(2, 3, 8, 8, 2, 1, 64, torch.float32, seed=13, buckets=2, far=4)
    for N, Sq, Sk in ((0, 8, 8), (3, 0, 8), (3, 8, 0), (3, 0, 0)):
        q, k = torch.ones((2, N, Sq, 2, 64), device="cuda"), torch.ones((2, N, Sk, 1, 64), device="cuda")
        o, lse, dq, dk, dv = torch.full_like(q, 7.0), torch.full((2, N, 2, Sq), 7.0, device="cuda"), torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(k, 7.0)
        c.dbias.fill_(7.0)
        c.plan.attention(q, k, k, o, lse_out=lse, bias=c.bias)
        c.plan.attention_backward(q, q, k, k, o, lse, dq, dk, dv, bias=c.bias, dbias=c.dbias)
        torch.cuda.synchronize()
        assert not any(bool(t.any()) for t in (o, dq, dk, dv, c.dbias)) and bool((lse == -INF).all())
    c.plan.destroy()


@pytest.mark.parametrize("D", [64, 128])
def test_gradients_against_differences(D):
    """float32: along one direction at a time, (f(x + h) - f(x - h)) / 2h of f = sum of o do.  The third derivative of a softmax's mean is
    below 10 times the spread of its values times the change of scores cubed, h^2 of which is left; the forward pass is good to 2^-20."""
    c = Case(1, 1, 150, 150, 2, 1, D, torch.float32, seed=14, window=40, sinks=2, buckets=8, far=30)
    c.forward()
    c.backward()
    h = 2.0 ** -7
    gen = generator(15)
    for name in ("q", "k", "v", "bias"):
        t = getattr(c, name)
        keep, way = t.clone(), ref.make(t.shape, torch.float32, gen)
        f = []
        for s in (1, -1):
            t.copy_(keep + s * h * way)
            c.forward()
            f.append((c.o.double() * c.do.double()).sum())
        t.copy_(keep)
        by_difference, by_gradient = ((f[0] - f[1]) / (2 * h)).item(), (getattr(c, "d" + name).double() * way.double()).sum().item()
        total = c.do.double().abs().sum().item()
        print("[case]", name, by_difference, by_gradient, flush=True)
        # directions of size one change a score by about one: the error of the difference is h^2 of the sum of |do| at most, and it
        # averages over 150 rows of 2 D independent terms
        assert abs(by_difference - by_gradient) <= 10 * h * h * total / math.sqrt(c.do.numel()) + 2.0 ** -19 * total / h
    c.plan.destroy()


def test_a_cache_of_more_than_four_gibibytes():
    """280000 tokens of 64 heads of 128 in bfloat16 are 4.6 GB each for keys and values: offsets pass 32 bits."""
    Sk, G, D, W, sinks = 280000, 64, 128, 100, 2
    gen = generator(16)
    cache = torch.zeros((2, 1, 1, Sk, G, D), device="cuda", dtype=torch.bfloat16)
    near = ref.make((2, 1, 1, W, G, D), torch.bfloat16, gen)
    cache[:, :, :, Sk - W:] = near
    first = ref.make((2, 1, 1, sinks, G, D), torch.bfloat16, gen)
    cache[:, :, :, :sinks] = first
    q = ref.make((1, 1, 1, G, D), torch.bfloat16, gen)
    o = torch.empty_like(q)
    with grawa.AttentionPlan(1, 1, Sk, G, G, D, window=W, sinks=sinks) as plan:
        plan.attention(q, cache[0], cache[1], o)
        torch.cuda.synchronize()
        seen = torch.cat((first, near), dim=3)
        value, off = ref.attention(q, seen[0], seen[1], torch.bfloat16)["o"]
        ref.check(o, value, off, "o")
        # the same for a block of queries, whose gradients are written out there
        Sq = 130
        q, do = (ref.make((1, 1, Sq, 2, D), torch.bfloat16, gen) for _ in range(2))
    k, v = cache[0][..., :1, :], cache[1][..., :1, :]
    grads = torch.full((2, 1, 1, Sk, G, D), 7.0, device="cuda", dtype=torch.bfloat16)[..., :1, :]
    o, dq, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((1, 1, 2, Sq), device="cuda")
    with grawa.AttentionPlan(1, 1, Sk, 2, 1, D, window=W, sinks=sinks) as plan:
        plan.attention(q, k, v, o, lse_out=lse)
        plan.attention_backward(do, q, k, v, o, lse, dq, grads[0], grads[1])
        torch.cuda.synchronize()
    low = Sk - Sq - W
    near = lambda t: torch.cat((t[:, :, :sinks], t[:, :, low:]), dim=2)  # noqa: E731
    # the same distances with the first tokens just before the others: they are seen by all in either place
    want = ref.attention(q, near(k), near(v), torch.bfloat16, window=W, sinks=sinks, do=do)
    for name, got in (("o", o), ("dq", dq), ("dk", near(grads[0])), ("dv", near(grads[1]))):
        ref.check(got, *want[name], name)
    assert not bool(grads[:, :, :, sinks:low].any())


def test_no_queries_with_first_tokens():
    """Keys without a query, a window and first tokens that stay visible: gradients of 0."""
    with grawa.AttentionPlan(1, 2, 300, 2, 1, 64, dtype=torch.float32, window=50, sinks=3) as plan:
        q, k, lse = torch.ones((1, 2, 0, 2, 64), device="cuda"), torch.ones((1, 2, 300, 1, 64), device="cuda"), torch.ones((1, 2, 2, 0), device="cuda")
        dk, dv = torch.full_like(k, 7.0), torch.full_like(k, 7.0)
        plan.attention(q, k, k, q)
        plan.attention_backward(q, q, k, k, q, lse, q, dk, dv)
        torch.cuda.synchronize()
        assert not bool(dk.any()) and not bool(dv.any())
