"""The whole sublayer as a training step runs it, y = x + dropout(ffn(norm(x))) and back, against the chain of formulas in 64 bits: from the tokens to every
gradient, with nothing of the library's in between.  And the same step replayed from a graph into arrays that hold other values, and with
infinities among the tokens.

How far the chain may be off, as a share of a result's size (both as roots of sums of squares): with bfloat16, eight bits, a rounding is off by
a uniform share of the last place, 2^-8 / sqrt 12 of a value at the mean of 1 / m over a binade, at most 0.0017 of a whole array.  The
longest way, to the gradient of the norm's weight, has nine of them (normalised tokens in the gate, in the up and in the norm itself, the masked
gradient, H, dG, dU, the gradient between the two operators, the result): sqrt 9 of one, 0.005; a product adds its terms' errors as it
adds the terms.  2^-7 is one and a half times that.  With float32 a result is a chain of four sums of up to 2^9 terms, whose roundings of
2^-24 add up to sqrt(2^9) 2^-24 each at the very most, 2^-18 in all."""
import math

import pytest
import torch

import sublayer_reference as ref
from paper_2403_04206_amd import grawa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
SHARE = {BF: 2.0 ** -7, F: 2.0 ** -18}
EPS, SITE, SEED, STEP = 1e-5, 6, 4321, 11
NAN = float("nan")


class Sublayer:
    def __init__(self, K, T, d, f, dtype, act, p, seed=1, at=3):
        self.size, self.dtype, self.act, self.p = (K, T, d, f), dtype, act, p
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        shapes = {"weight": (d,), "bias": (d,), "wg": (f, d), "wu": (f, d), "wd": (d, f)}
        P = at + sum(math.prod(s) for s in shapes.values()) + 7
        self.w, self.g = (torch.full((K, P), NAN, device=DEV, dtype=dtype) for _ in range(2))
        self.v, self.dv, self.used = {}, {}, torch.zeros(P, dtype=torch.bool, device=DEV)
        for n, s in shapes.items():
            e = at + math.prod(s)
            self.v[n], self.dv[n] = self.w[:, at:e].view((K,) + s), self.g[:, at:e].view((K,) + s)
            self.v[n].copy_(self.normal(K, *s) * {"weight": 0.2, "bias": 0.2}.get(n, s[-1] ** -0.5) + (n == "weight"))
            self.used[at:e] = True
            at = e
        self.x, self.dy = self.normal(K, T, d).to(dtype), self.normal(K, T, d).to(dtype)
        self.n, self.y, self.dz, self.dn, self.dx = (torch.full((K, T, d), NAN, device=DEV, dtype=dtype) for _ in range(5))
        self.stats = torch.full((K, T, 2), NAN, device=DEV)
        self.rng = torch.tensor([SEED, STEP], dtype=torch.int64, device=DEV)
        self.plan = grawa.SublayerPlan(K, T, d, f, dtype=dtype, activation=act)
        self.save = torch.full((self.plan.save_bytes(),), 0xff, dtype=torch.uint8, device=DEV)

    def normal(self, *shape):
        return torch.randn(shape, device=DEV, generator=self.gen)

    def forget(self):
        """Everything that a step writes holds NaN."""
        for t in (self.n, self.y, self.dz, self.dn, self.dx, self.stats, self.g):
            t.fill_(NAN)
        self.save.fill_(0xff)

    def step(self):
        w3, g3 = [self.v[n] for n in ("wg", "wu", "wd")], [self.dv[n] for n in ("wg", "wu", "wd")]
        self.plan.layer_norm(self.x, self.v["weight"], self.v["bias"], self.n, eps=EPS, stats_out=self.stats)
        self.plan.ffn(self.n, *w3, self.y, save=self.save, residual=self.x, p=self.p, rng=self.rng, site=SITE)
        grawa.dropout(self.dy, self.dz, self.p, self.rng, site=SITE)
        self.plan.ffn_backward(self.dz, self.n, *w3, self.save, self.dn, *g3)
        self.plan.layer_norm_backward(self.dn, self.x, self.v["weight"], self.stats, self.dx, self.dv["weight"], self.dv["bias"], add=self.dy)

    def results(self):
        return {"y": self.y, "dx": self.dx, **{"d" + n: t for n, t in self.dv.items()}}

    def exact(self):
        K, T, d, f = self.size
        x = self.x.double().requires_grad_()
        at = {n: t.double().requires_grad_() for n, t in self.v.items()}
        p = torch.tensor(self.p, dtype=F).double().item()
        keep = (ref.words(K * T, d, SEED, STEP, SITE).view(K, T, d) >= int(p * 2.0 ** 32)).to(DEV)
        outs = []
        for k in range(K):
            var, mean = torch.var_mean(x[k], 1, correction=0, keepdim=True)
            n = (x[k] - mean) / torch.sqrt(var + EPS) * at["weight"][k] + at["bias"][k]
            g = n @ at["wg"][k].T
            a = {"silu": lambda: g * torch.sigmoid(g), "gelu": lambda: 0.5 * g * torch.erfc(-g / 2 ** 0.5), "relu": lambda: torch.clamp(g, min=0)}[self.act]()
            z = (a * (n @ at["wu"][k].T)) @ at["wd"][k].T
            outs.append(x[k] + torch.where(keep[k], z / (1 - p), torch.zeros_like(z)))
        y = torch.stack(outs)
        grads = torch.autograd.grad(y, [x] + list(at.values()), self.dy.double())
        return {"y": y.detach(), "dx": grads[0], **{"d" + n: g for n, g in zip(at, grads[1:])}}


CASES = [(K, T, d, f, act, p) for K, T, d, f in ((2, 70, 72, 136), (3, 9, 64, 96), (1, 300, 200, 264), (2, 33, 99, 50)) for act, p in (("silu", 0.1), ("gelu", 0.5), ("relu", 0.25), ("silu", 0.0))]


# What bfloat16 makes of relu, whose derivative jumps at 0, is no matter of roundings alone: left to the block by itself.
@pytest.mark.parametrize("dtype,case", [(t, c) for t in (BF, F) for c in CASES if t is F or c[4] != "relu"])
def test_against_64_bits(dtype, case):
    print("[case] whole", dtype, case, flush=True)
    s = Sublayer(*case[:4], dtype, *case[4:])
    s.step()
    torch.cuda.synchronize()
    want, got = s.exact(), s.results()
    for n in want:
        off = (got[n].double() - want[n]).norm() / want[n].norm()
        assert off <= SHARE[dtype], (n, off.item())
    assert torch.isnan(s.g[:, ~s.used]).all() and torch.isnan(s.w[:, ~s.used]).all()
    s.plan.destroy()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T", [5, 96])
def test_replayed_into_other_values(dtype, T):
    """A step recorded into a graph and replayed over arrays that hold NaN, with other tokens and other step numbers, against the step by itself over NaN
    too; every result is finite and the gaps between the rows' parameters stay as they were."""
    s = Sublayer(2, T, 64, 136, dtype, "silu", 0.25)
    s.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    seen = []
    for i in range(4):
        s.rng[1] = i
        s.x.copy_(s.normal(*s.x.shape))
        runs = []
        for run in (graph.replay, s.step):
            s.forget()
            run()
            torch.cuda.synchronize()
            assert all(torch.isfinite(t).all() for t in s.results().values())
            assert torch.isnan(s.g[:, ~s.used]).all()
            runs.append({n: t.clone() for n, t in s.results().items()})
        assert all(torch.equal(runs[0][n], runs[1][n]) for n in runs[0])
        seen.append(runs[0])
    assert not torch.equal(seen[0]["y"], seen[1]["y"])
    graph.reset()
    s.plan.destroy()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T", [3, 40, 140])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), NAN])
def test_a_token_that_is_not_finite(dtype, T, bad):
    """Its own row of y and dx is not finite, the other tokens' rows have the same bits as without it, and so have all rows and gradients of the other worker."""
    a, b = (Sublayer(2, T, 72, 136, dtype, "gelu", 0.0) for _ in range(2))
    b.x[1, T - 1, 5] = bad
    for s in (a, b):
        s.step()
    torch.cuda.synchronize()
    assert torch.isfinite(a.y).all() and not torch.isfinite(b.y[1, T - 1]).any()
    assert torch.equal(a.y[0], b.y[0]) and torch.equal(a.y[1, :T - 1], b.y[1, :T - 1])
    assert torch.equal(a.dx[0], b.dx[0]) and torch.equal(a.dx[1, :T - 1], b.dx[1, :T - 1]) and not torch.isfinite(b.dx[1, T - 1]).any()
    for n in a.dv:
        assert torch.equal(a.dv[n][0], b.dv[n][0]), n
    a.plan.destroy()
    b.plan.destroy()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T", [3, 40, 140])
def test_infinite_inputs_of_the_block(dtype, T):
    """The block by itself: a token with an infinity gives a row that is not finite, and no other row is touched."""
    K, d, f = 2, 72, 136
    s = Sublayer(K, T, d, f, dtype, "silu", 0.0)
    w3 = [s.v[n] for n in ("wg", "wu", "wd")]
    x, y = s.x.clone(), torch.empty_like(s.x)
    s.plan.ffn(s.x, *w3, s.y)
    x[1, 0, 7] = float("inf")
    s.plan.ffn(x, *w3, y)
    torch.cuda.synchronize()
    assert not torch.isfinite(y[1, 0]).any()
    assert torch.equal(y[0], s.y[0]) and torch.equal(y[1, 1:], s.y[1, 1:])
    s.plan.destroy()
