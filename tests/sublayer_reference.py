"""The feed-forward sublayer's operators in 64 bits, one worker at a time with plain matrix products, and how far a kernel may be
from them.

The bounds are worst-case propagations of what the kernels are said to do, element by element:
  u   one rounding to the result's type: half of torch.finfo(dtype).eps, 2^-8 of a value for bfloat16, 2^-24 for float32
  v   one rounding of H, dG or dU: as u for bfloat16; float32 operands are split exactly, the products that are left out are below
      2^-22 of a product
  s   float32 sums: 2^-19 of the sum of the absolute values, for sums of up to 2^13 terms (the rounding errors of n ordered float32
      additions grow as sqrt(n) 2^-24, here 2^-17.5 at the very worst alignment of a matrix instruction's partial sums of 32)
"""
import math

import torch

U = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float32)}
V = {torch.bfloat16: U[torch.bfloat16], torch.float32: 2.0 ** -22}
S = 2.0 ** -19
TINY = 1e-30


def act(name, z):
    """The activation, its derivative, and a bound of the second one's change with z."""
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if name == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    on = (z > 0).double()
    return z * on, on


def ffn(x, wg, wu, wd, dy, name, dtype):
    """(outputs, bounds) of one worker; 64-bit matrices.  dy may be None."""
    u, v = U[dtype], V[dtype]
    G, Gb, Up, Ub = x @ wg.T, S * (x.abs() @ wg.abs().T), x @ wu.T, S * (x.abs() @ wu.abs().T)
    a, da = act(name, G)
    ab, dab = 1.2 * Gb + 2.0 ** -21 * a.abs(), Gb + 2.0 ** -21      # |act'| <= 1.2, |act''| <= 1 (the step of relu apart)
    H = a * Up
    Hb = ab * Up.abs() + a.abs() * Ub + ab * Ub + v * H.abs()
    y = H @ wd.T
    out = {"y": y}
    low = {"y": u * y.abs() + Hb @ wd.abs().T * (1 + u) + S * (H.abs() @ wd.abs().T)}
    if dy is None:
        return out, low
    dH, dHb = dy @ wd, S * (dy.abs() @ wd.abs())
    dG, dU = dH * Up * da, dH * a
    dGb = (dHb * Up.abs() + dH.abs() * Ub) * da.abs() + dH.abs() * Up.abs() * dab + v * dG.abs()
    dUb = dHb * a.abs() + dH.abs() * ab + v * dU.abs()
    if name == "relu":          # where the sign of G is not certain, the whole term is
        dGb = dGb + (dH * Up).abs() * (G.abs() <= Gb)
    for n, val, b in (
            ("dx", dG @ wg + dU @ wu, dGb @ wg.abs() + dUb @ wu.abs() + S * (dG.abs() @ wg.abs() + dU.abs() @ wu.abs())),
            ("dwg", dG.T @ x, dGb.T @ x.abs() + S * (dG.T.abs() @ x.abs())),
            ("dwu", dU.T @ x, dUb.T @ x.abs() + S * (dU.T.abs() @ x.abs())),
            ("dwd", dy.T @ H, dy.T.abs() @ Hb + S * (dy.T.abs() @ H.abs()))):
        out[n], low[n] = val, u * val.abs() + b * (1 + u)
    return out, low


def norm(x, w, b, eps, dtype, dy=None, add=None):
    """The same of the layer norm; x: [T, d]."""
    u = U[dtype]
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    h = (x - mean) * rstd
    size = x.abs().amax(1, keepdim=True) * rstd if x.numel() else rstd          # what a rounding of x - mean is relative to
    hb = S / 4 * (size + h.abs())
    y = h * w + (0 if b is None else b)
    out = {"y": y}
    low = {"y": u * y.abs() + hb * w.abs() + 2.0 ** -22 * ((h * w).abs() + (0 if b is None else b.abs()))}
    if dy is None:
        return out, low
    a = dy * w
    m1, m2 = a.mean(1, keepdim=True), (a * h).mean(1, keepdim=True)
    dx = rstd * (a - m1 - h * m2) + (0 if add is None else add)
    amax, hmax = a.abs().mean(1, keepdim=True), (a * h).abs().mean(1, keepdim=True)
    dxb = rstd * (S * (a.abs() + amax + h.abs() * hmax) + hb * m2.abs() + h.abs() * (hb * a.abs()).mean(1, keepdim=True))
    for n, val, bound in (("dx", dx, dxb + 2.0 ** -23 * (0 if add is None else add.abs())), ("dweight", (dy * h).sum(0), (dy.abs() * (hb + S * h.abs())).sum(0)),
                          ("dbias", dy.sum(0), S * dy.abs().sum(0))):
        out[n], low[n] = val, u * val.abs() + bound * (1 + u)
    return out, low


def words(rows, d, seed, step, site):
    """[rows, d] random words in Python's own whole numbers: Philox4x32 with 7 rounds, column / 4 and row in the counter."""
    m = 0xffffffff
    table = []
    for r in range(rows):
        line = []
        for quad in range(-(-d // 4)):
            c, k = [quad, r, site, step & m], [seed & m, (seed >> 32) & m]
            for _ in range(7):
                p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
                c = [(q >> 32) ^ c[1] ^ k[0], q & m, (p >> 32) ^ c[3] ^ k[1], p & m]
                k = [(k[0] + 0x9E3779B9) & m, (k[1] + 0xBB67AE85) & m]
            line += c
        table.append(line[:d])
    return torch.tensor(table, dtype=torch.int64).reshape(rows, d)


def assert_within(got, want, bound, what, dtype):
    got = got.double()
    assert torch.isfinite(got).all(), "%s: not finite" % what
    # results below the type's normal range lose bits that no bound above counts
    off = (got - want).abs() - bound - TINY
    worst = off.max().item() if off.numel() else -1.0
    assert worst <= 0, "%s: %g over its bound (worst ratio %g)" % (what, worst, ((got - want).abs() / (bound + TINY)).max().item())
