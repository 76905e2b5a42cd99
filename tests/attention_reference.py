"""The attention of K workers in 64 bits, with how far a result may be off, element by element.

A rounding is off by at most half a step relative to the value: U = 2^-8 for bfloat16, 2^-24 for float32; E = 2^-24 is float32's.

Head norm.  The sum of squares takes at most 13 roundings (8 in a lane, 4 over the lanes, the square) and its root halves them; root,
quotient, the two products, the angle (half a turn rounded to 24 bits: pi 2^-25, sine and cosine 2 steps more) and the turn: 24 in all,
32 E is taken, of |n_e| + |n_partner|.  Gradients: twice that of the terms' absolute values; a sum over m rows m E more.

Attention.  A score is a sum of D products in float32, then scaled, biased and taken from the maximum: off by
delta = (D + 8) E (scale sum |q||k| + |bias| + |lse| + 1) at most, the row's largest, and so are the exponential and its sum,
relatively.  A sum over n keys adds (n / 16 + 64) E: sixteen rows of sums and two halves go side by side.  bfloat16 rounds each
exponential once more, U.
  o:   sum P|v| (U + 2 delta + sums) + U |o|           (U before the sum: bfloat16 only, float32's is in the others)
  dS:  P (2 delta (|dP| + |D|) + D E sum |do|(|v| + |o|) + sum |do| (error of o)), and U |dS| where bfloat16 rounds it
  dq, dk: those times |k|, |q|, and U of the result;  dv: sum P|do| (U + 2 delta + sums) + U |dv|;  dbias: the sum of dS's, unrounded."""
import math

import torch

E = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def make(shape, dtype, gen, scale=1.0, mean=0.0):
    return (torch.randn(shape, device=gen.device, generator=gen) * scale + mean).to(dtype)


def angles(starts, S, frequencies):
    """[K, N, S, R / 2] in 64 bits."""
    pos = starts.double()[..., None] + torch.arange(S, device=starts.device, dtype=torch.float64)
    return pos[..., None] * torch.tensor(frequencies, device=starts.device, dtype=torch.float64)


def turn(x, angle, interleaved, back=False, size=False):
    """x [K, N, S, heads, D] turned; with size the sums of absolute values instead."""
    R = 2 * angle.shape[-1]
    if R == 0:
        return x.abs() if size else x.clone()
    i = torch.arange(R // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    y = x.abs() if size else x.clone()
    if size:
        y[..., a] = x[..., a].abs() + x[..., b].abs()
        y[..., b] = y[..., a]
        return y
    cos, sin = angle.cos()[..., None, :], angle.sin()[..., None, :] * (-1.0 if back else 1.0)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def head_norm(x, w, eps, angle, interleaved, dtype):
    """y and how far it may be off."""
    x, w, U = x.double(), w.double()[:, None, None, None], half_step(dtype)
    n = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w
    y = turn(n, angle, interleaved)
    return y, U * y.abs() + 32 * E * turn(n, angle, interleaved, size=True) + 1e-38


def head_norm_backward(dy, x, w, eps, angle, interleaved, dtype):
    """dx, dw and how far they may be off."""
    dy, x, w, U = dy.double(), x.double(), w.double()[:, None, None, None], half_step(dtype)
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    xr, dn, size = x * r, turn(dy, angle, interleaved, back=True), turn(dy, angle, interleaved, size=True)
    a, big = dn * w, size * w.abs()
    dx = r * (a - xr * (a * xr).mean(-1, keepdim=True))
    dw = (dn * xr).sum((1, 2, 3))
    rows = x.shape[1] * x.shape[2] * x.shape[3]
    off = U * dx.abs() + 64 * E * r * (big + xr.abs() * (big * xr.abs()).mean(-1, keepdim=True)) + 1e-38
    return dx, dw, off, U * dw.abs() + (64 + rows) * E * (size * xr.abs()).sum((1, 2, 3)) + 1e-38


def visible(start, length, Sq, Sk, window, sinks, device):
    p = torch.arange(start, start + Sq, device=device)[:, None]
    j = torch.arange(Sk, device=device)[None]
    seen = (j <= p) & (p < length) & (p >= 0)
    if window:
        seen &= (p - j < window) | (j < sinks)
    return seen, (p - j)


def attention(q, k, v, dtype, scale=None, window=0, sinks=0, bias=None, bucket_of=None, lengths=None, starts=None, do=None):
    """Every result and how far it may be off: {name: (value, off)}.  q [K, N, Sq, H, D], k and v [K, N, Sk, G, D]."""
    K, N, Sq, H, D = q.shape
    Sk, G = k.shape[2], k.shape[3]
    scale = D ** -0.5 if scale is None else scale
    U = half_step(dtype)
    inner = U if dtype is torch.bfloat16 else 0.0
    dev = q.device
    zeros = lambda *s: torch.zeros(s, device=dev, dtype=torch.float64)  # noqa: E731
    out = {"o": (zeros(K, N, Sq, H, D), zeros(K, N, Sq, H, D)), "lse": (torch.full((K, N, H, Sq), -math.inf, device=dev, dtype=torch.float64), zeros(K, N, H, Sq))}
    if do is not None:
        out.update(dq=(zeros(K, N, Sq, H, D), zeros(K, N, Sq, H, D)), dk=(zeros(K, N, Sk, G, D), zeros(K, N, Sk, G, D)),
                   dv=(zeros(K, N, Sk, G, D), zeros(K, N, Sk, G, D)))
        if bias is not None:
            out["dbias"] = (zeros(*bias.shape), zeros(*bias.shape))
    if bucket_of is not None:
        bucket_of = torch.tensor(bucket_of, device=dev)
    for w in range(K):
        for n in range(N):
            length = Sk if lengths is None else min(max(int(lengths[w, n]), 0), Sk)
            start = Sk - Sq if starts is None else int(starts[w, n])
            seen, apart = visible(start, length, Sq, Sk, window, sinks, dev)
            alive, some = seen.any(1), seen.any(0)
            for h in range(H):
                g = h // (H // G)
                # what nobody sees may hold anything
                Q = torch.where(alive[:, None], q[w, n, :, h].double(), 0.0)
                Ks, V = (torch.where(some[:, None], t[w, n, :, g].double(), 0.0) for t in (k, v))
                s = Q @ Ks.T * scale
                size = Q.abs() @ Ks.abs().T * scale + 1
                if bias is not None:
                    b = bias[w, h].double()[bucket_of[apart.clamp(0, len(bucket_of) - 1)]]
                    s = s + b
                    size = size + torch.where(b.isfinite(), b.abs(), 0.0)
                s = torch.where(seen, s, -math.inf)
                m = s.amax(1, keepdim=True) if Sk else torch.full((Sq, 1), -math.inf, device=dev, dtype=torch.float64)
                e = torch.where(s == -math.inf, 0.0, torch.exp(s - torch.where(m == -math.inf, 0.0, m)))
                total = e.sum(1, keepdim=True)
                P = e / torch.where(total == 0, 1.0, total)
                lse = torch.where(total == 0, -math.inf, m + torch.log(torch.where(total == 0, 1.0, total)))
                finite = torch.where(lse.isfinite(), lse.abs(), 0.0)
                delta = (D + 8) * E * (torch.where(seen, size, 0.0).amax(1, keepdim=True) + finite if Sk else finite)
                sums = (Sk / 16 + 64) * E
                o = P @ V
                o_off = (P @ V.abs()) * (inner + 2 * delta + sums) + U * o.abs() + 1e-38
                out["o"][0][w, n, :, h], out["o"][1][w, n, :, h] = o, o_off
                out["lse"][0][w, n, h], out["lse"][1][w, n, h] = lse[:, 0], (delta + sums + 4 * E * (finite + 1))[:, 0]
                if do is None:
                    continue
                go = torch.where(alive[:, None], do[w, n, :, h].double(), 0.0)
                dP, dot = go @ V.T, (go * o).sum(1, keepdim=True)
                dS = P * (dP - dot)
                off = P * (2 * delta * (dP.abs() + dot.abs()) + D * E * (go.abs() @ V.abs().T + (go * o).abs().sum(1, keepdim=True)) + (go.abs() * o_off).sum(1, keepdim=True))
                rounded = off + (inner + (Sk + Sq * H) / 16 * E + 64 * E) * dS.abs()
                out["dq"][0][w, n, :, h], out["dq"][1][w, n, :, h] = dS @ Ks * scale, rounded @ Ks.abs() * scale
                out["dk"][0][w, n, :, g] += dS.T @ Q * scale
                out["dk"][1][w, n, :, g] += rounded.T @ Q.abs() * scale
                out["dv"][0][w, n, :, g] += P.T @ go
                out["dv"][1][w, n, :, g] += (P * (inner + 2 * delta + (Sq * H / 16 + 64) * E)).T @ go.abs()
                if bias is not None:
                    at = bucket_of[apart.clamp(0, len(bucket_of) - 1)].flatten()
                    B = bias.shape[2]
                    out["dbias"][0][w, h] += torch.bincount(at, weights=dS.flatten(), minlength=B)
                    out["dbias"][1][w, h] += torch.bincount(at, weights=(off + (Sk + Sq * N) * E * dS.abs()).flatten(), minlength=B)
    for name in ("dq", "dk", "dv", "dbias"):
        if name in out:
            out[name] = (out[name][0], out[name][1] + U * out[name][0].abs() + 1e-38)
    return out


def check(got, want, off, what):
    """Every element within its bound; what is infinite has to be the same, what is no number too."""
    got = got.double()
    special = ~want.isfinite()
    same = torch.where(want.isnan(), got.isnan(), got == want)
    assert bool(same[special].all()), "%s: what is not finite differs" % what
    err, off = (got - want).abs()[~special], off[~special]
    bad = ~(err <= off)
    if bool(bad.any()):
        i = int((err / off).nan_to_num(nan=math.inf).argmax())
        raise AssertionError("%s: %d of %d are off, worst %.3g where %.3g is allowed" % (what, int(bad.sum()), bad.numel(), err[i], off[i]))
    return float((err / off).max()) if err.numel() else 0.0
