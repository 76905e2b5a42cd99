"""The attention of the workers that share a GPU, as measured: the norms of queries and keys with the position rotation, attention
through a sliding window with first tokens that stay visible, and its learned bias by buckets of the distance, forward and backward,
for K workers whose parameters are rows of one flat [K, P] array and whose gradients are written to the rows of another.

A case names what runs (`op`), the workers `K`, the sequences of each worker `N`, the new tokens of each sequence `S`, the tokens
that keys and values have room for `C`, the heads `H` of the queries and `G` of the keys and values (H / G query heads share one),
the width `D` of a head and the one type of activations, parameters and gradients (`dtype`), and
  "window"   a token sees itself and the window - 1 tokens before it; 0: all before it
  "sinks"    first tokens of a sequence that stay visible
  "ragged"   sequences have lengths of their own.  With S = C they begin at position 0 and what follows the length is padding; with
             S < C the new tokens are the last S of the length, which may be shorter than S
  "rotary"   elements of a head that are rotated, in pairs of halves or of neighbours ("interleaved"), for norms
  "start"    position of the first token, for norms
  "buckets"  entries of a head's bias, "far" the distance from which on all share the last one, for attention; 0: no bias
  "shift"    elements that stand before the parameters in each worker's row
Ops (one pass each):
  norm           y = rotate(x / sqrt(mean(x^2) + eps) * weight) of every head of queries and keys, as in evaluation
  norm_train     the same, and from dy: dx and the gradients of both weights
  attend         o = softmax(scale q k^T + bias) v over the visible tokens, as in evaluation or with a cache
  attend_train   the same, and from do: dq, dk, dv and dbias
A row that sees no token is 0, and so are the gradients of padding.
"""
import math
import random

import torch

own = False

EPS = 1e-6
BASE = 10000.0
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, K, N, S, C, H, G, D, dtype, window=0, sinks=0, ragged=False, rotary=0, interleaved=False, start=0, buckets=0, far=0, shift=0):
    c = dict(op=op, K=K, N=N, S=S, C=C, H=H, G=G, D=D, dtype=dtype, window=window, sinks=sinks, ragged=ragged, rotary=rotary,
             interleaved=interleaved, start=start, buckets=buckets, far=far, shift=shift)
    return c if name is None else dict(c, name=name)


def listed():
    # The sizes "350m" are those of the benchmark's transformer: width 1024, here 16 heads of 64.
    return [
        # one token of each of four workers through the norms: a call is nothing but its latency
        _case("qk_token", "norm", 4, 1, 1, 1, 16, 16, 64, "bf16", rotary=64, start=2047),
        # a training step of eight workers
        _case("qk_350m", "norm_train", 8, 1, 2048, 2048, 16, 16, 64, "bf16", rotary=64),
        # full precision, shared key heads, a part of the head rotated by neighbours, far positions
        _case("qk_odd_f32", "norm_train", 3, 2, 517, 517, 6, 2, 104, "f32", rotary=40, interleaved=True, start=1000003, shift=5),
        # one new token of each of four workers over a short cache
        _case("attend_token", "attend", 4, 1, 1, 2048, 16, 16, 64, "bf16"),
        # one new token of each of 32 ragged sequences over a long cache, eight heads of keys and values
        _case("attend_cache", "attend", 1, 32, 1, 16384, 32, 8, 128, "bf16", window=8192, sinks=4, ragged=True),
        # an evaluation batch of odd sizes: a window that ends inside tiles, padding, a head that is no power of two
        _case("attend_odd", "attend", 2, 5, 411, 411, 9, 3, 80, "bf16", window=129, sinks=5, ragged=True),
        # a training step of eight workers, every token sees all before it
        _case("attend_350m", "attend_train", 8, 1, 2048, 2048, 16, 16, 64, "bf16"),
        # one worker that has the card to itself, one long sequence through a window
        _case("attend_long", "attend_train", 1, 1, 16384, 16384, 32, 8, 128, "bf16", window=4096, sinks=4),
        # a padded batch in full precision
        _case("attend_f32", "attend_train", 4, 3, 600, 600, 16, 4, 64, "f32", window=256, sinks=2, ragged=True),
        # one new token of each of 8 sequences of two workers with the learned bias
        _case("bias_token", "attend", 2, 8, 1, 4096, 16, 16, 64, "bf16", ragged=True, buckets=32, far=128, shift=3),
        # a training step of eight workers with the learned bias
        _case("bias_350m", "attend_train", 8, 1, 2048, 2048, 16, 16, 64, "bf16", buckets=32, far=128),
        # the same in full precision: a padded batch, shared key heads, odd numbers of heads and buckets
        _case("bias_odd_f32", "attend_train", 2, 3, 333, 333, 6, 2, 40, "f32", window=200, sinks=3, ragged=True, buckets=19, far=77, shift=1),
    ]


def _places(case):
    """(start, length) of every sequence of every worker."""
    K, N, S, C = case["K"], case["N"], case["S"], case["C"]
    r = random.Random("%d %d %d %d" % (K, N, S, C))
    lengths = [r.randint(max(1, C // 8), C) if case["ragged"] else C for _ in range(K * N)]
    if case["ragged"] and K * N > 2:
        lengths[0], lengths[1] = C, max(1, S // 2)                  # a full one and one that is shorter than its new tokens
    return [(n - S if S < C else 0, n) for n in lengths]


def _pairs(case):
    """Pairs of tokens that see each other, and tokens of keys that some query sees."""
    W, sinks = case["window"] or case["C"] + 1, case["sinks"]
    pairs = keys = 0
    seen = {}
    for start, n in _places(case):
        if (start, n) not in seen:
            first, last = max(start, 0), min(start + case["S"], n) - 1
            count = sum(min(p + 1, W) + min(sinks, max(0, p + 1 - W)) for p in range(first, last + 1))
            low = max(0, first + 1 - W)
            seen[start, n] = (count, last + 1 - low + min(sinks, low) if last >= first else 0)
        pairs += seen[start, n][0]
        keys += seen[start, n][1]
    return pairs, keys


def _flops(case):
    if case["op"].startswith("norm"):
        return (28 if case["op"] == "norm_train" else 8) * case["K"] * case["N"] * case["S"] * (case["H"] + case["G"]) * case["D"]
    return (14 if case["op"] == "attend_train" else 4) * case["D"] * case["H"] * _pairs(case)[0]


def work(case):
    s = 2 if case["dtype"] == "bf16" else 4
    K, H, G, D = case["K"], case["H"], case["G"], case["D"]
    rows = K * case["N"] * case["S"]
    if case["op"].startswith("norm"):
        act, vec = rows * (H + G) * D * s, 2 * K * D * s
        return {"bytes": 4 * act + 2 * vec if case["op"] == "norm_train" else 2 * act + vec, "flops": _flops(case)}  # x, dy in; y, dx out
    keys, bias = _pairs(case)[1], K * H * case["buckets"] * s
    if case["op"] == "attend":
        return {"bytes": (2 * rows * H + 2 * keys * G) * D * s + bias, "flops": _flops(case)}
    return {"bytes": (4 * rows * H + 4 * keys * G) * D * s + 2 * bias, "flops": _flops(case)}  # q, k, v, do in; o, dq, dk, dv out


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(("norm", "norm_train", "attend", "attend", "attend_train", "attend_train"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    biased = op.startswith("attend") and rng.random() < 0.4
    most, size = (3.3e12, 2) if dtype == "bf16" else (3.0e11, 4)
    while True:
        K, N, C = _log_int(rng, 1, 8), _log_int(rng, 1, 32), _log_int(rng, 1, 16384)
        S = C
        if op == "attend" and rng.random() < 0.6:                   # over a cache: single tokens, a few, a chunk
            S = min(C, rng.choice((1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 1024))))
        G = rng.choice((1, 2, 3, 4, 8, 16))
        H = G * rng.choice((1, 1, 2, 3, 4, 8))
        D = rng.choice((64, 64, 128, 128, 16, 40, 72, 96, 112))
        if H > 64 or K * N * C * G * D * size > 5e8 or K * N * S * H * D * size > 2.5e8 or K * H * N * S * C > 8.5e9:
            continue
        extra = dict(shift=rng.choice((0, 0, 8, 1, 3)))
        if op.startswith("norm"):
            extra.update(rotary=rng.choice((D, D, D // 2, 2 * (D // 6), 0)), interleaved=rng.random() < 0.4, start=rng.choice((0, 1, C, _log_int(rng, 1, 1 << 24))))
            if K * N * S * (H + G) * D > 8 * 2048 * 32 * 64:
                continue
        else:
            extra.update(window=rng.choice((0, _log_int(rng, 1, 2 * C))), sinks=rng.choice((0, 0, 1, 4, _log_int(rng, 1, 200))), ragged=rng.random() < 0.5)
            if biased:
                b = rng.choice((2, 8, 19, 32, 64))
                extra.update(buckets=b, far=b + rng.choice((1, 30, 96, 400)))
        case = _case(None, op, K, N, S, C, H, G, D, dtype, **extra)
        if _flops(case) <= most:
            return case


# What a program has in hand: the parameters of each worker one after the other in its row of `w`, the gradients in `g` laid out
# alike; queries, keys and values side by side as one projection leaves them, or keys and values in a cache of their own.

def _row(case):
    at, off = {}, case["shift"]
    for name, shape in (("qweight", (case["D"],)), ("kweight", (case["D"],)), ("bias", (case["H"], case["buckets"]))):
        at[name] = (off, shape)
        off += math.prod(shape)
    return at, -(-off // 256) * 256


def _views(rows, case):
    at, _ = _row(case)
    return {n: rows[:, o:o + math.prod(s)].view((case["K"],) + s) for n, (o, s) in at.items() if math.prod(s)}


def _heads(fused, case, room):
    """Views of queries, keys and values side by side: [K, N, S, H or G, D]."""
    H, G, D = case["H"], case["G"], case["D"]
    parts = torch.split(fused, [H * D, G * D, G * D][:room], dim=3)
    return [t.unflatten(3, (n, D)) for t, n in zip(parts, (H, G, G))]


def _buckets_of(case):
    """The bucket of every distance up to the first that is in the last bucket: the first half of the buckets hold a distance each,
    the others grow by a common factor up to `far`.  In whole numbers: the floor of a logarithm has no borders to miss."""
    b, far = case["buckets"], case["far"]
    half = b // 2
    e, out, n = b - half, [], 0
    while not out or out[-1] < b - 1:
        j = 0
        if n >= half:
            while j < e and far ** (j + 1) * half ** e <= n ** e * half ** (j + 1):
                j += 1
        out.append(n if n < half else min(half + j, b - 1))
        n += 1
    return out


def prepare(case, seed):
    K, N, S, C, H, G, D, dtype = (case[n] for n in ("K", "N", "S", "C", "H", "G", "D", "dtype"))
    dtype = _DTYPES[dtype]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, mean=0.0):
        t = torch.randn(shape, device="cuda", generator=gen)
        return t.mul_(scale).add_(mean).to(dtype)

    _, P = _row(case)
    w = torch.zeros((K, P), device="cuda", dtype=dtype)
    v = _views(w, case)
    v["qweight"].copy_(normal(K, D, scale=0.1, mean=1.0))
    v["kweight"].copy_(normal(K, D, scale=0.1, mean=1.0))
    if case["buckets"]:
        v["bias"].copy_(normal(K, H, case["buckets"]))
    state = {"case": case, "w": w, "v": v, "g": torch.zeros((K, P), device="cuda", dtype=dtype)}
    state["dv"] = _views(state["g"], case)
    norm, train = case["op"].startswith("norm"), case["op"].endswith("train")
    room = 2 if norm else 3
    width = (H + (room - 1) * G) * D
    if norm or S == C:
        fused = normal(K, N, S, width)
        state["x"] = _heads(fused, case, room)
    else:
        fused = normal(K, N, S, H * D)
        state["x"] = [fused.unflatten(3, (H, D)), normal(K, N, C, G, D), normal(K, N, C, G, D)]
    if norm:
        for t in state["x"]:
            t[..., :max(1, D // 32)] *= 4.0                         # a few channels are large
        state["y"] = _heads(torch.empty_like(fused), case, room)
        state["starts"] = torch.full((K, N), case["start"], dtype=torch.int32, device="cuda")
    else:
        if case["sinks"]:
            state["x"][1][:, :, :case["sinks"]] *= 2.0              # first tokens draw more attention
        state["y"] = torch.empty((K, N, S, H, D), device="cuda", dtype=dtype)
        state["lse"] = torch.empty((K, N, H, S), device="cuda")
        places = torch.tensor(_places(case), dtype=torch.int32).view(K, N, 2)
        state["starts"], state["lengths"] = places[..., 0].contiguous().cuda(), places[..., 1].contiguous().cuda()
    if train:
        state["dy"] = _heads(normal(K, N, S, width, scale=1e-2), case, room) if norm else normal(K, N, S, H, D, scale=1e-2)
        state["dx"] = _heads(torch.empty_like(fused), case, room)
    if own:
        from paper_2403_04206_amd import grawa
        kinds = dict(dtype=dtype, window=case["window"], sinks=case["sinks"])
        if norm and case["rotary"]:
            kinds.update(frequencies=grawa.rotary_frequencies(case["rotary"], BASE), interleaved=case["interleaved"])
        if case["buckets"]:
            kinds.update(buckets=case["buckets"], bucket_of=grawa.log_buckets(case["buckets"], case["far"]))
        state["plan"] = grawa.AttentionPlan(K, N, C, H, G, D, **kinds)
    elif case["buckets"]:
        state["bucket_of"] = torch.tensor(_buckets_of(case), device="cuda")
    return state


# The plain forms, in 32 bits; angles in 64.

def _turn(x, case, positions, back=False):
    """x [K, N, S, heads, D] rotated by the angles of its positions [K, N, S], or back by them."""
    R = case["rotary"]
    if not R:
        return x
    i = torch.arange(R // 2, device="cuda", dtype=torch.float64)
    angle = positions.double()[..., None] * BASE ** (-2.0 * i / R)
    cos, sin = torch.cos(angle).float()[:, :, :, None], torch.sin(angle).float()[:, :, :, None]
    if back:
        sin = -sin
    y = x.clone()
    first, second = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_norm(state):
    c = state["case"]
    dtype = _DTYPES[c["dtype"]]
    positions = state["starts"][..., None] + torch.arange(c["S"], device="cuda")
    outs = {}
    for i, n in enumerate("qk"):
        x, w = state["x"][i].float(), state["v"][n + "weight"].float()[:, None, None, None]
        r = ((x * x).mean(-1, keepdim=True) + EPS) ** -0.5
        outs[n] = _turn(x * r * w, c, positions).to(dtype)
        if c["op"] == "norm_train":
            dn = _turn(state["dy"][i].float(), c, positions, back=True)
            a = dn * w
            outs["d" + n] = (r * (a - x * r * r * (a * x).mean(-1, keepdim=True))).to(dtype)
            outs["d" + n + "weight"] = (dn * x * r).sum((1, 2, 3)).to(dtype)
    return outs


def _plain_attend(state):
    c = state["case"]
    K, N, S, C, H, G, D, B = (c[n] for n in ("K", "N", "S", "C", "H", "G", "D", "buckets"))
    dtype, train, share = _DTYPES[c["dtype"]], c["op"] == "attend_train", H // G
    scale = D ** -0.5
    # [K, N, G, share, S, D] and [K, N, G, C, D], a worker's sequence after the other
    q = state["x"][0].float().permute(0, 1, 3, 2, 4).reshape(K * N, G, share, S, D)
    k, v = (t.float().permute(0, 1, 3, 2, 4).reshape(K * N, G, 1, C, D) for t in state["x"][1:])
    if train:
        dy = state["dy"].float().permute(0, 1, 3, 2, 4).reshape(K * N, G, share, S, D)
    starts, lengths = state["starts"].reshape(-1).long(), state["lengths"].reshape(-1).long()
    if B:
        table = state["v"]["bias"].float()[:, None].expand(K, N, H, B).reshape(K * N, G, share, B)
        by_distance = torch.zeros((S + C, B), device="cuda", dtype=torch.float64)
    o = torch.empty((K * N, G, share, S, D), device="cuda")
    dq, dk, dv = (torch.empty_like(o), torch.empty_like(k), torch.empty_like(v)) if train else (None, None, None)
    dbias = torch.zeros((K * N, G, share, B), device="cuda", dtype=torch.float64)
    j = torch.arange(C, device="cuda")
    rows = max(1, (1 << 28) // (G * share * S * C))                 # sequences at a time, then heads
    heads = G if rows > 1 or G * share * S * C <= 1 << 28 else max(1, (1 << 28) // (share * S * C))
    for a in range(0, K * N, rows):
        at = slice(a, a + rows)
        p = starts[at, None] + torch.arange(S, device="cuda")
        apart = p[:, :, None] - j
        seen = (apart >= 0) & ((p >= 0) & (p < lengths[at, None]))[:, :, None]
        if c["window"]:
            seen &= (apart < c["window"]) | (j < c["sinks"])
        hidden = ~seen[:, None, None]
        alive = seen.any(-1)[:, None, None, :, None]
        if B:
            bucket = state["bucket_of"][apart.clamp(0, len(state["bucket_of"]) - 1)]
        # what padding holds counts nowhere
        real = (j < lengths[at, None])[:, None, None, :, None]
        for h in range(0, G, heads):
            hs = slice(h, h + heads)
            qq = torch.where(alive, q[at, hs], 0.0)
            kk, vv = torch.where(real, k[at, hs], 0.0), torch.where(real, v[at, hs], 0.0)
            s = torch.matmul(qq, kk.transpose(-1, -2)) * scale
            if B:
                s += torch.take_along_dim(table[at, hs, :, None], bucket[:, None, None], dim=-1)
            s.masked_fill_(hidden, -math.inf)
            m = s.amax(-1, keepdim=True)
            s = torch.exp(s - torch.where(alive, m, 0.0))
            total = s.sum(-1, keepdim=True)
            s /= torch.where(alive, total, 1.0)
            o[at, hs] = torch.matmul(s, vv)
            if not train:
                continue
            g = torch.where(alive, dy[at, hs], 0.0)
            ds = torch.matmul(g, vv.transpose(-1, -2))
            ds = s * (ds - (g * o[at, hs]).sum(-1, keepdim=True))
            dv[at, hs] = torch.matmul(s.transpose(-1, -2), g).sum(2, keepdim=True)
            dq[at, hs] = torch.matmul(ds, kk) * scale
            dk[at, hs] = torch.matmul(ds.transpose(-1, -2), qq).sum(2, keepdim=True) * scale
            if B:
                for i in range(ds.shape[0]):                        # sums along the diagonals: row r is moved r places to the right
                    lines = torch.nn.functional.pad(ds[i].flip(-1), (0, S)).flatten(2)[..., :S * (C + S - 1)].unflatten(2, (S, C + S - 1)).sum(2, dtype=torch.float64)
                    apart0 = int(_places(c)[a + i][0]) - (C - 1)    # of the first diagonal
                    which = state["bucket_of"][(torch.arange(C + S - 1, device="cuda") + apart0).clamp(0, len(state["bucket_of"]) - 1)]
                    by_distance.zero_()
                    by_distance[torch.arange(C + S - 1, device="cuda"), which] = 1.0
                    dbias[a + i, hs] += torch.matmul(lines, by_distance[:C + S - 1])
    back = lambda t, n, L: t.reshape(K, N, n, L, D).permute(0, 1, 3, 2, 4).contiguous().to(dtype)  # noqa: E731
    outs = {"o": back(o, H, S)}
    if train:
        outs.update(dq=back(dq, H, S), dk=back(dk, G, C), dv=back(dv, G, C))
        if B:
            outs["dbias"] = dbias.reshape(K, N, H, B).sum(1).to(dtype)
    return outs


# The framework's own operators, as a program calls them.

def _own(state):
    c, plan, v, dv = state["case"], state["plan"], state["v"], state["dv"]
    x, y = state["x"], state["y"]
    if c["op"].startswith("norm"):
        plan.head_norm(*x, v["qweight"], v["kweight"], *y, eps=EPS, starts=state["starts"])
        if c["op"] == "norm":
            return {"q": y[0], "k": y[1]}
        plan.head_norm_backward(*state["dy"], *x, v["qweight"], v["kweight"], *state["dx"], dv["qweight"], dv["kweight"], eps=EPS, starts=state["starts"])
        return {"q": y[0], "dq": state["dx"][0], "dqweight": dv["qweight"], "k": y[1], "dk": state["dx"][1], "dkweight": dv["kweight"]}
    places = dict(bias=v.get("bias"), lengths=state["lengths"], starts=state["starts"])
    if c["op"] == "attend":
        plan.attention(*x, y, **places)
        return {"o": y}
    plan.attention(*x, y, lse_out=state["lse"], **places)
    dx = state["dx"]
    plan.attention_backward(state["dy"], *x, y, state["lse"], *dx, dbias=dv.get("bias"), **places)
    outs = {"o": y, "dq": dx[0], "dk": dx[1], "dv": dx[2]}
    if c["buckets"]:
        outs["dbias"] = dv["bias"]
    return outs


def run(state):
    if own:
        return _own(state)
    return _plain_norm(state) if state["case"]["op"].startswith("norm") else _plain_attend(state)


# The definition in 64 bits, a head at a time: gradients by torch's differentiation, rotations as products of complex numbers.

def _exact_norm(state):
    c = state["case"]
    R, D, train = c["rotary"], c["D"], c["op"] == "norm_train"
    pos = state["starts"].double()[:, :, None] + torch.arange(c["S"], device="cuda", dtype=torch.float64)
    freq = torch.tensor([math.exp(-math.log(BASE) * 2 * i / R) for i in range(R // 2)], device="cuda", dtype=torch.float64)
    angle = pos[..., None, None] * freq
    phase = torch.complex(torch.cos(angle), torch.sin(angle))
    outs = {}
    for i, n in enumerate("qk"):
        x = state["x"][i].double().requires_grad_(train)
        w = state["v"][n + "weight"].double().requires_grad_(train)
        with torch.set_grad_enabled(train):
            u = x / torch.sqrt(x.square().sum(4, keepdim=True) / D + EPS) * w.view(c["K"], 1, 1, 1, D)
            if R:
                z = u[..., :R].unflatten(4, (-1, 2)) if c["interleaved"] else torch.stack((u[..., :R // 2], u[..., R // 2:R]), dim=-1)
                z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * phase)
                z = z.flatten(4) if c["interleaved"] else torch.cat((z[..., 0], z[..., 1]), dim=4)
                u = torch.cat((z, u[..., R:]), dim=4)
        outs[n] = u.detach()
        if train:
            outs["d" + n], outs["d" + n + "weight"] = torch.autograd.grad(u, (x, w), state["dy"][i].double())
    return outs


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"].startswith("norm"):
        return _exact_norm(state)
    K, N, S, C, H, G, D, B = (case[n] for n in ("K", "N", "S", "C", "H", "G", "D", "buckets"))
    train = case["op"] == "attend_train"
    q, k, v = state["x"]
    zeros = lambda *shape: torch.zeros(shape, device="cuda", dtype=torch.float64)  # noqa: E731
    o, dq, dk, dv, dbias = zeros(K, N, S, H, D), zeros(K, N, S, H, D), zeros(K, N, C, G, D), zeros(K, N, C, G, D), zeros(K, H, B)
    places = _places(case)
    if B:
        limits = torch.tensor(_buckets_of(case), device="cuda")
    for w in range(K):
        for n in range(N):
            start, length = places[w * N + n]
            lo, hi = max(0, -start), min(S, length - start)         # new tokens that stand for something
            if lo >= hi:
                continue
            pos = torch.arange(start + lo, start + hi, device="cuda")[:, None]
            key = torch.arange(length, device="cuda")[None]
            near = pos - key < case["window"] if case["window"] else key >= 0
            mask = (key <= pos) & (near | (key < case["sinks"]))
            if B:
                bucket = limits[torch.clamp(pos - key, min=0, max=len(limits) - 1)]
            for h in range(H):
                g = h // (H // G)
                qh, kh, vh = (t.double().requires_grad_(train) for t in (q[w, n, lo:hi, h], k[w, n, :length, g], v[w, n, :length, g]))
                with torch.set_grad_enabled(train):
                    score = qh @ kh.T / math.sqrt(D)
                    if B:
                        score = score + state["v"]["bias"][w, h].double()[bucket]
                    y = torch.softmax(torch.where(mask, score, -math.inf), dim=1) @ vh
                o[w, n, lo:hi, h] = y.detach()
                if train:
                    grads = torch.autograd.grad(y, (qh, kh, vh, score), state["dy"][w, n, lo:hi, h].double())
                    dq[w, n, lo:hi, h] = grads[0]
                    dk[w, n, :length, g] += grads[1]
                    dv[w, n, :length, g] += grads[2]
                    if B:
                        dbias[w, h] += torch.bincount(bucket.flatten(), weights=grads[3].flatten(), minlength=B)
    if not train:
        return {"o": o}
    return {"o": o, "dq": dq, "dk": dk, "dv": dv, **({"dbias": dbias} if B else {})}
