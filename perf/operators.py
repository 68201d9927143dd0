"""Timed calls of the operators around the match windows: differential attention, rotary grid positions, layer norm.

Each case is one call.  ``run`` computes it with the package where ``own`` is true, otherwise in its plain form: elementary
torch operations in 32 bits, rounded once at the end.  ``exact`` computes the same in 64 bits.

Inputs of the attention follow the recipe of ``scram_inputs``: blurred keys, queries that are noisy copies of coherently
displaced keys (each half of the channels with a displacement of its own), maps as PatchMatch leaves them -- the displaced
targets of the two halves in turn, a tenth of them a pixel or two off, a few elsewhere.
"""
import math

import torch

own = False

_DEVICE = "cuda"
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _attend(op, name=None, **kw):
    c = dict(op=op, S=1, Hq=32, Wq=32, Hk=0, Wk=0, d=64, dtype="bf16", window=5, kappa=1, causal=False, first=0)
    c.update(kw)
    c["Hk"], c["Wk"] = c["Hk"] or c["Hq"], c["Wk"] or c["Wq"]
    return dict(c, name=name) if name else c


def _rotary(op, name=None, **kw):
    c = dict(op=op, S=1, T=1, H=32, W=32, d=64, dtype="bf16", tensors=2, nt=0, nh=8, nw=8, groups=2, interleaved=False,
             far=0, per_slice=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _norm(op, name=None, **kw):
    c = dict(op=op, rows=1024, channels=64, dtype="bf16", grad="bf16", affine=True)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new pixel of each of 32 slices of an autoregressive layer, half way down a 64 x 64 grid: latency counts
        _attend("attend", "attend_pixel", S=32, Hq=1, Wq=1, Hk=64, Wk=64, window=7, kappa=2, causal=True, first=2083),
        # the smallest workload of the package: launches and host time count
        _attend("attend", "attend_tiny", S=1, Hq=32, Wq=32, d=16, dtype="f32", window=3),
        # four heads of a 256 x 256 image, one match for each of the two maps
        _attend("attend", "attend_self256", S=4, Hq=256, Wq=256, window=5, kappa=2),
        # two images of different sizes, 32-bit
        _attend("attend", "attend_cross", S=8, Hq=128, Wq=128, Hk=192, Wk=192, d=32, dtype="f32", window=3, kappa=2),
        # a training step's gradients, 2 x 8 heads
        _attend("attend_backward", "attend_grad_self128", S=16, Hq=128, Wq=128, window=5, kappa=2),
        # gradients of a small autoregressive layer in 32-bit, ragged sides
        _attend("attend_backward", "attend_grad_ragged", S=4, Hq=93, Wq=125, d=32, dtype="f32", window=3, kappa=2, causal=True),
        # queries and keys of one new pixel per slice, each slice at a position of its own
        _rotary("rotary", "rotary_pixel", S=32, H=1, W=1, far=4096, per_slice=True),
        # queries and keys of four heads of a 256 x 256 image
        _rotary("rotary", "rotary_self256", S=4, H=256, W=256),
        # gradients of one tensor of a clip, 32-bit, adjacent pairs, a part of the channels not turned, far frames
        _rotary("rotary_backward", "rotary_grad_clip", S=6, T=16, H=45, W=80, d=100, dtype="f32", tensors=1,
                nt=12, nh=17, nw=17, groups=1, interleaved=True, far=1 << 20),
        # the rows of one head of a 256 x 256 image, with the statistics that training keeps
        _norm("norm", "norm_heads", rows=4 * 256 * 256, channels=64),
        # their gradients from the 32-bit gradients of the attention
        _norm("norm_backward", "norm_grad_heads", rows=4 * 256 * 256, channels=64, grad="f32"),
        # wide rows of a residual stream
        _norm("norm_backward", "norm_grad_wide", rows=8 * 32 * 32, channels=4096),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(["attend", "attend", "attend", "attend_backward", "attend_backward", "rotary", "rotary_backward", "norm",
                     "norm_backward", "norm_backward"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op.startswith("attend"):
        d, window, kappa = rng.choice([12, 16, 32, 64, 64, 128]), rng.choice([1, 3, 3, 5, 5, 7, 9]), rng.choice([1, 2, 2, 3, 4])
        S, H = log(1, 32), log(24, 400)
        W = max(20, min(640, int(H * math.exp(rng.uniform(-0.7, 0.7)))))
        while S * H * W * d * kappa * window ** 2 > 4 * 256 * 256 * 64 * 50:
            S, H, W = (max(1, S // 2), H, W) if S > 1 else (1, max(24, H * 3 // 4), max(20, W * 3 // 4))
        kw = dict(S=S, Hq=H, Wq=W, d=d, dtype=dtype, window=window, kappa=max(kappa, 2) if window == 1 else kappa)
        kind = rng.random()
        if kind < 0.2:  # another image as keys
            f = rng.choice([0.75, 1.5])
            kw.update(Hk=max(3, int(H * f)), Wk=max(3, int(W * f)))
        elif kind < 0.45:
            kw.update(causal=True)
        elif kind < 0.6 and op == "attend":  # the next pixels of one row
            kw.update(Hq=1, Wq=rng.choice([1, 1, 2, 7]), Hk=H, Wk=W + 7, causal=True)
            kw.update(first=rng.randrange(0, H * (W + 7) - 7))
        return _attend(op, **kw)
    if op.startswith("rotary"):
        groups = rng.choice([1, 1, 2])
        pairs = rng.choice([8, 16, 23, 32, 48, 64])
        T = rng.choice([1, 1, 1, log(2, 24)])
        nt = rng.randrange(1, pairs // 3 + 1) if T > 1 else 0
        nh = (pairs - nt) // 2
        d = groups * 2 * (pairs + rng.choice([0, 0, 3, 8]))
        S, H = log(1, 64), log(1, 300)
        W = max(1, min(500, int(H * math.exp(rng.uniform(-0.7, 0.7)))))
        while S * T * H * W * d > 2 * 4 * 256 * 256 * 64:
            S, T, H = (max(1, S // 2), T, H) if S > 1 else (1, max(1, T // 2), max(1, H * 3 // 4))
        return _rotary(op, S=S, T=T, H=H, W=W, d=d, dtype=dtype, tensors=rng.choice([1, 2]), nt=nt, nh=nh, nw=pairs - nt - nh,
                       groups=groups, interleaved=rng.random() < 0.5, far=rng.choice([0, 1000, 1 << 24]), per_slice=rng.random() < 0.3)
    channels = rng.choice([log(16, 256), 64, log(256, 12000), 8 * log(32, 1500)])
    rows = max(1, log(1, 8 * 32 * 32 * 4096) // channels)
    return _norm(op, rows=rows, channels=channels, dtype=dtype, grad=rng.choice([dtype, "f32"]), affine=rng.random() < 0.8)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _blur(x, sigma):
    """Gaussian blur of [S, H, W, c] along both grid axes, reflecting border."""
    for axis in (1, 2):
        n, r = x.shape[axis], int(4.0 * sigma + 0.5)
        t = torch.arange(-r, r + 1, device=_DEVICE)
        taps = torch.exp(-0.5 * (t / sigma) ** 2)
        at = (torch.arange(n, device=_DEVICE)[:, None] + t) % (2 * n)
        at = torch.where(at >= n, 2 * n - 1 - at, at)
        m = torch.zeros(n, n, device=_DEVICE).scatter_add_(1, at, (taps / taps.sum()).expand(n, -1).contiguous())
        x = torch.movedim(torch.tensordot(m, x, dims=([1], [axis])), 0, axis)
    return x


def _attend_inputs(c, gen):
    S, Hq, Wq, Hk, Wk, d = (c[k] for k in ("S", "Hq", "Wq", "Hk", "Wk", "d"))
    normal = lambda *s: torch.randn(*s, generator=gen, device=_DEVICE)  # noqa: E731
    whole = lambda n: torch.randint(n, (S, Hq, Wq), generator=gen, device=_DEVICE)  # noqa: E731
    kind, n, h = _TYPES[c["dtype"]], Hk * Wk, d // 2
    K = _blur(normal(S, Hk, Wk, d), 4.0).reshape(S, n, 2, h)
    K = K / K.norm(dim=3, keepdim=True)
    partial = c["causal"] and (Hq, Wq) != (Hk, Wk)
    own_at = c["first"] + torch.arange(Hq * Wq, device=_DEVICE).reshape(Hq, Wq)  # raster index, where causal
    if partial:
        x, y = own_at // Wk, own_at % Wk
    else:
        x = torch.arange(Hq, device=_DEVICE)[:, None] * (Hk / Hq)
        y = torch.arange(Wq, device=_DEVICE)[None, :] * (Wk / Wq)
    F = min(64.0, max(2.0, min(Hk, Wk) / 6))
    target, maps, q = [], [], []
    for half in (0, 1):
        f = _blur(torch.rand(S, Hq, Wq, 2, generator=gen, device=_DEVICE) - 0.5, 8.0)
        f = f * (F / f.norm(dim=3).amax(dim=(1, 2)).clamp(min=1e-6)[:, None, None, None])
        tr, tc = (x + f[..., 0]).round().long().clamp(0, Hk - 1), (y + f[..., 1]).round().long().clamp(0, Wk - 1)
        t = torch.where(torch.rand(S, Hq, Wq, generator=gen, device=_DEVICE) < 0.05, whole(Hk * Wk), tr * Wk + tc)
        t = torch.minimum(t, own_at) if c["causal"] else t
        target.append(t)
        q.append(4.0 * torch.gather(K[:, :, half], 1, t.reshape(S, -1, 1).expand(-1, -1, h)) + 0.3 * normal(S, Hq * Wq, h))
    for e in range(c["kappa"]):  # the halves' targets in turn; later ones some pixels away
        off = (torch.rand(S, Hq, Wq, generator=gen, device=_DEVICE) < 0.1).long()
        r = (target[e % 2] // Wk + off * (whole(5) - 2) + 2 * (e // 2)).clamp(0, Hk - 1)
        v = (target[e % 2] % Wk + off * (whole(5) - 2) + 2 * (e // 2)).clamp(0, Wk - 1)
        maps.append(torch.minimum(r * Wk + v, own_at) if c["causal"] else r * Wk + v)
    V = normal(S, Hk, Wk, d)
    # an output's gradient, in part along the values that the second map takes
    dO = normal(S, Hq, Wq, d) + 0.5 * torch.gather(V.reshape(S, -1, d), 1, target[1].reshape(S, -1, 1).expand(-1, -1, d)).reshape(S, Hq, Wq, d)
    return dict(Q=torch.cat(q, 2).reshape(S, Hq, Wq, d).to(kind), K=K.reshape(S, Hk, Wk, d).to(kind), V=V.to(kind), dO=dO.to(kind),
                lam=0.5 + 0.2 * normal(S), maps=torch.stack(maps).to(torch.int32))


def prepare(case, seed):
    gen = torch.Generator(device=_DEVICE).manual_seed(int(seed))
    c = dict(case)
    if c["op"].startswith("attend"):
        return dict(c, **_attend_inputs(case, gen))
    kind = _TYPES[c["dtype"]]
    if c["op"].startswith("rotary"):
        shape = (c["S"], c["T"], c["H"], c["W"], c["d"])
        c["X"] = [torch.randn(*shape, generator=gen, device=_DEVICE).to(kind) for _ in range(c["tensors"])]
        c["origin"] = torch.randint(c["far"] + 1, (c["S"] if c["per_slice"] else 1, 3), generator=gen, device=_DEVICE, dtype=torch.int32)
        return c
    rows, n = c["rows"], c["channels"]
    # activations: an offset and a spread of their own in every row
    x = torch.randn(rows, n, generator=gen, device=_DEVICE)
    x = x * (0.5 + torch.rand(rows, 1, generator=gen, device=_DEVICE)) + torch.randn(rows, 1, generator=gen, device=_DEVICE)
    c["X"] = x.to(kind)
    c["weight"] = (1.0 + 0.2 * torch.randn(n, generator=gen, device=_DEVICE)).to(kind) if c["affine"] else None
    c["bias"] = (0.2 * torch.randn(n, generator=gen, device=_DEVICE)).to(kind) if c["affine"] else None
    if c["op"] == "norm_backward":  # what the forward pass left
        c["dY"] = torch.randn(rows, n, generator=gen, device=_DEVICE).to(_TYPES[c["grad"]])
        xf = c["X"].float()
        c["mean"] = xf.mean(1)
        c["rstd"] = torch.rsqrt(xf.var(1, unbiased=False) + 1e-5)
    return c


# ---------------------------------------------------------------------------
# one call
# ---------------------------------------------------------------------------
def _sections(c):
    return c["nt"], c["nh"], c["nw"]


def _own(c):
    import paper_1905_10308_amd as scram

    if c["op"] == "attend":
        return scram.differential_attend(c["Q"], c["K"], c["V"], c["maps"], c["lam"], c["window"], causal=c["causal"], first=c["first"])
    if c["op"] == "attend_backward":
        return scram.differential_attend_backward(c["Q"], c["K"], c["V"], c["maps"], c["lam"], c["dO"], c["window"], causal=c["causal"],
                                                  first=c["first"])
    if c["op"].startswith("rotary"):
        turn = scram.rotary if c["op"] == "rotary" else scram.rotary_backward
        return turn(*c["X"], sections=_sections(c), origin=c["origin"], groups=c["groups"], interleaved=c["interleaved"])
    if c["op"] == "norm":
        return scram.layer_norm(c["X"], c["weight"], c["bias"], stats=True)
    return scram.layer_norm_backward(c["dY"], c["X"], c["mean"], c["rstd"], c["weight"])


def _slots(c, maps):
    """The keys of every query's windows: flat key [n, kappa w^2] over all slices, and whether it counts."""
    S, Hk, Wk, half = c["S"], c["Hk"], c["Wk"], c["window"] // 2
    plane = c["Hq"] * c["Wq"]
    m = maps.reshape(c["kappa"], S * plane).long().t()
    u, v = m // Wk, m % Wk
    step = torch.arange(-half, half + 1, device=_DEVICE)
    r = (u[:, :, None, None] + step[:, None]).expand(-1, -1, -1, c["window"]).reshape(S * plane, -1)
    q = (v[:, :, None, None] + step).expand(-1, -1, c["window"], -1).reshape(S * plane, -1)
    ok = (r >= 0) & (r < Hk) & (q >= 0) & (q < Wk)
    # not in an earlier window of the query
    held = ((r[:, :, None] - u[:, None]).abs() <= half) & ((q[:, :, None] - v[:, None]).abs() <= half)
    mine = torch.arange(c["kappa"], device=_DEVICE).repeat_interleave(c["window"] ** 2)
    ok &= ~(held & (torch.arange(c["kappa"], device=_DEVICE) < mine[:, None])).any(2)
    at = torch.arange(S * plane, device=_DEVICE)
    if c["causal"]:
        ok &= r * Wk + q <= (c["first"] + at % plane)[:, None]
    return (at // plane * (Hk * Wk))[:, None] + torch.where(ok, r * Wk + q, 0), ok


def _plain_attend(c):
    n, h, d, S = c["S"] * c["Hq"] * c["Wq"], c["d"] // 2, c["d"], c["S"]
    scale = h ** -0.5
    at, ok = _slots(c, c["maps"])
    q = c["Q"].reshape(n, 1, 2, h).float()
    k = c["K"].reshape(-1, 2, h)[at].float()
    v = c["V"].reshape(-1, d)[at].float()
    lam = c["lam"].repeat_interleave(n // S)[:, None]
    s = torch.where(ok[..., None], scale * (q * k).sum(3), -math.inf)
    top = s.amax(1, keepdim=True)
    e = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    p = e / e.sum(1, keepdim=True).clamp(min=1e-30)  # no key at all: zeros
    a = p[..., 0] - lam * p[..., 1]
    if c["op"] == "attend":
        return (a[..., None] * v).sum(1).reshape(c["Q"].shape).to(c["Q"].dtype)
    do = c["dO"].reshape(n, 1, d).float()
    dp = (do * v).sum(2)[..., None]
    D = (p * dp).sum(1, keepdim=True)
    ds = scale * p * (dp - D) * torch.stack([torch.ones_like(lam), -lam], 2)
    dQ = (ds[..., None] * k).sum(1)
    dK = torch.zeros(c["K"].numel() // d, d, device=_DEVICE).index_add_(0, at.reshape(-1), (ds[..., None] * q).reshape(-1, d))
    dV = torch.zeros(c["V"].numel() // d, d, device=_DEVICE).index_add_(0, at.reshape(-1), (a[..., None] * do).reshape(-1, d))
    return dQ.reshape(c["Q"].shape), dK.reshape(c["K"].shape), dV.reshape(c["V"].shape), -D[:, 0, 1].reshape(S, -1).sum(1)


def _angles(c):
    """Angle of every pair in 64 bits: [slices (or 1), T, H, W, 1, pairs]."""
    nt, nh, nw = _sections(c)
    f = lambda m: 10000.0 ** (-torch.arange(m, device=_DEVICE, dtype=torch.float64) / max(m, 1))  # noqa: E731
    at = lambda axis, m, *s: (c["origin"][:, axis, None] + torch.arange(m, device=_DEVICE)).double().reshape(-1, *s, 1, 1)  # noqa: E731
    whole = lambda x: x.expand(-1, c["T"], c["H"], c["W"], -1, -1)  # noqa: E731
    return torch.cat([whole(at(0, c["T"], c["T"], 1, 1) * f(nt)), whole(at(1, c["H"], 1, c["H"], 1) * f(nh)),
                      whole(at(2, c["W"], 1, 1, c["W"]) * f(nw))], 5)


def _plain_rotary(c):
    angle = _angles(c) * (1.0 if c["op"] == "rotary" else -1.0)
    cos, sin, P = angle.cos().float(), angle.sin().float(), sum(_sections(c))

    def turn(x):
        y = x.reshape(*x.shape[:4], c["groups"], -1).float()
        a, b = (y[..., 0:2 * P:2], y[..., 1:2 * P:2]) if c["interleaved"] else (y[..., :P], y[..., P:2 * P])
        a, b = a * cos - b * sin, a * sin + b * cos
        front = torch.stack([a, b], 6).flatten(5) if c["interleaved"] else torch.cat([a, b], 5)
        return torch.cat([front, y[..., 2 * P:]], 5).reshape(x.shape).to(x.dtype)

    return tuple(map(turn, c["X"])) if c["tensors"] > 1 else turn(c["X"][0])


def _plain_norm(c):
    x = c["X"].float()
    w = c["weight"].float() if c["affine"] else 1.0
    if c["op"] == "norm":
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = torch.rsqrt((x * x).mean(1) + 1e-5)
        y = x * rstd[:, None] * w + (c["bias"].float() if c["affine"] else 0.0)
        return y.to(c["X"].dtype), mean, rstd
    dy, r = c["dY"].float(), c["rstd"][:, None]
    xh = (x - c["mean"][:, None]) * r
    g = dy * w
    dx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx.to(c["dY"].dtype), (dy * xh).sum(0), dy.sum(0)


def run(state):
    if own:
        return _own(state)
    if state["op"].startswith("attend"):
        return _plain_attend(state)
    return _plain_rotary(state) if state["op"].startswith("rotary") else _plain_norm(state)


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"].startswith("attend"):
        d, q, k = c["d"], c["S"] * c["Hq"] * c["Wq"], c["S"] * c["Hk"] * c["Wk"]
        keys = c["kappa"] * c["window"] ** 2
        # a key outside every window need not be read; its gradient is written all the same
        read = min(k, q * keys) * 2 * d * e + q * d * e + 4 * c["kappa"] * q + 4 * c["S"]
        if c["op"] == "attend":
            return {"bytes": read + q * d * e, "flops": 4 * d * keys * q}
        return {"bytes": read + q * d * e + 4 * d * q + 8 * d * k + 4 * c["S"], "flops": 10 * d * keys * q}
    if c["op"].startswith("rotary"):
        n = c["tensors"] * c["S"] * c["T"] * c["H"] * c["W"] * c["d"]
        return {"bytes": 2 * n * e, "flops": 3 * n}
    n, g, w = c["rows"] * c["channels"], 2 if c["grad"] == "bf16" else 4, c["channels"] * c["affine"] * e
    if c["op"] == "norm":
        return {"bytes": 2 * n * e + 8 * c["rows"] + 2 * w, "flops": 8 * n}
    return {"bytes": n * (e + 2 * g) + 8 * c["rows"] + 8 * c["channels"] + w, "flops": 14 * n}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def _exact_attend(c):
    """A window at a time over the query grid, as two dense-looking softmaxes; gradients by differentiation."""
    S, Hk, Wk, h, b = c["S"], c["Hk"], c["Wk"], c["d"] // 2, c["window"] // 2
    plane = c["Hq"] * c["Wq"]
    Q, K, V, dO = (c[k].reshape(-1, c["d"]).double() for k in ("Q", "K", "V", "dO"))
    lam, maps = c["lam"].double(), c["maps"].reshape(c["kappa"], -1).long()
    grads = c["op"] == "attend_backward"
    leaves = [t.requires_grad_(grads) for t in (Q, K, V, lam)]
    total = [torch.zeros_like(t) for t in leaves]
    out = torch.zeros_like(Q)
    # the union of the windows as a list of flat keys per query, each once
    size = max(1, (1 << 27) // (c["kappa"] * c["window"] ** 2 * c["d"]))
    for lo in range(0, S * plane, size):
        i = torch.arange(lo, min(lo + size, S * plane), device=_DEVICE)
        base, keys, good = i // plane * (Hk * Wk), [], []
        for e in range(c["kappa"]):
            for a in range(-b, b + 1):
                for o in range(-b, b + 1):
                    u, v = maps[e, i] // Wk + a, maps[e, i] % Wk + o
                    ok = (u >= 0) & (u < Hk) & (v >= 0) & (v < Wk)
                    if c["causal"]:
                        ok = ok & (u * Wk + v <= c["first"] + i % plane)
                    keys.append(torch.where(ok, u * Wk + v, -1))
        keys = torch.stack(keys, 1).sort(1).values  # a key of several windows stands in neighbouring places
        good = (keys >= 0) & torch.cat([torch.ones_like(keys[:, :1], dtype=torch.bool), keys[:, 1:] != keys[:, :-1]], 1)
        at = base[:, None] + keys.clamp(min=0)
        k, q = K[at], Q[i]
        bias = torch.zeros(keys.shape, dtype=torch.float64, device=_DEVICE).masked_fill(~good, -1e300)
        p = [torch.softmax((k[..., s] * q[:, None, s]).sum(2) / math.sqrt(h) + bias, 1) * good for s in (slice(0, h), slice(h, 2 * h))]
        o = ((p[0] - lam[i // plane][:, None] * p[1])[..., None] * V[at]).sum(1)
        if grads:
            for t, g in zip(total, torch.autograd.grad(o, leaves, dO[i])):
                t += g
        else:
            out[i] = o.detach()
    if not grads:
        return out.reshape(c["Q"].shape)
    return tuple(t.reshape(c[k].shape) for t, k in zip(total, ("Q", "K", "V", "lam")))


def _exact_rotary(c):
    """Pairs as complex numbers, turned one axis at a time."""
    nt, nh, nw = _sections(c)
    sign = 1.0 if c["op"] == "rotary" else -1.0
    got = []
    for x in c["X"]:
        y = x.reshape(*x.shape[:4], c["groups"], -1).double().clone()
        done = 0
        for axis, (m, n) in enumerate(((nt, c["T"]), (nh, c["H"]), (nw, c["W"]))):
            pos = c["origin"][:, axis].double()[:, None] + torch.arange(n, device=_DEVICE, dtype=torch.float64)
            for j in range(m):
                a = sign * pos * math.exp(-math.log(10000.0) * j / m)
                z = torch.polar(torch.ones_like(a), a).reshape(-1, *[n if k == axis else 1 for k in range(3)], 1)
                i0, i1 = (2 * done, 2 * done + 1) if c["interleaved"] else (done, done + nt + nh + nw)
                z = z * torch.complex(y[..., i0], y[..., i1])
                y[..., i0], y[..., i1] = z.real, z.imag
                done += 1
        got.append(y.reshape(x.shape))
    return tuple(got) if c["tensors"] > 1 else got[0]


def _exact_norm(c):
    x = c["X"].double()
    w = c["weight"].double() if c["affine"] else torch.ones_like(x[0])
    if c["op"] == "norm":
        var, mean = torch.var_mean(x, 1, unbiased=False)
        y = (x - mean[:, None]) / (var + 1e-5).sqrt()[:, None] * w + (c["bias"].double() if c["affine"] else 0.0)
        return y, mean, 1.0 / (var + 1e-5).sqrt()
    # the row's Jacobian (the statistics are inputs of the call): g less its projections on 1 and on xh
    dy, rows = c["dY"].double(), x.shape[1]
    xh = torch.addcmul(-c["mean"].double()[:, None] * c["rstd"].double()[:, None], x, c["rstd"].double()[:, None])
    g = dy * w
    along = torch.stack([torch.ones_like(xh), xh], 1)
    dx = (g - (torch.matmul(along, g[..., None]) * along).sum(1) / rows) * c["rstd"].double()[:, None]
    return dx, torch.matmul(dy.t()[:, None], xh.t()[..., None]).reshape(-1), torch.matmul(torch.ones_like(dy[:, 0]), dy)


def exact(case, seed):
    c = prepare(case, seed)
    if c["op"].startswith("attend"):
        return _exact_attend(c)
    return _exact_rotary(c) if c["op"].startswith("rotary") else _exact_norm(c)
