"""Timed calls of the operators for grids small enough to attend to every key: dense attention with a learned bias by
relative position, that bias by buckets of distance, group norm with an activation, each with its gradients.

Each case is one call.  ``run`` computes it with the package where ``own`` is true, otherwise in its plain form: elementary
torch operations in 32 bits, rounded once at the end.  ``exact`` computes the same in 64 bits.

Attention inputs: rows of order one, each query near the key of a place some pixels from its own, by as much as gives that
key about as much weight as all others together (less where the channels are few).  Biases fall off with the distance.
"""
import math

import torch

own = False

_DEVICE = "cuda"
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _attend(op, name=None, **kw):
    """S slices of queries on an Hq x Wq grid, S / share slices of keys on an Hk x Wk one.  ``place``: "" queries at the keys'
    own places from 0 on, "each" a run of them per slice at a place of its own.  ``fill``: keys that count differ per slice."""
    c = dict(op=op, S=1, share=1, Hq=32, Wq=32, Hk=0, Wk=0, d=64, dtype="bf16", bias=0, causal=False, place="", fill=False)
    c.update(kw)
    c["Hk"], c["Wk"] = c["Hk"] or c["Hq"], c["Wk"] or c["Wq"]
    return dict(c, name=name) if name else c


def _relative(op, name=None, **kw):
    c = dict(op=op, heads=8, H=64, W=64, near=8, far=8, dtype="bf16")
    c.update(kw)
    return dict(c, name=name) if name else c


def _group(op, name=None, **kw):
    c = dict(op=op, N=2, H=32, W=32, C=64, groups=8, dtype="bf16", grad="bf16", affine=True, act="silu")
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new pixel of each of 4 x 16 slices, two query heads to a key head, each image at a place of its own: latency counts
        _attend("attend", "attend_pixel", S=64, share=2, Hq=1, Wq=1, Hk=64, Wk=64, bias=16, causal=True, place="each"),
        # an image's pixels against a caption's features, padded to the longest of the batch, 32-bit
        _attend("attend", "attend_caption", S=16, Hq=64, Wq=64, Hk=1, Wk=157, d=32, dtype="f32", fill=True),
        # a coarse level of an image model: 2 x 8 heads of a 32 x 32 grid, with a learned bias
        _attend("attend", "attend_coarse", S=16, Hq=32, Wq=32, bias=8),
        # four heads of a 128 x 128 image: the whole map that the windows approximate
        _attend("attend", "attend_self128", S=4, Hq=128, Wq=128),
        # a training step's gradients, 2 x 8 heads of a 64 x 64 grid, those of the bias among them
        _attend("attend_backward", "attend_grad_self64", S=16, Hq=64, Wq=64, bias=8),
        # gradients of an autoregressive layer over one long row of pixels, four query heads to a key head
        _attend("attend_backward", "attend_grad_row", S=16, share=4, Hq=1, Wq=2500, d=128, causal=True),
        # the bias of 8 heads on a 64 x 64 grid from its table, every training step
        _relative("relative", "relative_self64"),
        # the table's gradient from that of a 128 x 128 grid's bias, 16 heads, 32-bit
        _relative("relative_backward", "relative_grad_self128", heads=16, H=128, W=128, near=6, far=10, dtype="f32"),
        # the smallest level of an image model: launches and host time count
        _group("group", "group_tiny", N=2, H=8, W=8, C=256, groups=32),
        # the finest level
        _group("group", "group_self256", N=4, H=256, W=256, C=128, groups=32),
        # a training step's gradients, half way down
        _group("group_backward", "group_grad_self128", N=4, H=128, W=128, C=256, groups=32),
        # gradients of ragged images, groups of five channels, 32-bit, no activation
        _group("group_backward", "group_grad_ragged", N=3, H=93, W=125, C=100, groups=20, dtype="f32", grad="f32", act=""),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(["attend", "attend", "attend", "attend_backward", "attend_backward", "attend_backward", "relative", "relative_backward",
                     "group", "group", "group_backward", "group_backward"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op.startswith("attend"):
        d, share = rng.choice([16, 20, 32, 64, 64, 128]), rng.choice([1, 1, 1, 2, 3])
        heads, kind = rng.choice([1, 2, 4]), rng.random()
        S = heads * share * log(1, 8)
        H = log(2, 128)
        W = max(1, min(160, int(H * math.exp(rng.uniform(-0.9, 0.9)))))
        kw = dict(S=S, share=share, d=d, dtype=dtype)
        if kind < 0.2:  # another grid's keys, padded
            kw.update(Hq=H, Wq=W, Hk=rng.choice([1, max(1, H // 2), H + 3]), Wk=log(1, 300), fill=rng.random() < 0.6)
        elif kind < 0.35:  # one long row
            kw.update(Hq=1, Wq=log(2, 9000), causal=rng.random() < 0.6, bias=rng.choice([0, 0, heads]))
        elif kind < 0.55 and op == "attend":  # the next pixels of one row, a place for each image
            kw.update(Hq=1, Wq=rng.choice([1, 1, 2, 7]), Hk=H, Wk=W + 8, causal=True, place="each", bias=rng.choice([0, heads]))
        else:
            kw.update(Hq=H, Wq=W, causal=rng.random() < 0.3, bias=rng.choice([0, heads, heads]))
        c = _attend(op, **kw)
        while c["S"] * c["Hq"] * c["Wq"] * c["Hk"] * c["Wk"] * max(d, 64) * (2.5 if op != "attend" else 1) > 4 * 16384 ** 2 * 64:
            if c["S"] > heads * share:
                c["S"] = max(1, c["S"] // (2 * heads * share)) * heads * share
            else:
                for k in ("Hq", "Wq", "Hk", "Wk"):
                    c[k] = max(1, c[k] * 3 // 4)
                if (kw["Hq"], kw["Wq"]) == (kw.get("Hk", kw["Hq"]), kw.get("Wk", kw["Wq"])):
                    c["Hk"], c["Wk"] = c["Hq"], c["Wq"]
        return c
    if op.startswith("relative"):
        H = log(1, 256)
        W = max(1, min(400, int(H * math.exp(rng.uniform(-0.7, 0.7))))) if rng.random() < 0.8 else log(2, 8000)
        H = H if W <= 400 else 1
        return _relative(op, heads=rng.choice([1, 4, 6, 8, 16, 32]), H=H, W=W, near=rng.choice([0, 2, 4, 8, 13]), far=rng.choice([1, 4, 8, 16]), dtype=dtype)
    width, groups = rng.choice([1, 2, 4, 4, 5, 8, 16, 24]), rng.choice([1, 4, 8, 16, 32, 32])
    N, H = log(1, 16), log(2, 256)
    W = max(1, min(320, int(H * math.exp(rng.uniform(-0.7, 0.7)))))
    while N * H * W * width * groups > 4 * 256 * 256 * 128 // (2 if op != "group" else 1):
        N, H, W = (max(1, N // 2), H, W) if N > 1 else (1, max(1, H * 3 // 4), max(1, W * 3 // 4))
    return _group(op, N=N, H=H, W=W, C=width * groups, groups=groups, dtype=dtype, grad=rng.choice([dtype, "f32"]),
                  affine=rng.random() < 0.8, act=rng.choice(["", "silu", "silu"]))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _spread(n, lo, hi, gen):
    """n whole numbers spread evenly over lo .. hi, in an order of the seed's."""
    at = torch.linspace(lo, hi, n, dtype=torch.float64).round().to(torch.int32).to(_DEVICE)
    return at[torch.randperm(n, generator=gen, device=_DEVICE)]


def _edges(near, far, span):
    """The distances at which the buckets of one side of an axis begin: 1, 2, .., near, then ``far`` of them in equal ratios to
    the axis' span."""
    e = list(range(1, near + 1))
    for j in range(1, far + 1):
        e.append(max(int(max(near, 1) * (max(span, 2) / max(near, 1)) ** (j / (far + 1))), (e[-1] if e else 0) + 1))
    return tuple(e)


def _attend_inputs(c, gen):
    S, Sk, Hq, Wq, Hk, Wk, d = c["S"], c["S"] // c["share"], c["Hq"], c["Wq"], c["Hk"], c["Wk"], c["d"]
    nq, nk, kind = Hq * Wq, Hk * Wk, _TYPES[c["dtype"]]
    normal = lambda *s: torch.randn(*s, generator=gen, device=_DEVICE)  # noqa: E731
    K = normal(Sk, nk, d)
    x = dict(first=None, lengths=None, bias=None)
    start = torch.zeros(S, 1, dtype=torch.long, device=_DEVICE)
    if c["place"]:  # the slices of one image's heads stand at the same place
        images = max(1, S // max(1, c["bias"] or c["share"]))
        x["first"] = _spread(images, nk // 2, nk - nq, gen).clamp(0, nk - nq).repeat_interleave(S // images)
        start = x["first"].long()[:, None]
    own_at = start + torch.arange(nq, device=_DEVICE) * (1 if c["place"] else nk) // (1 if c["place"] else nq)
    far = torch.randint(-2 * Wk - 2, 3, (S, nq), generator=gen, device=_DEVICE)
    target = (own_at + far).clamp(0, nk - 1)
    rows = K.repeat_interleave(c["share"], 0)
    seen = own_at.double() + 1.0 if c["causal"] else torch.full_like(own_at, nk, dtype=torch.float64)
    near = ((seen.log() + 0.5) / d ** 0.5).clamp(max=1.0).float()[..., None]
    Q = 0.7 * normal(S, nq, d) + near * torch.gather(rows, 1, target[..., None].expand(-1, -1, d))
    x["Q"], x["K"] = Q.reshape(S, Hq, Wq, d).to(kind), K.reshape(Sk, Hk, Wk, d).to(kind)
    x["V"] = normal(Sk, Hk, Wk, d).to(kind)
    if c["fill"]:
        x["lengths"] = _spread(Sk, (nk + 1) // 2, nk, gen)
    if c["bias"]:
        y, z = (torch.arange(1 - n, n, device=_DEVICE).abs().float() for n in (Hk, Wk))
        slope = 0.02 + 0.3 * torch.rand(c["bias"], 1, 1, generator=gen, device=_DEVICE)
        x["bias"] = (0.3 * normal(c["bias"], 2 * Hk - 1, 2 * Wk - 1) - slope * torch.log1p(y[:, None] + z) * 2.0).to(kind)
    if c["op"] == "attend_backward":
        x["dO"] = normal(S, Hq, Wq, d).to(kind)
    return x


def prepare(case, seed):
    gen = torch.Generator(device=_DEVICE).manual_seed(int(seed))
    c = dict(case)
    if c["op"].startswith("attend"):
        return dict(c, **_attend_inputs(c, gen))
    kind = _TYPES[c["dtype"]]
    normal = lambda *s: torch.randn(*s, generator=gen, device=_DEVICE)  # noqa: E731
    if c["op"].startswith("relative"):
        c["edges"] = (_edges(c["near"], c["far"], c["H"]), _edges(c["near"], c["far"], c["W"]))
        sides = [2 * (c["near"] + c["far"]) + 1] * 2
        if c["op"] == "relative":
            c["table"] = normal(c["heads"], *sides).to(kind)
        else:
            c["dbias"] = normal(c["heads"], 2 * c["H"] - 1, 2 * c["W"] - 1).to(kind)
        return c
    # activations: an offset and a spread of their own in every image and channel
    shape = (c["N"], c["H"], c["W"], c["C"])
    x = normal(*shape) * (0.5 + torch.rand(c["N"], 1, 1, c["C"], generator=gen, device=_DEVICE)) + normal(c["N"], 1, 1, c["C"])
    c["X"] = x.to(kind)
    c["weight"] = (1.0 + 0.2 * normal(c["C"])).to(kind) if c["affine"] else None
    c["bias"] = (0.2 * normal(c["C"])).to(kind) if c["affine"] else None
    if c["op"] == "group_backward":  # what the forward pass left
        c["dY"] = normal(*shape).to(_TYPES[c["grad"]])
        var, mean = torch.var_mean(c["X"].reshape(c["N"], -1, c["groups"], c["C"] // c["groups"]).double(), (1, 3), unbiased=False)
        c["mean"], c["rstd"] = mean.float(), torch.rsqrt(var + 1e-5).float()
    return c


# ---------------------------------------------------------------------------
# one call
# ---------------------------------------------------------------------------
def _own(c):
    import paper_1905_10308_amd as scram

    if c["op"].startswith("attend"):
        kw = dict(bias=c["bias"], causal=c["causal"], first=0 if c["first"] is None else c["first"], lengths=c["lengths"])
        if c["op"] == "attend":
            return scram.dense_attend(c["Q"], c["K"], c["V"], **kw)
        return scram.dense_attend_backward(c["Q"], c["K"], c["V"], c["dO"], **kw)
    if c["op"] == "relative":
        return scram.relative_bias(c["table"], c["H"], c["W"], edges=c["edges"])
    if c["op"] == "relative_backward":
        return scram.relative_bias_backward(c["dbias"], edges=c["edges"])
    if c["op"] == "group":
        return scram.group_norm(c["X"], c["groups"], c["weight"], c["bias"], activation=c["act"] or None, stats=True)
    return scram.group_norm_backward(c["dY"], c["X"], c["mean"], c["rstd"], c["weight"], c["bias"], activation=c["act"] or None)


def _offsets(c):
    """Flat place in a head's bias of every (query, key) pair: [1 or S, nq, nk]."""
    Hk, Wk = c["Hk"], c["Wk"]
    at = torch.arange(c["Hq"] * c["Wq"], device=_DEVICE)[None]
    if c["first"] is not None:
        at = at + c["first"].long()[:, None]
    k = torch.arange(Hk * Wk, device=_DEVICE)
    flat = lambda p: p // Wk * (2 * Wk - 1) + p % Wk  # noqa: E731
    return flat(k) - flat(at)[..., None] + (Hk - 1) * (2 * Wk - 1) + Wk - 1


def _plain_weights(c):
    """Softmax weights [S, nq, nk] of every query; zeros where it sees no key."""
    S, share, nq, nk, d = c["S"], c["share"], c["Hq"] * c["Wq"], c["Hk"] * c["Wk"], c["d"]
    q, k = c["Q"].reshape(S // share, share * nq, d).float(), c["K"].reshape(S // share, nk, d).float()
    s = torch.matmul(q, k.transpose(1, 2).contiguous()).reshape(S, nq, nk) * d ** -0.5
    if c["bias"] is not None:
        at, heads = _offsets(c), c["bias"].shape[0]
        table = c["bias"].reshape(heads, -1).float()
        if at.shape[0] == 1:
            s = (s.reshape(S // heads, heads, nq, nk) + table[:, at[0]]).reshape(S, nq, nk)
        else:
            s = s + table[(torch.arange(S, device=_DEVICE) % heads)[:, None, None], at]
    j = torch.arange(nk, device=_DEVICE)
    if c["causal"]:
        at = torch.arange(nq, device=_DEVICE)[None] if c["first"] is None else c["first"][:, None] + torch.arange(nq, device=_DEVICE)
        s = torch.where(j <= at[..., None], s, -math.inf)
    if c["lengths"] is not None:
        s = torch.where(j < c["lengths"].repeat_interleave(share)[:, None, None], s, -math.inf)
    top = s.amax(2, keepdim=True)
    e = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(2, keepdim=True)
    return e / torch.where(total == 0.0, 1.0, total)


def _plain_attend(c):
    v = c["V"].reshape(c["V"].shape[0], -1, c["d"]).float()
    p = _plain_weights(c).reshape(v.shape[0], -1, v.shape[1])
    return torch.matmul(p, v).reshape(c["Q"].shape).to(c["Q"].dtype)


def _plain_attend_backward(c):
    S, share, nq, nk, d = c["S"], c["share"], c["Hq"] * c["Wq"], c["Hk"] * c["Wk"], c["d"]
    Sk, kind = S // share, c["Q"].dtype
    p = _plain_weights(c).reshape(Sk, share * nq, nk)
    q, do = (c[n].reshape(Sk, share * nq, d).float() for n in ("Q", "dO"))
    k, v = (c[n].reshape(Sk, nk, d).float() for n in ("K", "V"))
    dV = torch.matmul(p.transpose(1, 2).contiguous(), do)
    dp = torch.matmul(do, v.transpose(1, 2).contiguous())
    ds = p * (dp - (p * dp).sum(2, keepdim=True))
    del p, dp
    dQ = torch.matmul(ds, k) * d ** -0.5
    dK = torch.matmul(ds.transpose(1, 2).contiguous(), q) * d ** -0.5
    got = (dQ.reshape(c["Q"].shape).to(kind), dK.reshape(c["K"].shape).to(kind), dV.reshape(c["V"].shape).to(kind))
    if c["bias"] is None:
        return got
    heads = c["bias"].shape[0]
    each = ds.reshape(-1, heads, nq * nk).sum(0)
    dB = torch.zeros(heads, c["bias"][0].numel(), device=_DEVICE).index_add_(1, _offsets(c).reshape(-1), each)
    return (*got, dB.reshape(c["bias"].shape).to(kind))


def _buckets(n, edges):
    """The bucket of every offset 1 - n .. n - 1."""
    e = torch.tensor(edges, device=_DEVICE)
    off = torch.arange(1 - n, n, device=_DEVICE)
    return len(edges) + off.sign() * (e <= off.abs()[:, None]).sum(1)


def _plain_relative(c):
    by, bx = _buckets(c["H"], c["edges"][0]), _buckets(c["W"], c["edges"][1])
    ny, nx = (2 * len(e) + 1 for e in c["edges"])
    if c["op"] == "relative":
        return c["table"][:, by][:, :, bx].contiguous()
    # a cell of the far buckets adds up tens of thousands of numbers: 64 bits
    g = c["dbias"].double()
    got = torch.zeros(c["heads"], ny, g.shape[2], device=_DEVICE, dtype=torch.float64).index_add_(1, by, g)
    got = torch.zeros(c["heads"], ny, nx, device=_DEVICE, dtype=torch.float64).index_add_(2, bx, got)
    return got.to(c["dbias"].dtype)


def _plain_group(c):
    N, C, G = c["N"], c["C"], c["groups"]
    x = c["X"].reshape(N, -1, G, C // G).float()
    w = c["weight"].reshape(G, -1).float() if c["affine"] else 1.0
    b = c["bias"].reshape(G, -1).float() if c["affine"] else 0.0
    if c["op"] == "group":
        mean = x.mean((1, 3))
        x = x - mean[:, None, :, None]
        rstd = torch.rsqrt((x * x).mean((1, 3)) + 1e-5)
        y = x * rstd[:, None, :, None] * w + b
        y = y / (1.0 + torch.exp(-y)) if c["act"] else y
        return y.reshape(c["X"].shape).to(c["X"].dtype), mean, rstd
    r = c["rstd"][:, None, :, None]
    xh = (x - c["mean"][:, None, :, None]) * r
    dy = c["dY"].reshape(x.shape).float()
    if c["act"]:
        z = xh * w + b
        sig = 1.0 / (1.0 + torch.exp(-z))
        dy = dy * sig * (1.0 + z * (1.0 - sig))
    g = dy * w
    dx = r * (g - g.mean((1, 3), keepdim=True) - xh * (g * xh).mean((1, 3), keepdim=True))
    return dx.reshape(c["X"].shape).to(c["dY"].dtype), (dy * xh).sum((0, 1)).reshape(C), dy.sum((0, 1)).reshape(C)


def run(state):
    if own:
        return _own(state)
    if state["op"] == "attend":
        return _plain_attend(state)
    if state["op"] == "attend_backward":
        return _plain_attend_backward(state)
    return _plain_relative(state) if state["op"].startswith("relative") else _plain_group(state)


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"].startswith("attend"):
        S, Sk, d, nq, nk = c["S"], c["S"] // c["share"], c["d"], c["Hq"] * c["Wq"], c["Hk"] * c["Wk"]
        first = (nk // 2 + nk - nq) / 2 if c["place"] else 0.0  # the mean over the slices
        seen = first + (nq + 1) / 2 if c["causal"] else 0.75 * nk if c["fill"] else nk
        keys = min(nk, first + nq) if c["causal"] else 0.75 * nk if c["fill"] else nk  # those that some query sees
        bias = c["bias"] * (2 * c["Hk"] - 1) * (2 * c["Wk"] - 1)
        bias = min(bias, S * nq * seen) if nq < nk else bias
        read = (S * nq + 2 * Sk * keys) * d * e + bias * e
        if c["op"] == "attend":
            return {"bytes": read + S * nq * d * e, "flops": 4 * d * S * nq * seen}
        # dO and the gradients (of keys that do not count too)
        return {"bytes": read + 2 * S * nq * d * e + 2 * Sk * nk * d * e + bias * e, "flops": 10 * d * S * nq * seen}
    if c["op"].startswith("relative"):
        n = c["heads"] * (2 * c["H"] - 1) * (2 * c["W"] - 1)
        return {"bytes": (n + c["heads"] * (2 * (c["near"] + c["far"]) + 1) ** 2) * e, "flops": n}
    n, g, w = c["N"] * c["H"] * c["W"] * c["C"], 2 if c["grad"] == "bf16" else 4, 2 * c["C"] * c["affine"] * e
    if c["op"] == "group":
        return {"bytes": 2 * n * e + 8 * c["N"] * c["groups"] + w, "flops": 8 * n + 4 * n * bool(c["act"])}
    return {"bytes": n * (e + 2 * g) + 8 * c["N"] * c["groups"] + 8 * c["C"] + w, "flops": 14 * n + 10 * n * bool(c["act"])}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def _exact_attend(c):
    """A run of queries of one slice at a time; gradients by differentiation."""
    S, share, nq, Hk, Wk, d = c["S"], c["share"], c["Hq"] * c["Wq"], c["Hk"], c["Wk"], c["d"]
    nk, grads = Hk * Wk, c["op"] == "attend_backward"
    heads = 0 if c["bias"] is None else c["bias"].shape[0]
    wide = lambda t: None if t is None else t.double()  # noqa: E731
    Q, K, V, B = wide(c["Q"].reshape(S, nq, d)), wide(c["K"].reshape(-1, nk, d)), wide(c["V"].reshape(-1, nk, d)), wide(c["bias"])
    out = torch.zeros_like(Q)
    dQ, dK, dV = torch.zeros_like(Q), torch.zeros_like(K), torch.zeros_like(V)
    dB = None if B is None else torch.zeros_like(B)
    j = torch.arange(nk, device=_DEVICE)
    for s in range(S):
        begin = 0 if c["first"] is None else int(c["first"][s])
        live = nk if c["lengths"] is None else int(c["lengths"][s // share])
        size = max(1, (1 << 27) // nk)
        for lo in range(0, nq, size):
            i = torch.arange(lo, min(lo + size, nq), device=_DEVICE)
            leaves = [Q[s, i], K[s // share], V[s // share]] + ([B[s % heads]] if heads else [])
            leaves = [t.clone().requires_grad_(grads) for t in leaves]
            q, k, v = leaves[:3]
            a = q @ k.t() / math.sqrt(d)
            at = begin + i
            if heads:
                a = a + leaves[3][(j // Wk)[None] - (at // Wk)[:, None] + Hk - 1, (j % Wk)[None] - (at % Wk)[:, None] + Wk - 1]
            hidden = (j >= live)[None].expand(len(i), -1)
            if c["causal"]:
                hidden = hidden | (j[None] > at[:, None])
            o = torch.softmax(a.masked_fill(hidden, -math.inf), 1).masked_fill(hidden, 0.0) @ v
            if not grads:
                out[s, i] = o
                continue
            got = torch.autograd.grad(o, leaves, c["dO"].reshape(S, nq, d)[s, i].double())
            dQ[s, i] = got[0]
            dK[s // share] += got[1]
            dV[s // share] += got[2]
            if heads:
                dB[s % heads] += got[3]
    if not grads:
        return out.reshape(c["Q"].shape)
    return (dQ.reshape(c["Q"].shape), dK.reshape(c["K"].shape), dV.reshape(c["V"].shape), *([dB] if heads else []))


def _exact_relative(c):
    """An axis at a time, as a product with the matrix of ones where an offset has a bucket."""
    hot = []
    for n, edges in zip((c["H"], c["W"]), c["edges"]):
        m = torch.zeros(2 * len(edges) + 1, 2 * n - 1, dtype=torch.float64)
        for off in range(1 - n, n):
            b = sum(1 for e in edges if e <= abs(off))
            m[len(edges) + (b if off > 0 else -b), off + n - 1] = 1.0
        hot.append(m.to(_DEVICE))
    if c["op"] == "relative":
        return torch.stack([hot[0].t() @ t @ hot[1] for t in c["table"].double()])
    return torch.stack([hot[0] @ t @ hot[1].t() for t in c["dbias"].double()])


def _exact_group(c):
    N, C, G = c["N"], c["C"], c["groups"]
    x = c["X"].double().reshape(N, -1, G, C // G).transpose(1, 2).reshape(N, G, -1)
    w = (c["weight"].double() if c["affine"] else torch.ones(C, dtype=torch.float64, device=_DEVICE)).requires_grad_(True)
    b = (c["bias"].double() if c["affine"] else torch.zeros(C, dtype=torch.float64, device=_DEVICE)).requires_grad_(True)
    back = lambda t: t.reshape(N, G, -1, C // G).transpose(1, 2).reshape(c["X"].shape)  # noqa: E731
    act = torch.nn.functional.silu if c["act"] else (lambda t: t)
    if c["op"] == "group":
        var, mean = torch.var_mean(x, 2, unbiased=False)
        y = back((x - mean[..., None]) / (var + 1e-5).sqrt()[..., None]) * w + b
        return act(y).detach(), mean, 1.0 / (var + 1e-5).sqrt()
    # the statistics are inputs of the call: the group's Jacobian projects off 1 and xh
    r, m = c["rstd"].double()[..., None], c["mean"].double()[..., None]
    xh = back((x - m) * r).requires_grad_(True)
    g, dw, db = torch.autograd.grad(act(xh * w + b), (xh, w, b), c["dY"].double())
    g = g.reshape(N, -1, G, C // G).transpose(1, 2).reshape(N, G, -1)
    flat = (x - m) * r
    dx = (g - g.mean(2, keepdim=True) - flat * (g * flat).mean(2, keepdim=True)) * r
    return back(dx), dw, db


def exact(case, seed):
    c = prepare(case, seed)
    if c["op"].startswith("attend"):
        return _exact_attend(c)
    return _exact_relative(c) if c["op"].startswith("relative") else _exact_group(c)
