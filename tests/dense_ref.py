"""Plain 64-bit definitions of attention over every key, its bias by buckets and group norm (no test functions here).

Beside each result stands how far a computation in 32 bits (with weights and score gradients rounded to bf16 for
their products, where the rows are bf16) may be off, from the sums of the absolute values of what was added up.
"""
import math

import torch

U32 = 2.0 ** -24  # half a step of fp32, relative
HALF = {torch.float32: U32, torch.bfloat16: 2.0 ** -8}
#: fp32 holds nothing under 2^-126 in full: a weight that small, or its product with another factor, may come out as 0
TINY = 8 * 2.0 ** -126


def places(S, Hq, Wq, Wk, first, device):
    """Row and column on the key grid of every query: two of [S, nq]."""
    start = torch.as_tensor(first, device=device).long().expand(S)
    at = start[:, None] + torch.arange(Hq * Wq, device=device)
    return at // Wk, at % Wk, at


def scores(Q, K, scale, bias, causal, first, lengths):
    """[S, nq, nk] scores, minus infinity where a key is not seen; and the sum of their parts' absolute values."""
    S, Hq, Wq, d = Q.shape
    Sk, Hk, Wk, _ = K.shape
    q = Q.reshape(S, -1, d).double()
    k = K.reshape(Sk, -1, d).double().repeat_interleave(S // Sk, 0)
    a = scale * (q @ k.transpose(1, 2))
    reach = abs(scale) * (q.abs() @ k.abs().transpose(1, 2))
    j = torch.arange(Hk * Wk, device=Q.device)
    if bias is not None or causal:
        y, x, at = places(S, Hq, Wq, Wk, first, Q.device)
    if bias is not None:
        head = (torch.arange(S, device=Q.device) % bias.shape[0])[:, None, None]
        b = bias.double()[head, j // Wk - y[..., None] + Hk - 1, j % Wk - x[..., None] + Wk - 1]
        a = a + b
        reach = reach + b.detach().abs().clamp(max=1e30)
    if causal:
        a = a.masked_fill(j > at[..., None], -math.inf)
    if lengths is not None:
        a = a.masked_fill(j >= lengths.long().repeat_interleave(S // Sk)[:, None, None], -math.inf)
    return a, reach


def attend(Q, K, V, scale=None, bias=None, causal=False, first=0, lengths=None):
    """[S, Hq, Wq, dv], differentiable; zeros where a query sees no key."""
    S, Hq, Wq, d = Q.shape
    scale = d ** -0.5 if scale is None else scale
    a, _ = scores(Q, K, scale, bias, causal, first, lengths)
    p = weights(a)
    v = V.reshape(V.shape[0], -1, V.shape[-1]).double().repeat_interleave(S // V.shape[0], 0)
    return (p @ v).reshape(S, Hq, Wq, -1)


def weights(a):
    none = (a == -math.inf).all(2, keepdim=True)
    return torch.softmax(a.masked_fill(none, 0.0), 2).masked_fill(none, 0.0)


def attend_all(Q, K, V, dO, scale=None, bias=None, causal=False, first=0, lengths=None):
    """(out, dQ, dK, dV[, dbias]) and as many tolerances."""
    S, Hq, Wq, d = Q.shape
    Sk, Hk, Wk, dv = V.shape
    g, nk, kind, dev = S // Sk, Hk * Wk, Q.dtype, Q.device
    half, low = HALF[kind], HALF[kind] if kind != torch.float32 else 0.0
    scale = d ** -0.5 if scale is None else scale
    a, reach = scores(Q, K, scale, bias, causal, first, lengths)
    p = weights(a)
    on = (a > -math.inf).double()
    q, do = (t.reshape(S, -1, t.shape[-1]).double() for t in (Q, dO))
    k, v = (t.reshape(Sk, nk, -1).double().repeat_interleave(g, 0) for t in (K, V))
    # a score: the products' sum, scaled, the bias added, the maximum or the sum's logarithm taken off
    # (keys that a bias of the lowest values hides have weight 0 in any arithmetic, unless they are all there is)
    off = U32 * (((d + 8) * reach) * (a > -1e30)).amax(2, keepdim=True) + 4 * (math.log2(nk) + 2) * U32
    # a weight: twice that (it and the sum), the exponentials and a sum over the keys, one after another
    rel = 2 * off + (nk + 24) * U32
    pv = p @ v.abs()
    out = p @ v
    out_tol = (rel + low + (nk + 4) * U32) * pv + half * out.abs() + TINY * (on @ v.abs())
    dp, dpa = do @ v.transpose(1, 2), do.abs() @ v.abs().transpose(1, 2)
    D, Da = (p * dp).sum(2, keepdim=True), (p * dpa).sum(2, keepdim=True)
    ds, dsa = p * (dp - D), p * (dpa + Da)
    ds_tol = (2 * rel + (2 * dv + 16) * U32) * dsa + TINY * on * (1 + dpa + Da)
    w_tol = ds_tol + low * (ds.abs() + ds_tol)  # as an operand of the products
    many = (g * q.shape[1] + 8) * U32
    keys = lambda x: x.reshape(Sk, g, nk, -1).sum(1)  # noqa: E731
    s = abs(scale)
    dQ, dK, dV = scale * (ds @ k), scale * keys(ds.transpose(1, 2) @ q), keys(p.transpose(1, 2) @ do)
    dQ_tol = s * ((w_tol + (nk + 8) * U32 * dsa) @ k.abs()) + half * dQ.abs()
    dK_tol = s * keys((w_tol + many * dsa).transpose(1, 2) @ q.abs()) + half * dK.abs()
    dV_tol = keys(((rel + low + many) * p + TINY * on).transpose(1, 2) @ do.abs()) + half * dV.abs()
    got, tol = [out.reshape(S, Hq, Wq, dv), dQ.reshape(Q.shape), dK.reshape(K.shape), dV.reshape(V.shape)], []
    tol = [t.reshape(x.shape) for t, x in zip((out_tol, dQ_tol, dK_tol, dV_tol), got)]
    if bias is not None:
        y, x, _ = places(S, Hq, Wq, Wk, first, dev)
        j = torch.arange(nk, device=dev)
        flat = (j // Wk - y[..., None] + Hk - 1) * (2 * Wk - 1) + j % Wk - x[..., None] + Wk - 1
        heads = bias.shape[0]
        flat = (flat + ((torch.arange(S, device=dev) % heads) * bias[0].numel())[:, None, None]).reshape(-1)
        add = lambda t: torch.zeros(bias.numel(), dtype=torch.float64, device=dev).index_add_(0, flat, t.reshape(-1)).reshape(bias.shape)  # noqa: E731
        dB = add(ds)
        got.append(dB)
        tol.append(add(ds_tol + (S // heads * Hq * Wq + 8) * U32 * dsa) + half * dB.abs())
    return got, tol


def buckets(n, edges):
    """Bucket of every offset 1 - n .. n - 1."""
    got = []
    for t in range(1 - n, n):
        k = sum(1 for e in edges if e <= abs(t))
        got.append(len(edges) + (k if t >= 0 else -k))
    return torch.tensor(got)


def relative_bias(table, H, W, edges):
    by, bx = (buckets(n, e).to(table.device) for n, e in zip((H, W), edges))
    return table[:, by][:, :, bx]


def relative_bias_backward(dbias, edges):
    """The table's gradient in 64 bits, and the sums of the absolute values."""
    H, W = (dbias.shape[1] + 1) // 2, (dbias.shape[2] + 1) // 2
    by, bx = (buckets(n, e).to(dbias.device) for n, e in zip((H, W), edges))
    shape = (dbias.shape[0], 2 * len(edges[0]) + 1, 2 * len(edges[1]) + 1)

    def add(x):
        rows = torch.zeros(shape[0], shape[1], x.shape[2], dtype=torch.float64, device=x.device).index_add_(1, by, x)
        return torch.zeros(shape, dtype=torch.float64, device=x.device).index_add_(2, bx, rows)

    return add(dbias.double()), add(dbias.double().abs())


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, act=None):
    """(result, mean, rstd), differentiable."""
    N, C = x.shape[0], x.shape[-1]
    y = x.double().reshape(N, -1, groups, C // groups)
    mean = y.mean((1, 3))
    var = ((y - mean[:, None, :, None]) ** 2).mean((1, 3))
    rstd = (var + eps) ** -0.5
    z = ((y - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(N, -1, C)
    z = z * (1.0 if weight is None else weight.double()) + (0.0 if bias is None else bias.double())
    return (z / (1.0 + torch.exp(-z)) if act else z).reshape(x.shape), mean, rstd


def group_norm_backward(dy, x, mean, rstd, weight=None, bias=None, act=None):
    """(dx, dweight, dbias) of the statistics given, and the sums of absolute values that they are held to."""
    N, C, G = x.shape[0], x.shape[-1], mean.shape[1]
    m, r = (t.double()[:, None, :, None] for t in (mean, rstd))
    xh = ((x.double().reshape(N, -1, G, C // G) - m) * r).reshape(N, -1, C)
    w = torch.ones(C, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    dz = dy.double().reshape(N, -1, C)
    if act:
        z = xh * w + (0.0 if bias is None else bias.double())
        sig = 1.0 / (1.0 + torch.exp(-z))
        dz = dz * sig * (1.0 + z * (1.0 - sig))
    parts = lambda t: t.reshape(N, -1, G, C // G)  # noqa: E731
    g = parts(dz * w)
    mg, mx = g.mean((1, 3), keepdim=True), (g * parts(xh)).mean((1, 3), keepdim=True)
    dx = r * (g - mg - parts(xh) * mx)
    ga = g.abs()
    reach = r * (ga + ga.mean((1, 3), keepdim=True) + parts(xh).abs() * (ga * parts(xh).abs()).mean((1, 3), keepdim=True))
    return ((dx.reshape(x.shape), (dz * xh).sum((0, 1)), dz.sum((0, 1))),
            (reach.reshape(x.shape), (dz * xh).abs().sum((0, 1)), dz.abs().sum((0, 1))))
