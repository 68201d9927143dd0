"""Plain 64-bit definitions of the operators around the attention (no test functions here).

Differential attention is computed densely: a truth value for every (query, key) pair of a slice says whether
the key is in the query's set.  Beside each result stands the sum of the absolute values of what was added up
for it, from which the tests derive how far a 32-bit computation may be off.
"""
import math

import torch

#: half a step of each type, relative to the value: one rounding is off by at most this
U32 = 2.0 ** -24
#: fp32 holds nothing under 2^-126 in full: a weight that small may come out as 0, and so may what is left of its
#: exponential, its product with the normaliser or with lam, its parts in fewer bits, and its score's gradient's three parts
TINY = 8 * 2.0 ** -126
HALF = {torch.float32: U32, torch.bfloat16: 2.0 ** -8}


def key_mask(maps, Hq, Wq, Hk, Wk, window, causal=False, first=None):
    """[S, n, keys] whether key j lies in the union of query i's windows; maps [kappa, S, Hq, Wq]."""
    kappa, S = maps.shape[:2]
    m = maps.reshape(kappa, S, -1).long().clamp(0, Hk * Wk - 1)
    j = torch.arange(Hk * Wk, device=maps.device)
    near = ((j // Wk - (m // Wk)[..., None]).abs() <= window // 2) & ((j % Wk - (m % Wk)[..., None]).abs() <= window // 2)
    mask = near.any(0)
    if causal:
        start = torch.zeros(S, dtype=torch.long, device=maps.device) if first is None else torch.as_tensor(first, device=maps.device).long().expand(S)
        mask &= j <= (start[:, None] + torch.arange(Hq * Wq, device=maps.device))[..., None]
    return mask


def differential(Q, K, V, mask, lam, scale, dO=None):
    """Output [S, n, dv] and its tolerance's sum; with dO also (dQ, dK, dV, dlam) and theirs."""
    S, d = Q.shape[0], Q.shape[-1]
    q, k, v = (t.reshape(S, -1, t.shape[-1]).double() for t in (Q, K, V))
    h, lam = d // 2, lam.double()[:, None, None]
    p, delta = [], 0.0
    for s in (slice(0, h), slice(h, d)):
        a = scale * (q[..., s] @ k[..., s].transpose(1, 2))
        p.append(torch.softmax(a.masked_fill(~mask, -math.inf), 2).nan_to_num(0.0))
        # a score: its products' sum (at most 12 roundings deep, 2 more for the scale in base 2 and the exponent's argument)
        reach = abs(scale) * (q[..., s].abs() @ k[..., s].abs().transpose(1, 2))
        delta = max(delta, float(reach.detach().masked_fill(~mask, 0.0).max()) * 14 * U32)
    w = p[0] - lam * p[1]
    pw = p[0] + lam.abs() * p[1]
    # a weight is off by twice its score's error (it and the normaliser) and by the exponentials' two roundings; the sums over
    # a query's keys by a rounding each, and a few for the products and the end
    rel = 2 * delta + (float(mask.sum(2).max()) + 24) * U32
    on = mask.double()
    out, out_tol = w @ v, rel * (pw @ v.abs()) + TINY * (1 + lam.abs()) * (on @ v.abs())
    if dO is None:
        return out, out_tol
    do = dO.reshape(S, -1, d if V.shape[-1] == d else V.shape[-1]).double()
    dp, dpa = do @ v.transpose(1, 2), do.abs() @ v.abs().transpose(1, 2)
    D, Da = [(x * dp).sum(2, keepdim=True) for x in p], [(x * dpa).sum(2, keepdim=True) for x in p]
    c = [torch.ones_like(lam), -lam]
    ds = [c[i] * p[i] * (dp - D[i]) * scale for i in (0, 1)]
    dsa = [c[i].abs() * p[i] * (dpa + Da[i]) * abs(scale) for i in (0, 1)]
    tiny = [TINY * on * (1 + c[i].abs() * (dpa + Da[i]) * abs(scale)) for i in (0, 1)]
    halves = (slice(0, h), slice(h, d))
    dQ = torch.cat([ds[i] @ k[..., s] for i, s in enumerate(halves)], 2)
    dK = torch.cat([ds[i].transpose(1, 2) @ q[..., s] for i, s in enumerate(halves)], 2)
    dV = w.transpose(1, 2) @ do
    dlam = -D[1].sum((1, 2))
    # dQ may be formed with a fixed vector taken off the keys: twice the largest key bounds what is added up
    kmax = k.abs().amax(1, keepdim=True)
    tol = rel + 16 * U32
    many = float(mask.sum(1).max()) * U32  # a key's queries, one after another
    dQ_tol = torch.cat([(3 * tol * dsa[i] + tiny[i]).sum(2, keepdim=True) * 2 * kmax[..., s] for i, s in enumerate(halves)], 2)
    dK_tol = torch.cat([((2 * tol + many) * dsa[i] + tiny[i]).transpose(1, 2) @ q[..., s].abs() for i, s in enumerate(halves)], 2)
    dV_tol = ((tol + many) * pw + TINY * (1 + lam.abs()) * on).transpose(1, 2) @ do.abs()
    dlam_tol = 2 * tol * Da[1].sum((1, 2))
    return out, out_tol, (dQ, dK, dV, dlam), (dQ_tol, dK_tol, dV_tol, dlam_tol)


def frequencies(sections, base=10000.0):
    return [base ** (-j / m) for m in sections for j in range(m)]


def rotary(x, sections, freqs, origin, groups=1, interleaved=False, inverse=False):
    """x [S, T, H, W, d], origin [S or 1, 3]: a pair at a time, in 64 bits."""
    y = x.double().reshape(*x.shape[:4], groups, -1).clone()
    P, k = sum(sections), 0
    for axis, m in enumerate(sections):
        n = x.shape[1 + axis]
        pos = origin[:, axis, None].double() + torch.arange(n, device=x.device, dtype=torch.float64)
        pos = pos.reshape(-1, *[n if a == axis else 1 for a in range(3)], 1)
        for _ in range(m):
            t = pos * freqs[k] * (-1.0 if inverse else 1.0)
            i, j = (2 * k, 2 * k + 1) if interleaved else (k, k + P)
            a, b = y[..., i].clone(), y[..., j].clone()
            y[..., i], y[..., j] = a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos()
            k += 1
    return y.reshape(x.shape)


def layer_norm(x, weight, bias, eps):
    x = x.double()
    mean = x.mean(-1)
    var = ((x - mean[..., None]) ** 2).mean(-1)
    rstd = (var + eps) ** -0.5
    y = (x - mean[..., None]) * rstd[..., None]
    y = y * (1.0 if weight is None else weight.double()) + (0.0 if bias is None else bias.double())
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[..., None], rstd.double()[..., None]
    xh = (x - mean) * rstd
    g = dy * (1.0 if weight is None else weight.double())
    dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    rows = tuple(range(x.dim() - 1))
    return dx, (dy * xh).sum(rows), dy.sum(rows)
