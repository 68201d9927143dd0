"""The plain 64-bit definitions that the dense operators are tested against, against differences and torch (CPU)."""
import math

import pytest

torch = pytest.importorskip("torch")
import dense_ref as ref  # noqa: E402


def make(S, Sk, Hq, Wq, Hk, Wk, d, heads=0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    bias = normal(heads, 2 * Hk - 1, 2 * Wk - 1) if heads else None
    return normal(S, Hq, Wq, d), normal(Sk, Hk, Wk, d), normal(Sk, Hk, Wk, d), normal(S, Hq, Wq, d), bias


CALLS = [
    dict(shape=(2, 2, 3, 4, 3, 4, 5)),
    dict(shape=(6, 2, 3, 4, 3, 4, 5), heads=3, causal=True),
    dict(shape=(4, 2, 2, 3, 5, 2, 7), lengths=[0, 6]),
    dict(shape=(4, 4, 1, 3, 4, 4, 6), heads=2, causal=True, first=[0, 5, 13, 9]),
    dict(shape=(2, 1, 2, 4, 5, 4, 6), heads=1, first=7),
]


@pytest.mark.parametrize("c", CALLS, ids=lambda c: str(c["shape"]))
def test_gradients(c):
    """The formulas' gradients against differentiation of the definition, and that against differences."""
    Q, K, V, dO, bias = make(*c["shape"], heads=c.get("heads", 0))
    lengths = None if "lengths" not in c else torch.tensor(c["lengths"], dtype=torch.int32)
    kw = dict(causal=c.get("causal", False), first=c.get("first", 0), lengths=lengths)
    ref.HALF[torch.float64] = 0.0
    got, tol = ref.attend_all(Q, K, V, dO, bias=bias, **kw)
    leaves = [t.clone().requires_grad_(True) for t in (Q, K, V) + ((bias,) if bias is not None else ())]
    call = lambda *t: ref.attend(*t[:3], bias=t[3] if bias is not None else None, **kw)  # noqa: E731
    out = call(*leaves)
    assert torch.allclose(out, got[0], atol=1e-12)
    for g, w in zip(got[1:], torch.autograd.grad((out * dO).sum(), leaves)):
        assert torch.allclose(g, w, atol=1e-11)
    assert all(bool((t >= 0).all()) for t in tol)
    gen = torch.Generator().manual_seed(3)
    for i, leaf in enumerate(leaves):
        step = torch.randn(leaf.shape, generator=gen, dtype=torch.float64)
        at = [t.detach() for t in leaves]
        f = lambda h: (call(*at[:i], at[i] + h * step, *at[i + 1:]) * dO).sum()  # noqa: E731
        assert abs(float((f(1e-5) - f(-1e-5)) / 2e-5) - float((got[1 + i] * step).sum())) < 1e-6


def test_against_torch():
    Q, K, V, _, _ = make(3, 3, 4, 5, 4, 5, 8)
    flat = lambda t: t.reshape(3, -1, 8)  # noqa: E731
    want = torch.nn.functional.scaled_dot_product_attention(flat(Q), flat(K), flat(V), is_causal=True)
    assert torch.allclose(flat(ref.attend(Q, K, V, causal=True)), want, atol=1e-12)
    x = torch.randn(2, 3, 5, 12, dtype=torch.float64)
    w, b = torch.randn(12, dtype=torch.float64), torch.randn(12, dtype=torch.float64)
    want = torch.nn.functional.silu(torch.nn.functional.group_norm(x.permute(0, 3, 1, 2), 4, w, b, 1e-5)).permute(0, 2, 3, 1)
    assert torch.allclose(ref.group_norm(x, 4, w, b, 1e-5, "silu")[0], want, atol=1e-12)


def test_a_pair_s_bias_by_hand():
    """One query in the middle of a 3 x 3 grid: the key below it meets [H, W - 1] of the plane, and so on."""
    z = torch.zeros(1, 3, 3, 4, dtype=torch.float64)
    plane = torch.full((1, 5, 5), -math.inf, dtype=torch.float64)
    plane[0, 3, 2] = 0.0  # one row below, same column
    v = torch.arange(9.0, dtype=torch.float64).reshape(1, 3, 3, 1).expand(1, 3, 3, 4)
    out = ref.attend(z, z, v, bias=plane)[0, :, :, 0]
    assert out.tolist() == [[3, 4, 5], [6, 7, 8], [0, 0, 0]]  # the last row sees no key


@pytest.mark.parametrize("act", [None, "silu"])
def test_group_norm_gradients(act):
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(2, 3, 5, 12, generator=gen, dtype=torch.float64).requires_grad_(True)
    w, b = (torch.randn(12, generator=gen, dtype=torch.float64).requires_grad_(True) for _ in range(2))
    dy = torch.randn(2, 3, 5, 12, generator=gen, dtype=torch.float64)
    y, mean, rstd = ref.group_norm(x, 4, w, b, 1e-5, act)
    want = torch.autograd.grad((y * dy).sum(), (x, w, b))
    got, _ = ref.group_norm_backward(dy, x.detach(), mean.detach(), rstd.detach(), w.detach(), b.detach(), act)
    for g, t in zip(got, want):
        assert torch.allclose(g, t, atol=1e-11)


def test_buckets_by_hand():
    assert ref.buckets(5, (1, 3)).tolist() == [0, 0, 1, 1, 2, 3, 3, 4, 4]
    assert ref.buckets(3, ()).tolist() == [0] * 5
    assert ref.buckets(4, (2,)).tolist() == [0, 0, 1, 1, 1, 2, 2]
    d = torch.randn(2, 5, 9, dtype=torch.float64)
    got, _ = ref.relative_bias_backward(d, ((1,), (1, 3)))
    t = torch.randn(2, 3, 5, dtype=torch.float64)
    assert abs(float((ref.relative_bias(t, 3, 5, ((1,), (1, 3))) * d).sum() - (got * t).sum())) < 1e-12
