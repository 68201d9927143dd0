"""The 64-bit definitions that the GPU tests compare with: their gradients against differentiation and differences."""
import pytest
import torch

import layer_ref as ref


def _case(causal=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    S, H, W, d = 2, 4, 5, 8
    Q, K, V, dO = (torch.randn(S, H, W, d, generator=g, dtype=torch.float64) for _ in range(4))
    maps = torch.randint(0, H * W, (2, S, H, W), generator=g)
    lam = torch.tensor([0.7, -0.3], dtype=torch.float64)
    return Q, K, V, dO, lam, ref.key_mask(maps, H, W, H, W, 3, causal)


@pytest.mark.parametrize("causal", [False, True])
def test_differential_gradients(causal):
    Q, K, V, dO, lam, mask = _case(causal)
    leaves = [t.clone().requires_grad_(True) for t in (Q, K, V, lam)]
    loss = lambda *t: (ref.differential(t[0], t[1], t[2], mask, t[3], 0.5)[0] * dO.reshape(2, -1, 8)).sum()  # noqa: E731
    want = torch.autograd.grad(loss(*leaves), leaves)
    got = ref.differential(Q, K, V, mask, lam, 0.5, dO)[2]
    for x, y in zip(got, want):
        assert torch.allclose(x.reshape(y.shape), y, rtol=1e-9, atol=1e-11)
    for i, t in enumerate((Q, K, V, lam)):  # central differences along one direction: off by about h^2
        step = torch.randn(t.shape, generator=torch.Generator().manual_seed(7 + i), dtype=torch.float64)
        at = lambda s: loss(*[u + s * step if u is t else u for u in (Q, K, V, lam)])  # noqa: B023, E731
        slope = (at(1e-5) - at(-1e-5)) / 2e-5
        assert abs(slope - (want[i] * step).sum()) < 1e-7 * (1 + (want[i] * step).abs().sum())


def test_differential_of_an_empty_set_is_zero():
    Q, K, V, dO, lam, mask = _case()
    mask[0, 3] = False
    out, _, grads, _ = ref.differential(Q, K, V, mask, lam, 0.5, dO)
    assert (out[0, 3] == 0).all() and (grads[0][0, 3] == 0).all() and all(g.isfinite().all() for g in grads)


def test_norm_gradients():
    g = torch.Generator().manual_seed(1)
    x, dy = (torch.randn(6, 9, generator=g, dtype=torch.float64) for _ in range(2))
    w, b = (torch.randn(9, generator=g, dtype=torch.float64) for _ in range(2))
    leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
    want = torch.autograd.grad((ref.layer_norm(*leaves, 1e-3)[0] * dy).sum(), leaves)
    _, mean, rstd = ref.layer_norm(x, w, b, 1e-3)
    for p, q in zip(ref.layer_norm_backward(dy, x, mean, rstd, w), want):
        assert torch.allclose(p, q, rtol=1e-10, atol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_turns_back_and_keeps_products_of_equal_shifts(interleaved):
    g = torch.Generator().manual_seed(2)
    x, y = (torch.randn(1, 3, 4, 5, 14, generator=g, dtype=torch.float64) for _ in range(2))
    kw = dict(sections=(2, 1, 3), freqs=ref.frequencies((2, 1, 3)), interleaved=interleaved)
    turn = lambda t, o, **k: ref.rotary(t, origin=torch.tensor([o]), **kw, **k)  # noqa: E731
    assert torch.allclose(turn(turn(x, (4, 5, 6)), (4, 5, 6), inverse=True), x)
    # the score of two rows depends on their distance alone
    a = (turn(x, (0, 0, 0)) * turn(y, (2, 1, 3))).sum(-1)
    b = (turn(x, (7, 9, 8)) * turn(y, (9, 10, 11))).sum(-1)
    assert torch.allclose(a, b)
    assert torch.equal(turn(x, (1, 1, 1))[..., 12:], x[..., 12:])
