"""The operators together, as a layer uses them: norm, positions, maps, differential attention, norm; and back."""
import pytest

torch = pytest.importorskip("torch")
import layer_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu


def test_forward_runs_the_operators_in_turn(scram):
    gen = torch.Generator(device="cuda").manual_seed(1)
    S, H, W, d = 2, 24, 31, 64
    Q, K, V = (torch.randn(S, H, W, d, generator=gen, device="cuda").bfloat16() for _ in range(3))
    w = [torch.randn(d // 2, generator=gen, device="cuda").bfloat16() for _ in range(4)]
    lam = torch.rand(S, generator=gen, device="cuda")
    at = dict(sections=(0, 6, 6), origin=(0, 2, 3))
    out, J = scram.forward(Q, K, V, 4, 9, 5, kappa=2, sep=2, lam=lam, norm=w, positions=at)
    two = lambda t: t.view(S, H, W, 2, d // 2)  # noqa: E731
    q, k = (scram.layer_norm(two(t), *w[i:i + 2]).view(t.shape) for t, i in ((Q, 0), (K, 2)))
    q, k = scram.rotary(q, k, groups=2, **at)
    maps = scram.patchmatch_kappa(q, k, 2, 4, 9, sep=2)
    assert torch.equal(J, maps) and torch.equal(out, scram.differential_attend(q, k, V, maps, lam, 5))
    # without the differential: one group a row, the plain attend
    out, J = scram.forward(Q, K, V, 3, 9, 3, positions=dict(sections=(0, 8, 8)))
    q, k = scram.rotary(Q, K, sections=(0, 8, 8))
    maps = scram.patchmatch_kappa(q, k, 1, 3, 9)
    assert torch.equal(J, maps) and torch.equal(out, scram.sparse_attend(q, k, V, maps, 3))
    # images of two sizes: a call each
    K2, V2 = (torch.randn(S, 17, 19, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    out, J = scram.forward(Q, K2, V2, 3, 9, 3, lam=lam, positions={})
    assert torch.equal(out, scram.differential_attend(scram.rotary(Q, groups=2), scram.rotary(K2, groups=2), V2, J, lam, 3))


def test_gradients_of_a_layer(scram):
    """Gradients back through the layer against 64-bit differentiation of its definition (maps held fixed)."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    S, H, W, d = 2, 16, 18, 64
    h, eps = d // 2, 1e-5
    Q, K, V, dY = (torch.randn(S, H, W, d, generator=gen, device="cuda") for _ in range(4))
    w = [1.0 + 0.3 * torch.randn(h, generator=gen, device="cuda") for _ in range(4)]
    wo, bo = (torch.randn(d, generator=gen, device="cuda") for _ in range(2))
    lam = 0.5 + 0.2 * torch.rand(S, generator=gen, device="cuda")
    at = dict(sections=(0, 8, 8), groups=2)
    two = lambda t: t.reshape(S, H, W, 2, h)  # noqa: E731

    q, mq, rq = scram.layer_norm(two(Q), w[0], w[1], stats=True)
    k, mk, rk = scram.layer_norm(two(K), w[2], w[3], stats=True)
    qr, kr = scram.rotary(q.view(Q.shape), k.view(K.shape), **at)
    J = scram.patchmatch_kappa(qr, kr, 2, 4, 3, sep=2)
    o = scram.differential_attend(qr, kr, V, J, lam, 5)
    y, mo, ro = scram.layer_norm(o, wo, bo, stats=True)
    do, dwo, dbo = scram.layer_norm_backward(dY, o, mo, ro, wo)
    dq, dk, dV, dlam = scram.differential_attend_backward(qr, kr, V, J, lam, do, 5)
    dq, dk = scram.rotary_backward(dq, dk, **at)
    dQ, dw0, db0 = scram.layer_norm_backward(two(dq), two(Q), mq, rq, w[0])
    dK, dw2, db2 = scram.layer_norm_backward(two(dk), two(K), mk, rk, w[2])
    got = [dQ, dK, dV, dlam, dw0, db0, dw2, db2, dwo, dbo]

    mask = ref.key_mask(J, H, W, H, W, 5)
    leaves = [t.double().clone().requires_grad_(True) for t in (Q, K, V, lam, *w, wo, bo)]
    freqs, zero = ref.frequencies(at["sections"]), torch.zeros(1, 3, device="cuda")

    def turn(t):  # differentiable: the rotation is linear, so its gradient is that of the pairs
        P, pos = 16, [torch.arange(n, device="cuda", dtype=torch.float64) for n in (H, W)]
        a = torch.cat([(pos[0][:, None, None] * torch.tensor(freqs[:8], device="cuda", dtype=torch.float64)).expand(H, W, 8),
                       (pos[1][None, :, None] * torch.tensor(freqs[8:], device="cuda", dtype=torch.float64)).expand(H, W, 8)], 2)[:, :, None]
        x, y = t[..., :P], t[..., P:]
        return torch.cat([x * a.cos() - y * a.sin(), x * a.sin() + y * a.cos()], 4).reshape(S, H, W, d)

    Ql, Kl, Vl, ll, *wl = leaves
    ql = turn(ref.layer_norm(two(Ql), wl[0], wl[1], eps)[0])
    kl = turn(ref.layer_norm(two(Kl), wl[2], wl[3], eps)[0])
    assert torch.allclose(ql.float(), ref.rotary(q.view(S, 1, H, W, d), at["sections"], freqs, zero, 2)[:, 0].float(), atol=1e-4)
    ol = ref.differential(ql, kl, Vl, mask, ll, h ** -0.5)[0].reshape(S, H, W, d)
    yl = ref.layer_norm(ol, wl[4], wl[5], eps)[0]
    want = torch.autograd.grad((yl * dY.double()).sum(), leaves)
    # every step is held to its own tolerance elsewhere; together they stay within a few hundred roundings of the largest value
    # (the layer's inner derivatives are of order one: normalised rows, weights of order one)
    assert float((y.double() - yl).abs().max()) < 1e-3 * float(yl.abs().max())
    for i, (g, x) in enumerate(zip(got, (want[0], want[1], want[2], want[3], want[4], want[5], want[6], want[7], want[8], want[9]))):
        err = float((g.double().reshape(x.shape) - x).norm() / x.norm())
        assert err < 500 * ref.U32, f"gradient {i}: {err:.2e}"
