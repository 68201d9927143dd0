"""Differential attention where an error cannot hide in a worst-case bound: inputs whose sums cancel, vanish or leave a row out."""
import pytest

torch = pytest.importorskip("torch")
import layer_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U32 = ref.U32


def rows(gen, kind, *shape, size=1.0):
    return (size * torch.randn(*shape, generator=gen, device="cuda")).to(kind)


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("kappa,window", [(1, 3), (2, 5), (3, 7), (4, 9)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nearly_equal_maps_cancel_to_32_bits(scram, d, kappa, window, dtype):
    """Two keys with values 1 and -1, lam = 1, scores of the two maps that differ by at most 2^-16: the output is what is left of
    two results of up to 0.25, and only errors of 32 bits may be left with it.

    Scores c + f (c of 8 bits below 1/2, f a small multiple of 2^-21) are exact in fp32.  Counted in U32 = 2^-24, per map:
    the scale in base 2 and the exponent's argument, at most 0.72 each, and two exponentials of 1 step (2 U32) move the keys' log
    ratio by 0.72 * 2 * ln 2 + 4 < 5.1, the result by half of that; the sums of the weights and of the values are rounded at
    most three times each, the values' partial sums at most 0.63 of the normaliser: 0.25 * 3 + 0.63 * 3 < 2.7; the reciprocal
    (2), product and difference 0.25 * 4 = 1.  Two maps: 2 * (2.6 + 2.7 + 1) < 13.  The result, at most 2^-17 + 13 U32, is
    rounded to bf16: 2^-8 of that, 0.5 and little more.
    """
    gen = torch.Generator(device="cuda").manual_seed(31)
    S, H, W, kind, h = 2, 64, 80, TYPES[dtype], d // 2
    n = H * W
    c = torch.randint(64, 128, (S, n), generator=gen, device="cuda") / 256.0 * torch.where(torch.rand(S, n, generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    f = torch.randint(-31, 32, (2, S, n), generator=gen, device="cuda") * 2.0 ** -21
    Q = torch.zeros(S, H, W, d, dtype=kind, device="cuda")
    K = torch.zeros(S, 1, 2, d, dtype=kind, device="cuda")
    V = torch.ones(S, 1, 2, d, dtype=kind, device="cuda")
    for m in (0, 1):
        Q.view(S, n, d)[..., m * h] = c.to(kind)
        Q.view(S, n, d)[..., m * h + 1] = f[m].to(kind)
        K[:, 0, 0, m * h:m * h + 2] = 1.0
    V[:, 0, 1] = -1.0
    s = [(Q.view(S, n, d)[..., m * h].double() + Q.view(S, n, d)[..., m * h + 1].double()) for m in (0, 1)]
    want = torch.tanh(s[0] / 2) - torch.tanh(s[1] / 2)
    J = torch.randint(0, 2, (kappa, S, H, W), generator=gen, device="cuda").to(torch.int32)
    out = scram.differential_attend(Q, K, V, J, torch.ones(S, device="cuda"), window, scale=1.0)
    off = (out.view(S, n, d).double() - want[..., None]).abs().amax() / U32
    assert float(off) <= 14.0, f"off by {float(off):.1f} U32"


@pytest.mark.parametrize("d,window,kappa", [(64, 5, 2), (32, 3, 1), (128, 7, 4), (64, 9, 1), (16, 5, 2)])
@pytest.mark.parametrize("Hq", [2, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_finite_rows_after_the_query_do_not_reach_it(scram, dtype, Hq, d, window, kappa):
    """Half of the first matches lie behind the last query, whose key may be any number: not a bit of the output, of dQ or of dlam
    changes with those rows, and all gradients are the definition's."""
    gen = torch.Generator(device="cuda").manual_seed(32)
    S, H, W, kind = 1, Hq + 5, 65, TYPES[dtype]
    n = Hq * W
    K, V = rows(gen, kind, S, H, W, d), rows(gen, kind, S, H, W, d)
    Q, dO = rows(gen, kind, S, Hq, W, d), rows(gen, kind, S, Hq, W, d)
    lam = torch.rand(S, generator=gen, device="cuda")
    own = torch.arange(n, device="cuda").reshape(Hq, W)
    J = ((own + 2 * torch.arange(kappa, device="cuda")[:, None, None, None]) % n).expand(kappa, S, Hq, W).to(torch.int32).contiguous()
    J[0] = torch.where(torch.rand(J[0].shape, generator=gen, device="cuda") < 0.5, n + J[0] % (5 * W), J[0])
    mask = ref.key_mask(J, Hq, W, H, W, window, True)
    behind = [t.view(S, H * W, d)[:, n:] for t in (K, V)]
    for t in behind:
        t.zero_()
    want, tol, wg, tg = ref.differential(Q, K, V, mask, lam, (d // 2) ** -0.5, dO)
    first = None
    for size in (0.0, 1.0, 1e3, 1e6, 1e20):
        for t in behind:
            t.copy_(rows(gen, kind, *t.shape, size=size))
        got = (scram.differential_attend(Q, K, V, J, lam, window, causal=True),
               *scram.differential_attend_backward(Q, K, V, J, lam, dO, window, causal=True))
        off = (got[0].double().reshape(want.shape) - want).abs()
        assert (off <= tol + ref.HALF[kind] * (want.abs() + tol)).all(), ("output", size)
        for name, g, w, t in zip(("dQ", "dK", "dV", "dlam"), got[1:], wg, tg):
            off = (g.double().reshape(w.shape) - w).abs()
            assert (off <= t).all(), (name, size, float(off.max()))
        first = first or got
        assert all(torch.equal(got[i], first[i]) for i in (0, 1, 4)), size


def one_key_maps(kind, gen, kappa, S, H, W, b):
    """int32 [kappa, S, H, W] under the causal mask or windows of one key: sets of one key, the query's own (two far keys for
    "spread", one key of all queries for "same")."""
    at = torch.arange(H * W, device="cuda").reshape(H, W)
    if kind == "corner":  # the window whose first key is the query: the others lie after it
        at = (at // W + b).clamp(max=H - 1) * W + (at % W + b).clamp(max=W - 1)
    elif kind == "spread":
        at = torch.randint(0, H * W, (S, H, W), generator=gen, device="cuda")
    elif kind == "same":
        at = torch.full_like(at, H * W // 3)
    return at.expand(kappa, S, H, W).to(torch.int32).contiguous()


@pytest.mark.parametrize("S", [1, 40])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("kind,window,kappa,causal", [("corner", 3, 1, True), ("corner", 5, 2, True), ("corner", 9, 4, True), ("corner", 7, 8, True),
                                                      ("spread", 1, 2, False), ("spread", 1, 4, True), ("same", 1, 3, False), ("own", 1, 1, False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sets_of_one_key_leave_the_scores_alone(scram, dtype, kind, window, kappa, causal, d, S):
    """Both softmaxes of one key are 1 whatever its score: dQ and dK are exactly 0, dV is (1 - lam) dO summed."""
    gen = torch.Generator(device="cuda").manual_seed(33)
    H, W, dt, b = 23, 26, TYPES[dtype], window // 2
    Q, K, V, dO = (rows(gen, dt, S, H, W, d, size=2.0) for _ in range(4))
    lam = torch.rand(S, generator=gen, device="cuda")
    J = one_key_maps(kind, gen, kappa, S, H, W, b)
    mask = ref.key_mask(J, H, W, H, W, window, causal)
    one = mask.sum(2) == 1
    assert one.any() and (one | ~mask.any(2) if kind != "corner" else one.view(S, H, W)[:, :H - b, :W - b]).all()
    wants = ref.differential(Q, K, V, mask, lam, (d // 2) ** -0.5, dO)[2:]
    dQ, dK, dV, dlam = scram.differential_attend_backward(Q, K, V, J, lam, dO, window, causal=causal)
    assert (dQ.view(S, H * W, d)[one] == 0).all()
    alone = ~(mask & ~one[..., None]).any(1)  # keys that only such queries hold
    assert (dK.view(S, H * W, d)[alone] == 0).all()
    for name, g, w, t in zip(("dQ", "dK", "dV", "dlam"), (dQ, dK, dV, dlam), *wants):
        off = (g.double().reshape(w.shape) - w).abs()
        assert (off <= t).all(), (name, float(off.max()))


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_passes_sets_of_one_key(scram, dtype, d):
    """An infinite dO, a NaN query and an infinite key's score in sets of one key: their rows are not finite, all others right."""
    gen = torch.Generator(device="cuda").manual_seed(34)
    S, H, W, dt = 3, 23, 26, TYPES[dtype]
    Q, K, V, dO = (rows(gen, dt, S, H, W, d) for _ in range(4))
    lam = torch.tensor([0.4, 0.7, 0.9], device="cuda")
    J = one_key_maps("corner", gen, 2, S, H, W, 2)
    mask = ref.key_mask(J, H, W, H, W, 5, True)
    _, _, want, tol = ref.differential(Q, K, V, mask, lam, (d // 2) ** -0.5, dO)
    bad = [60, 190]
    dO[0].view(-1, d)[bad[0], 5] = float("inf")
    Q[1].view(-1, d)[bad[1], d - 1] = float("nan")
    dQ, dK, dV, dlam = scram.differential_attend_backward(Q, K, V, J, lam, dO, 5, causal=True)
    assert mask[:, bad].sum() == 2 * S
    for s, i in ((0, bad[0]), (1, bad[1])):
        assert not dQ[s].view(-1, d)[i].isfinite().all() and not dV[s].view(-1, d)[i].isfinite().all() and not dlam[s].isfinite()
    hit = torch.zeros(S, H * W, dtype=torch.bool, device="cuda")
    hit[0, bad[0]] = hit[1, bad[1]] = True
    for name, g, w, t in zip(("dQ", "dK", "dV"), (dQ, dK, dV), want, tol):
        off = (g.view(S, H * W, d).double() - w).abs()
        assert (off[~hit] <= t[~hit]).all(), name
    assert abs(float(dlam[2] - want[3][2])) <= float(tol[3][2])


@pytest.mark.parametrize("H,W,window,kappa", [(256, 256, 5, 1), (1024, 1024, 3, 1), (512, 512, 5, 2), (256, 256, 17, 1), (256, 256, 1, 2)])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 16), ("f32", 64), ("f32", 128)])
def test_a_key_of_all_queries_sums_to_32_bits(scram, dtype, d, H, W, window, kappa):
    """All matches on one key, scores of 0, dO of ones: every key of the window gets n (1 - lam) / w^2, n terms that are alike.

    In U32: a weight, 2^-log2(w^2), carries the logarithm's rounding and last place (3 * 8 / 2 at most, times ln 2) and the
    exponential's 2, that of the second map 1 more, and their difference is half of the first: 2 * (11 + 12 + 1) < 50.  The sums
    may be rounded by 3 sqrt(n / (2 teams)) (runs of the square root of a lane group's steps, two terms a step, then as many
    runs; at least 2 lane groups to a key), and 8 more.
    """
    n = H * W
    kind = TYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(35)
    Q = torch.zeros(1, H, W, d, dtype=kind, device="cuda")
    K, V = rows(gen, kind, 1, H, W, d), rows(gen, kind, 1, H, W, d)
    J = torch.full((kappa, 1, H, W), (H // 2) * W + W // 2, dtype=torch.int32, device="cuda")
    dV = scram.differential_attend_backward(Q, K, V, J, torch.full((1,), 0.5, device="cuda"), torch.ones_like(Q), window)[2][0]
    b = window // 2
    got = dV[H // 2 - b:H // 2 + b + 1, W // 2 - b:W // 2 + b + 1].double()
    want = n * 0.5 / window ** 2
    off = float((got / want - 1).abs().max()) / U32
    lanes = d * (2 if dtype == "bf16" else 4) // 32  # of a lane group; a wave takes a key
    bound = 58 + 3 * (n / (2 * (64 / lanes))) ** 0.5
    assert off <= bound, f"off by {off:.0f} U32, may be {bound:.0f}"
    assert (dV.abs().sum(2) > 0).sum() == window ** 2


@pytest.mark.parametrize("window,kappa", [(3, 1), (5, 2), (9, 4), (1, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_grid_of_one_key(scram, dtype, window, kappa):
    """Every set is the one key: the output is (1 - lam) v, dV the sum of (1 - lam) dO, dQ and dK are 0."""
    gen = torch.Generator(device="cuda").manual_seed(36)
    S, H, W, d, kind = 3, 41, 37, 64, TYPES[dtype]
    Q, dO, K, V = rows(gen, kind, S, H, W, d), rows(gen, kind, S, H, W, d), rows(gen, kind, S, 1, 1, d), rows(gen, kind, S, 1, 1, d)
    lam = torch.rand(S, generator=gen, device="cuda")
    J = torch.zeros(kappa, S, H, W, dtype=torch.int32, device="cuda")
    want, tol, wg, tg = ref.differential(Q, K, V, torch.ones(S, H * W, 1, dtype=torch.bool, device="cuda"), lam, 32 ** -0.5, dO)
    out = scram.differential_attend(Q, K, V, J, lam, window)
    assert ((out.double().reshape(want.shape) - want).abs() <= tol + ref.HALF[kind] * (want.abs() + tol)).all()
    dQ, dK, dV, dlam = scram.differential_attend_backward(Q, K, V, J, lam, dO, window)
    assert (dQ == 0).all() and (dK == 0).all()
    for g, w, t in ((dV, wg[2], tg[2]), (dlam, wg[3], tg[3])):
        assert ((g.double().reshape(w.shape) - w).abs() <= t).all()
