"""Differential attention and its gradients against the dense 64-bit definition, through the public entry points."""
import pytest

torch = pytest.importorskip("torch")
import layer_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows(gen, kind, *shape, size=1.0):
    return (size * torch.randn(*shape, generator=gen, device="cuda")).to(kind)


def maps_of(kind, gen, kappa, S, Hq, Wq, Hk, Wk, causal=False):
    """int32 [kappa, S, Hq, Wq]: random, constant, the queries' own places, two far corners by turns, or own places with a
    share of random ones, a step apart from map to map."""
    n = Hk * Wk
    at = torch.arange(Hq * Wq, device="cuda").reshape(Hq, Wq)
    own = (at // Wq * Hk // Hq) * Wk + at % Wq * Wk // Wq
    rnd = torch.randint(0, n, (kappa, S, Hq, Wq), generator=gen, device="cuda")
    if kind == "random":
        m = rnd
    elif kind == "constant":
        m = torch.full_like(rnd, n // 2)
    elif kind == "corners":
        m = torch.where(at % 2 == 0, 0, n - 1).expand(kappa, S, Hq, Wq)
    else:
        m = (own + 2 * torch.arange(kappa, device="cuda")[:, None, None, None]).expand(kappa, S, Hq, Wq) % n
        if kind == "mixed":
            m = torch.where(torch.rand(m.shape, generator=gen, device="cuda") < 0.15, rnd, m)
    return m.to(torch.int32).contiguous()


def check(got, want, tol, what):
    got = got.double().reshape(want.shape)
    assert got.isfinite().all(), f"{what}: not finite"
    off = (got - want).abs()
    over = (off - tol).max()
    assert over <= 0, f"{what}: off by {float(off.max()):.3e}, {float((off / tol.clamp(min=1e-300)).max()):.2f} of its tolerance"


def run(scram, c, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    S, Hq, Wq, Hk, Wk, d, kind = c["S"], *c["q"], *c.get("k", c["q"]), c["d"], TYPES[c["dtype"]]
    dv, causal = c.get("dv", d), c.get("causal", False)
    Q, K = rows(gen, kind, S, Hq, Wq, d, size=1.5), rows(gen, kind, S, Hk, Wk, d)
    V, dO = rows(gen, kind, S, Hk, Wk, dv), rows(gen, kind, S, Hq, Wq, dv)
    lam = 0.6 + 0.4 * torch.randn(S, generator=gen, device="cuda")
    J = maps_of(c.get("maps", "mixed"), gen, c["kappa"], S, Hq, Wq, Hk, Wk)
    mask = ref.key_mask(J, Hq, Wq, Hk, Wk, c["window"], causal)
    scale = c.get("scale", (d // 2) ** -0.5)
    given = {} if "scale" not in c else dict(scale=scale)
    arg = J[0] if c["kappa"] == 1 else J
    out = scram.differential_attend(Q, K, V, arg, lam, c["window"], causal=causal, **given)
    grads = scram.differential_attend_backward(Q, K, V, arg, lam, dO, c["window"], causal=causal, **given)
    torch.cuda.synchronize()
    want, tol, wg, tg = ref.differential(Q, K, V, mask, lam, scale, dO)
    assert out.dtype == kind and out.shape == (S, Hq, Wq, dv)
    check(out, want, tol + ref.HALF[kind] * (want.abs() + tol), "output")
    empty = ~mask.any(2)
    assert (out.reshape(S, -1, dv)[empty] == 0).all() and (grads[0].reshape(S, -1, d)[empty] == 0).all()
    for name, g, w, t, like in zip(("dQ", "dK", "dV", "dlam"), grads, wg, tg, (Q, K, V, lam)):
        assert g.dtype == torch.float32 and g.shape == like.shape
        check(g, w, t, name)


SHAPES = [
    dict(S=2, q=(17, 23), d=16, window=3, kappa=1),
    dict(S=2, q=(16, 24), d=32, window=5, kappa=1),
    dict(S=1, q=(33, 29), d=64, window=3, kappa=2),
    dict(S=3, q=(24, 24), d=64, window=7, kappa=2, causal=True),
    dict(S=2, q=(19, 31), d=128, window=5, kappa=1, causal=True),
    dict(S=2, q=(13, 11), k=(21, 18), d=64, window=5, kappa=2),
    dict(S=2, q=(26, 22), k=(9, 7), d=32, window=7, kappa=1),
    dict(S=1, q=(1, 70), d=64, window=3, kappa=1, causal=True),
    dict(S=1, q=(67, 1), d=32, window=5, kappa=2),
    dict(S=5, q=(1, 1), d=64, window=3, kappa=1),
    dict(S=2, q=(2, 3), d=64, window=7, kappa=4, causal=True),
    dict(S=1, q=(20, 20), d=64, window=9, kappa=3),
    dict(S=1, q=(18, 21), d=32, window=17, kappa=2),
    dict(S=1, q=(14, 15), d=64, window=3, kappa=8, causal=True),
    dict(S=1, q=(21, 14), d=128, window=7, kappa=4),
    dict(S=2, q=(15, 16), d=64, window=1, kappa=3),
    dict(S=1, q=(70, 66), d=64, window=5, kappa=2),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", SHAPES, ids=lambda c: f"{c['q'][0]}x{c['q'][1]}_d{c['d']}_w{c['window']}_k{c['kappa']}" + ("_causal" if c.get("causal") else ""))
def test_shapes(scram, c, dtype):
    run(scram, dict(c, dtype=dtype))


def many(c):
    """The same with slices enough for more than 4096 queries: those of fewer take another way forward."""
    return dict(c, S=4096 // (c["q"][0] * c["q"][1]) + 1)


MANY = SHAPES[:-1] + [
    dict(S=1, q=(20, 23), d=64, window=9, kappa=1, causal=True),
    dict(S=1, q=(24, 17), d=128, window=9, kappa=2),
    dict(S=1, q=(13, 30), k=(30, 13), d=32, window=9, kappa=4),
    dict(S=1, q=(1, 2), k=(40, 1), d=64, window=7, kappa=2),
    dict(S=1, q=(5, 4), k=(1, 33), d=32, window=5, kappa=3),
    dict(S=1, q=(16, 16), k=(2, 2), d=64, window=3, kappa=2),
]


@pytest.mark.parametrize("maps", ["mixed", "random", "constant", "corners"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", MANY, ids=lambda c: f"{c['q'][0]}x{c['q'][1]}_d{c['d']}_w{c['window']}_k{c['kappa']}" + ("_causal" if c.get("causal") else ""))
def test_many_slices(scram, c, dtype, maps):
    run(scram, dict(many(c), dtype=dtype, maps=maps), seed=12)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", [40, 140])
@pytest.mark.parametrize("c", [dict(d=64, window=3, kappa=1), dict(d=32, window=5, kappa=2, causal=True), dict(d=16, window=7, kappa=1, causal=True),
                               dict(d=128, window=5, kappa=1)], ids=["w3", "w5_two_causal", "w7_causal", "wide"])
def test_more_strips_of_keys(scram, c, S, dtype):
    """Fewer waves take each strip of keys where there are many of them."""
    run(scram, dict(c, S=S, q=(23, 26), maps="mixed" if S == 40 else "random", dtype=dtype), seed=14)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("maps", ["constant", "corners"])
@pytest.mark.parametrize("c", [dict(d=64, window=7, kappa=1), dict(d=32, window=3, kappa=3, causal=True), dict(d=64, window=15, kappa=2)],
                         ids=["w7", "w3_three_causal", "w15_two"])
def test_keys_of_thousands_of_queries(scram, c, maps, dtype):
    run(scram, dict(c, S=1, q=(70, 66), maps=maps, dtype=dtype), seed=15)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 128])
@pytest.mark.parametrize("maps", ["mixed", "random", "constant"])
@pytest.mark.parametrize("kappa,causal,S", [(2, False, 3), (4, True, 140)])
def test_windows_of_one_key(scram, kappa, causal, S, maps, d, dtype):
    run(scram, dict(S=S, q=(23, 26), d=d, window=1, kappa=kappa, causal=causal, maps=maps, dtype=dtype), seed=23)


@pytest.mark.parametrize("window,kappa", [(11, 1), (13, 2), (15, 1), (19, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_windows(scram, window, kappa, dtype):
    run(scram, dict(S=12, q=(19, 21), d=64, window=window, kappa=kappa, causal=kappa == 2, dtype=dtype), seed=16)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,kappa", [(5, 1), (3, 2)])
def test_gradients_that_are_not_finite_reach_their_keys_alone(scram, window, kappa, dtype):
    """One query's dO holds an infinity, another's row a NaN: their own rows and their keys' are hit, all others are right."""
    gen = torch.Generator(device="cuda").manual_seed(17)
    S, H, W, d, kind = 2, 22, 25, 64, TYPES[dtype]
    Q, K, V, dO = (rows(gen, kind, S, H, W, d) for _ in range(4))
    lam = torch.tensor([0.4, 0.7], device="cuda")
    J = maps_of("mixed", gen, kappa, S, H, W, H, W)
    mask = ref.key_mask(J, H, W, H, W, window)
    _, _, want, tol = ref.differential(Q, K, V, mask, lam, 32 ** -0.5, dO)
    bad = [100, 333]
    dO[0].view(-1, d)[bad[0], 5] = float("inf")
    Q[0].view(-1, d)[bad[1], 50] = float("nan")
    dQ, dK, dV, dlam = scram.differential_attend_backward(Q, K, V, J, lam, dO, window)
    hit_q = torch.zeros(S, H * W, dtype=torch.bool, device="cuda")
    hit_q[0, bad] = True
    hit_k = mask[0, bad].any(0)
    hit_k = torch.stack([hit_k, torch.zeros_like(hit_k)])
    for name, g, w, t, hit in zip(("dQ", "dK", "dV"), (dQ, dK, dV), want, tol, (hit_q, hit_k, hit_k)):
        off = (g.view(S, H * W, d).double() - w).abs()
        # (a query's good keys' rows also hold sums of the clean terms that the bad queries would have given: not compared)
        assert (off[~hit] <= t[~hit]).all(), name
        assert (~g.view(S, H * W, d).isfinite()).any(2)[hit].all(), name
    assert not dlam[0].isfinite() and abs(float(dlam[1] - want[3][1])) <= float(tol[3][1])


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_scores_far_apart(scram, d, causal):
    """Scores of hundreds: references are raised on the way, weights underflow, a query's first match may have no weight."""
    run(scram, dict(many(dict(S=1, q=(18, 22), d=d, window=5, kappa=2)), scale=4.0, causal=causal, dtype="bf16", maps="random"), seed=13)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("maps", ["random", "constant", "own", "corners"])
@pytest.mark.parametrize("c", [dict(S=2, q=(24, 28), d=64, window=5, kappa=2), dict(S=1, q=(32, 24), d=32, window=3, kappa=1, causal=True),
                               dict(S=1, q=(24, 24), d=128, window=7, kappa=1), dict(S=1, q=(25, 27), d=16, window=7, kappa=3)],
                         ids=["two", "causal", "wide", "narrow"])
def test_maps(scram, c, maps, dtype):
    run(scram, dict(c, maps=maps, dtype=dtype), seed=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,dv", [(2, 2), (6, 6), (12, 5), (20, 20), (34, 64), (96, 96), (64, 16), (128, 100)])
def test_padded_widths(scram, d, dv, dtype):
    run(scram, dict(S=2, q=(9, 12), d=d, dv=dv, window=3, kappa=2, dtype=dtype), seed=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.0, -0.4, 3.0])
def test_scales(scram, scale, dtype):
    run(scram, dict(S=1, q=(18, 20), d=64, window=5, kappa=1, scale=scale, dtype=dtype), seed=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_key_sets_have_no_score_gradient(scram, dtype):
    gen = torch.Generator(device="cuda").manual_seed(4)
    Q, K, V, dO = (rows(gen, TYPES[dtype], 1, 12, 13, 64) for _ in range(4))
    lam = torch.tensor([0.5], device="cuda")
    J = maps_of("mixed", gen, 1, 1, 12, 13, 12, 13)
    out = scram.differential_attend(Q, K, V, J, lam, 1)
    # one key: both maps give it weight 1
    want = (V.reshape(-1, 64)[J.reshape(-1).long()].double() * 0.5).reshape(out.shape)
    assert torch.equal(out, want.to(out.dtype))
    dQ, dK, dV, dlam = scram.differential_attend_backward(Q, K, V, J, lam, dO, 1)
    assert (dQ == 0).all() and (dK == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("run_of", [1, 7, 40])
def test_new_pixels_of_a_grid(scram, run_of, dtype):
    """A run of queries at a place of their own per slice, as numbers and from the device, equals the same rows of the
    definition."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    S, H, W, d, kind = 3, 14, 18, 64, TYPES[dtype]
    K, V = rows(gen, kind, S, H, W, d), rows(gen, kind, S, H, W, d)
    Q, dO = rows(gen, kind, S, 1, run_of, d, size=1.5), rows(gen, kind, S, 1, run_of, d)
    lam = torch.rand(S, generator=gen, device="cuda")
    J = maps_of("random", gen, 2, S, 1, run_of, H, W)
    at = torch.tensor([0, 101, H * W - run_of], dtype=torch.int32, device="cuda")
    for first, place in ((at, at.cpu()), (57, torch.full((S,), 57))):
        out = scram.differential_attend(Q, K, V, J, lam, 7, causal=True, first=first)
        grads = scram.differential_attend_backward(Q, K, V, J, lam, dO, 7, causal=True, first=first)
        mask = ref.key_mask(J, 1, run_of, H, W, 7, True, place)
        want, tol, wg, tg = ref.differential(Q, K, V, mask, lam, 32 ** -0.5, dO)
        check(out, want, tol + ref.HALF[kind] * (want.abs() + tol), "output")
        for g, w, t in zip(grads, wg, tg):
            check(g, w, t, "gradient")
    # whole rows
    Q = rows(gen, kind, S, 2, W, d)
    J = maps_of("random", gen, 1, S, 2, W, H, W)
    out = scram.differential_attend(Q, K, V, J, lam, 5, causal=True, first=3 * W)
    want, tol = ref.differential(Q, K, V, ref.key_mask(J, 2, W, H, W, 5, True, torch.full((S,), 3 * W)), lam, 32 ** -0.5)
    check(out, want, tol + ref.HALF[kind] * (want.abs() + tol), "rows")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("few", [False, True])
def test_rows_outside_the_sets_do_not_reach_the_result(scram, few, dtype):
    """Keys after the query hold NaN and infinities, as a cache's unwritten rows may; so do keys that no window holds."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    S, H, W, d, kind = 2, (12 if few else 80), 65, 64, TYPES[dtype]
    Hq, first = (1, 5 * W) if few else (H, 0)
    last = first + Hq * W - 1
    K, V = rows(gen, kind, S, H, W, d), rows(gen, kind, S, H, W, d)
    Q, dO = rows(gen, kind, S, Hq, W, d), rows(gen, kind, S, Hq, W, d)
    lam = torch.rand(S, generator=gen, device="cuda")
    J = maps_of("random", gen, 2, S, Hq, W, H, W)
    if not few:  # the queries before row 60 only see keys before it; the rest sees all of them
        J = torch.where(torch.arange(H, device="cuda")[:, None] < 60, J % (60 * W), J).to(torch.int32).contiguous()
    bad_from = (last + 1) if few else 60 * W
    Kb, Vb = K.clone(), V.clone()
    Kb.view(S, H * W, d)[:, bad_from:] = float("nan")
    Vb.view(S, H * W, d)[:, bad_from:] = float("inf")
    Vb.view(S, H * W, d)[:, bad_from + 1::3] = float("nan")
    seen = slice(0, Hq) if few else slice(0, 57)  # with windows of half side 3 within row 59
    J[..., seen, :] = torch.minimum(J[..., seen, :], torch.full_like(J[..., seen, :], bad_from - 1))
    # against the definition with those rows zeroed (a query near them may be computed another way, in another order)
    Kz, Vz = K.clone(), V.clone()
    Kz.view(S, H * W, d)[:, bad_from:], Vz.view(S, H * W, d)[:, bad_from:] = 0, 0
    mask = ref.key_mask(J, Hq, W, H, W, 7, True, torch.full((S,), first))
    assert not mask[:, : (Hq if few else 57) * W, bad_from:].any()
    want, tol, wg, tg = ref.differential(Q, Kz, Vz, mask, lam, 32 ** -0.5, dO)
    tol = tol + ref.HALF[kind] * (want.abs() + tol)
    cut = lambda x: x.reshape(S, Hq, W, d)[:, seen]  # noqa: E731
    for k, v in ((K, V), (Kb, Vb)):
        check(scram.differential_attend(Q, k, v, J, lam, 7, causal=True, first=first)[:, seen], cut(want), cut(tol), "output")
    if few:
        grads = scram.differential_attend_backward(Q, Kb, Vb, J, lam, dO, 7, causal=True, first=first)
        for name, g, w, t in zip(("dQ", "dK", "dV", "dlam"), grads, wg, tg):
            check(g, w, t, name)
        assert all((g.view(S, H * W, d)[:, bad_from:] == 0).all() for g in grads[1:3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq", [2, 64])
def test_matches_after_the_query_may_hold_anything(scram, Hq, dtype):
    """The rows behind the last query hold NaN and infinities, and half of the first matches are there."""
    gen = torch.Generator(device="cuda").manual_seed(21)
    S, H, W, d, kind = 1, Hq + 5, 65, 64, TYPES[dtype]
    n = Hq * W
    K, V = rows(gen, kind, S, H, W, d), rows(gen, kind, S, H, W, d)
    Q, dO = rows(gen, kind, S, Hq, W, d), rows(gen, kind, S, Hq, W, d)
    lam = torch.rand(S, generator=gen, device="cuda")
    J = maps_of("own", gen, 2, S, Hq, W, H, W) % n
    J[0] = torch.where(torch.rand(J[0].shape, generator=gen, device="cuda") < 0.5, n + J[0] % (5 * W), J[0])
    mask = ref.key_mask(J, Hq, W, H, W, 5, True)
    K.view(S, H * W, d)[:, n:], V.view(S, H * W, d)[:, n:] = 0, 0
    want, tol, wg, tg = ref.differential(Q, K, V, mask, lam, 32 ** -0.5, dO)
    K.view(S, H * W, d)[:, n:], V.view(S, H * W, d)[:, n:] = float("nan"), float("inf")
    check(scram.differential_attend(Q, K, V, J, lam, 5, causal=True), want, tol + ref.HALF[kind] * (want.abs() + tol), "output")
    for name, g, w, t in zip(("dQ", "dK", "dV", "dlam"), scram.differential_attend_backward(Q, K, V, J, lam, dO, 5, causal=True), wg, tg):
        check(g, w, t, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_finite_reach_their_queries_alone(scram, dtype):
    gen = torch.Generator(device="cuda").manual_seed(7)
    S, H, W, d, kind = 1, 70, 72, 64, TYPES[dtype]
    Q, K, V = (rows(gen, kind, S, H, W, d) for _ in range(3))
    lam = torch.tensor([0.4], device="cuda")
    J = maps_of("own", gen, 2, S, H, W, H, W)
    bad = 33 * W + 35
    V.view(-1, d)[bad, 3] = float("inf")
    out = scram.differential_attend(Q, K, V, J, lam, 5).view(-1, d)
    mask = ref.key_mask(J, H, W, H, W, 5)[0]
    hit = mask[:, bad]
    clean = V.clone()
    clean.view(-1, d)[bad, 3] = 0
    want, tol = ref.differential(Q, K, clean, mask[None], lam, 32 ** -0.5)
    want, tol = want[0], tol[0] + ref.HALF[kind] * (want[0].abs() + tol[0])
    keep = torch.ones_like(want, dtype=torch.bool)
    keep[hit, 3] = False
    assert not out[hit, 3].isfinite().any()
    assert ((out.double() - want).abs() <= tol)[keep].all()
    K.view(-1, d)[bad, 40] = float("nan")  # a score of the second map
    out = scram.differential_attend(Q, K, clean, J, lam, 5).view(-1, d)
    assert out[hit].isnan().all() and out[~hit].isfinite().all()


@pytest.mark.parametrize("n", [1, 40, 5000])
def test_memory_behind_the_results_is_left_alone(scram, n):
    gen = torch.Generator(device="cuda").manual_seed(8)
    K, V = rows(gen, torch.bfloat16, 1, 9, 33, 64), rows(gen, torch.bfloat16, 1, 9, 33, 64)
    Q = rows(gen, torch.bfloat16, 1, 1, n, 64)
    J = torch.randint(-50, 9 * 33 + 50, (1, 1, n), generator=gen, device="cuda").to(torch.int32)  # also beyond the grid: clamped
    store = torch.full((n + 64, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    got = scram.differential_attend(Q, K, V, J, torch.ones(1, device="cuda"), 7, out=store[32:32 + n].view(1, 1, n, 64))
    assert got.isfinite().all() and (store[:32] == 7).all() and (store[32 + n:] == 7).all()


def test_offsets_past_32_bits(scram):
    """A slice of more than 4 GiB of key rows, and slices whose rows lie past 4 GiB."""
    for S, H, W in ((1, 4200, 8192), (40, 1024, 1024)):
        K = torch.zeros(S, H, W, 64, dtype=torch.bfloat16, device="cuda")
        V = torch.zeros_like(K)
        gen = torch.Generator(device="cuda").manual_seed(9)
        tail = rows(gen, torch.bfloat16, 2, 40, 64)
        K.view(-1, 64)[-40:], V.view(-1, 64)[-40:] = tail[0], tail[1]
        Q = torch.zeros(S, 1, 8, 64, dtype=torch.bfloat16, device="cuda")
        Q[-1] = rows(gen, torch.bfloat16, 1, 8, 64)
        J = torch.full((S, 1, 8), H * W - 1, dtype=torch.int32, device="cuda") - torch.arange(8, dtype=torch.int32, device="cuda")
        lam = torch.full((S,), 0.5, device="cuda")
        out = scram.differential_attend(Q, K, V, J, lam, 3)[-1]
        # the last slice's last three rows of columns W - 10 .. as a grid of their own
        k, v = (t[-1, H - 3:, W - 12:].reshape(1, 3, 12, 64) for t in (K, V))
        mine = (2 * 12 + (J[-1] % W - (W - 12)))[None, None]
        want, tol = ref.differential(Q[-1][None], k, v, ref.key_mask(mine, 1, 8, 3, 12, 3), lam[:1], 32 ** -0.5)
        check(out, want[0].reshape(out.shape), (tol + 2.0 ** -8 * (want.abs() + tol)).reshape(out.shape), "tail")
        del K, V


def test_graph_replays_equal_eager(scram):
    gen = torch.Generator(device="cuda").manual_seed(10)
    S, H, W, d = 2, 40, 37, 64
    Q, K, V, dO = (rows(gen, torch.bfloat16, S, H, W, d) for _ in range(4))
    J, lam = maps_of("mixed", gen, 2, S, H, W, H, W), torch.rand(S, generator=gen, device="cuda")
    ws = torch.empty(scram.differential_attend_backward_workspace_bytes(S, H, W, H, W, 2, d=d, dtype=Q.dtype), dtype=torch.uint8, device="cuda")
    at = torch.zeros(S, dtype=torch.int32, device="cuda")
    got = {}

    def step():
        got["o"] = scram.differential_attend(Q, K, V, J, lam, 5, causal=True, first=at)
        got["g"] = scram.differential_attend_backward(Q, K, V, J, lam, dO, 5, causal=True, first=at, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    caught = dict(got)
    for rep in range(4):
        Q.copy_(rows(gen, torch.bfloat16, S, H, W, d))  # new inputs in the same places
        lam.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        assert torch.equal(caught["o"], got["o"]), rep
        assert torch.equal(caught["g"][0], got["g"][0]) and torch.equal(caught["g"][3], got["g"][3])
        for x, y in zip(caught["g"][1:3], got["g"][1:3]):  # summed in the order in which the inverse map was filled
            assert torch.allclose(x, y, rtol=1e-5, atol=1e-5 * float(y.abs().max()))


def test_two_streams_at_once(scram):
    gen = torch.Generator(device="cuda").manual_seed(11)
    made = []
    for dtype, W in ((torch.bfloat16, 96), (torch.float32, 80)):
        Q, K, V, dO = (rows(gen, dtype, 2, 96, W, 64) for _ in range(4))
        made.append((Q, K, V, maps_of("mixed", gen, 2, 2, 96, W, 96, W), torch.rand(2, generator=gen, device="cuda"), dO))
    go = lambda a: (scram.differential_attend(*a[:5], 5), *scram.differential_attend_backward(*a, 5))  # noqa: E731
    want = [go(a) for a in made]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(3):
        got = []
        for a, s in zip(made, streams):
            with torch.cuda.stream(s):
                got.append(go(a))
        torch.cuda.synchronize()
        for w, g in zip(want, got):
            for i in (0, 1, 4):
                assert torch.equal(w[i], g[i])
            for i in (2, 3):
                assert torch.allclose(w[i], g[i], rtol=1e-5, atol=1e-5 * float(w[i].abs().max()))


def test_two_graphs_share_a_workspace(scram):
    """Captured in turn over one workspace and replayed in any order, one after the other."""
    gen = torch.Generator(device="cuda").manual_seed(18)
    made = []
    for H, W, window, causal in ((31, 40, 5, True), (44, 28, 3, False)):
        Q, K, V, dO = (rows(gen, torch.bfloat16, 2, H, W, 64) for _ in range(4))
        made.append(((Q, K, V, maps_of("mixed", gen, 2, 2, H, W, H, W), torch.rand(2, generator=gen, device="cuda"), dO, window), causal))
    size = max(scram.differential_attend_backward_workspace_bytes(*a[0].shape[:3], *a[0].shape[1:3], 2, d=64, dtype=a[0].dtype) for a, _ in made)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    want = [scram.differential_attend_backward(*a, causal=c) for a, c in made]
    graphs, got = [], []
    torch.cuda.synchronize()
    for a, c in made:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(scram.differential_attend_backward(*a, causal=c, workspace=ws))
    for turn in (0, 1, 1, 0, 1):
        for g in got[turn]:
            g.fill_(3.0)
        ws.fill_(0x5A)
        graphs[turn].replay()
        torch.cuda.synchronize()
        for i, (w, g) in enumerate(zip(want[turn], got[turn])):
            assert torch.equal(w, g) if i in (0, 3) else torch.allclose(w, g, rtol=1e-5, atol=1e-5 * float(w.abs().max()))


@pytest.mark.parametrize("c", [dict(S=2, q=(72, 67), d=64, window=5, kappa=2), dict(S=1, q=(9, 1100), d=64, window=3, kappa=1, causal=True),
                               dict(S=2, q=(12, 700), d=32, window=3, kappa=2), dict(S=20, q=(1, 300), d=32, window=7, kappa=1),
                               dict(S=16, q=(300, 1), d=64, window=3, kappa=1), dict(S=2, q=(56, 56), k=(23, 31), d=64, window=9, kappa=1),
                               dict(S=2, q=(50, 50), d=128, window=5, kappa=2), dict(S=3, q=(31, 70), d=16, window=7, kappa=1)],
                         ids=lambda c: f"{c['q'][0]}x{c['q'][1]}_d{c['d']}_w{c['window']}")
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_results_do_not_depend_on_the_launch(scram, c, dtype):
    """The same calls through a build with other lane-group tiles, bands of tiles and dispatch order."""
    from paper_1905_10308_amd import binding

    gen = torch.Generator(device="cuda").manual_seed(22)
    S, Hq, Wq, Hk, Wk, d, kind = c["S"], *c["q"], *c.get("k", c["q"]), c["d"], TYPES[dtype]
    Q, dO = rows(gen, kind, S, Hq, Wq, d, size=1.5), rows(gen, kind, S, Hq, Wq, d)
    K, V = rows(gen, kind, S, Hk, Wk, d), rows(gen, kind, S, Hk, Wk, d)
    J, lam = maps_of("mixed", gen, c["kappa"], S, Hq, Wq, Hk, Wk), torch.rand(S, generator=gen, device="cuda")
    go = lambda: (scram.differential_attend(Q, K, V, J, lam, c["window"], causal=c.get("causal", False)),  # noqa: E731
                  *scram.differential_attend_backward(Q, K, V, J, lam, dO, c["window"], causal=c.get("causal", False)))
    want = go()
    saved = binding.lib()
    binding._lib = binding.load(binding.ORDER_LIB_PATH)
    try:
        for _ in range(2):
            got = go()
            torch.cuda.synchronize()
            for i, (g, w) in enumerate(zip(got, want)):
                # dK and dV: in the order that the inverse map was filled in; dlam: its parts in the order of the tiles
                assert torch.equal(g, w) if i < 2 else torch.allclose(g, w, rtol=1e-5, atol=1e-5 * float(w.abs().max())), i
    finally:
        binding._lib = saved
