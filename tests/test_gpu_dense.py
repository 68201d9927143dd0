"""Attention over every key and its gradients against their 64-bit definitions, through the public entry points."""
import math

import pytest

torch = pytest.importorskip("torch")
import dense_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def near(got, want, tol, what=""):
    off = (got.double() - want).abs()
    assert got.isfinite().all(), f"{what}: not finite"
    assert (off <= tol).all(), f"{what}: off by {float(off.max()):.3e}, {float((off / tol.clamp(min=1e-300)).max()):.2f} of its tolerance"


def make(c, dtype, seed=0):
    """Inputs of a case: rows of order one, queries leaning towards a key; a bias that falls off with the distance."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = TYPES[dtype]
    S, Sk, Hq, Wq, Hk, Wk, d = c["shape"]
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    K, V, Q = normal(Sk, Hk, Wk, d), normal(Sk, Hk, Wk, d) + 0.5, normal(S, Hq, Wq, d)
    t = torch.randint(Hk * Wk, (S, Hq * Wq), generator=gen, device="cuda")
    pick = torch.gather(K.reshape(Sk, -1, d).repeat_interleave(S // Sk, 0), 1, t[..., None].expand(-1, -1, d))
    Q = Q + c.get("lean", 1.0) * pick.reshape(Q.shape)
    bias = None
    if c.get("heads"):
        bias = (normal(c["heads"], 2 * Hk - 1, 2 * Wk - 1)).to(kind)
    first = c.get("first", 0)
    first = torch.tensor(first, dtype=torch.int32, device="cuda") if isinstance(first, list) else first
    lengths = torch.tensor(c["lengths"], dtype=torch.int32, device="cuda") if "lengths" in c else None
    kw = dict(bias=bias, causal=c.get("causal", False), first=first, lengths=lengths)
    return Q.to(kind), K.to(kind), V.to(kind), normal(S, Hq, Wq, d).to(kind), kw


def check(scram, c, dtype, seed=0, scale=None):
    Q, K, V, dO, kw = make(c, dtype, seed)
    want, tol = ref.attend_all(Q, K, V, dO, scale, **kw)
    got = [scram.dense_attend(Q, K, V, scale, **kw), *scram.dense_attend_backward(Q, K, V, dO, scale, **kw)]
    assert len(got) == len(want)
    for name, g, w, t in zip(("out", "dQ", "dK", "dV", "dbias"), got, want, tol):
        assert g.dtype == Q.dtype and g.shape == w.shape
        near(g, w, t, f"{name} of {c}")
    return got


CASES = [
    dict(shape=(1, 1, 1, 1, 1, 1, 16)),
    dict(shape=(1, 1, 1, 1, 1, 1, 64), heads=1, causal=True),
    dict(shape=(3, 3, 1, 2, 1, 2, 32), heads=3),
    dict(shape=(2, 2, 3, 5, 3, 5, 64), heads=2),
    dict(shape=(2, 2, 7, 9, 7, 9, 16), heads=1, causal=True),
    dict(shape=(6, 2, 5, 13, 5, 13, 32), heads=3, causal=True),
    dict(shape=(6, 3, 9, 7, 4, 11, 64), lengths=[44, 0, 17]),
    dict(shape=(2, 1, 16, 16, 16, 16, 128), heads=2),
    dict(shape=(4, 2, 12, 17, 12, 17, 64), heads=4, causal=True),
    dict(shape=(2, 2, 8, 8, 8, 8, 64)),
    dict(shape=(2, 2, 1, 129, 1, 129, 64), heads=2, causal=True),
    dict(shape=(2, 2, 1, 128, 1, 128, 32), causal=True),
    dict(shape=(1, 1, 1, 257, 1, 257, 16), heads=1),
    dict(shape=(2, 2, 1, 65, 1, 63, 64)),
    dict(shape=(2, 2, 33, 1, 33, 1, 64), heads=1),
    dict(shape=(1, 1, 2, 100, 2, 100, 32), heads=1, causal=True),
    dict(shape=(2, 2, 3, 65, 3, 65, 64), heads=2),
    dict(shape=(4, 2, 1, 3, 9, 10, 64), heads=2, causal=True, first=[0, 29, 87, 51]),
    dict(shape=(4, 1, 1, 1, 9, 10, 128), causal=True, first=[0, 29, 89, 51]),
    dict(shape=(4, 4, 1, 1, 30, 31, 64), heads=4, causal=True, first=[929, 0, 463, 64]),
    dict(shape=(2, 2, 2, 10, 7, 10, 32), heads=1, first=33),
    dict(shape=(2, 2, 2, 10, 7, 10, 32), heads=2, causal=True, first=50, lengths=[70, 12]),
    dict(shape=(3, 1, 4, 5, 4, 5, 3), heads=3),
    dict(shape=(2, 2, 5, 6, 5, 6, 20), heads=2, causal=True),
    dict(shape=(2, 1, 6, 7, 9, 2, 100), lengths=[11]),
    dict(shape=(2, 2, 20, 33, 20, 33, 64), heads=2, lean=2.0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", CASES, ids=lambda c: "x".join(map(str, c["shape"])) + ("c" if c.get("causal") else "") + ("b" if c.get("heads") else ""))
def test_forward_and_gradients(scram, c, dtype):
    check(scram, c, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
def test_widths(scram, d, dtype):
    check(scram, dict(shape=(3, 3, 11, 13, 11, 13, d), heads=3), dtype, seed=d)
    check(scram, dict(shape=(2, 2, 10, 15, 10, 15, d), causal=True), dtype, seed=d + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_scales(scram, scale, dtype):
    check(scram, dict(shape=(2, 1, 6, 11, 6, 11, 32), heads=2, lean=0.0), dtype, scale=scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_key_is_certain(scram, dtype):
    """Its weight is 1: the output is its value, and neither queries nor keys have a gradient."""
    for c in (dict(shape=(4, 2, 3, 5, 1, 1, 64)), dict(shape=(2, 2, 9, 9, 9, 9, 64), lengths=[1, 1]),
              dict(shape=(2, 2, 1, 1, 9, 9, 32), causal=True, heads=2)):
        Q, K, V, dO, kw = make(c, dtype)
        S, Sk = Q.shape[0], K.shape[0]
        only = V.reshape(Sk, -1, V.shape[-1])[:, :1].repeat_interleave(S // Sk, 0)
        assert torch.equal(scram.dense_attend(Q, K, V, **kw).reshape(S, -1, V.shape[-1]), only.expand(-1, Q.shape[1] * Q.shape[2], -1))
        grads = scram.dense_attend_backward(Q, K, V, dO, **kw)
        assert not grads[0].any() and not grads[1].any()
        assert not grads[2].reshape(Sk, -1, V.shape[-1])[:, 1:].any()
        if kw["bias"] is not None:
            assert not grads[3].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nearly_certain_keys(scram, dtype):
    """What one large weight leaves to the others: dp - D is the difference of two nearly equal numbers."""
    S, n, d = 2, 24, 64
    gen = torch.Generator(device="cuda").manual_seed(5)
    K = torch.randn(S, 1, n, d, generator=gen, device="cuda")
    K = (8.0 * K / K.norm(dim=3, keepdim=True)).to(TYPES[dtype])
    Q = (1.6 * K.float()).to(TYPES[dtype])  # a score of 12.8 against the others' few
    V, dO = (torch.randn(S, 1, n, d, generator=gen, device="cuda").to(TYPES[dtype]) for _ in range(2))
    want, tol = ref.attend_all(Q, K, V, dO)
    got = scram.dense_attend_backward(Q, K, V, dO)
    for name, g, w, t in zip(("dQ", "dK", "dV"), got, want[1:], tol[1:]):
        near(g, w, t, name)
    # as a whole they keep what their type holds (a D from the rounded output is off by several times dQ here)
    for g, w in zip(got[:2], want[1:3]):
        assert float((g.double() - w).norm() / w.norm()) < (4 * 2.0 ** -8 if dtype == "bf16" else 1e-3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_in_the_bias(scram, dtype):
    """Minus infinity hides keys, up to a query's last; the lowest value hides them behind others, not all of them."""
    c = dict(shape=(2, 2, 6, 7, 6, 7, 32), heads=2)
    Q, K, V, dO, kw = make(c, dtype)
    lowest = torch.finfo(TYPES[dtype]).min
    for value in (-math.inf, lowest):
        bias = kw["bias"].clone()
        bias[0, 6:] = value          # keys below the query
        bias[0, :, 3:6] = value      # and near columns
        bias[1] = value              # every offset of head 1
        kw["bias"] = bias
        want, tol = ref.attend_all(Q, K, V, dO, **kw)
        got = [scram.dense_attend(Q, K, V, **kw), *scram.dense_attend_backward(Q, K, V, dO, **kw)]
        for name, g, w, t in zip(("out", "dQ", "dK", "dV", "dbias"), got, want, tol):
            near(g, w, t, f"{name}, {value}")
        if value == -math.inf:
            assert not got[0][1].any() and not got[1][1].any() and not got[3][1].any() and not got[4][1].any()
        else:
            near(got[0][1], V[1].double().mean((0, 1)).expand(6, 7, 32), tol[0][1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_keys_that_do_not_count_are_not_read(scram, dtype):
    """NaN behind a slice's length, and behind the last place of its queries, reaches nothing; their gradients are zeros."""
    for c in (dict(shape=(4, 2, 5, 6, 9, 11, 64), lengths=[40, 0]), dict(shape=(4, 2, 1, 2, 9, 11, 64), heads=2, causal=True, first=[40, 40, 1, 1]),
              dict(shape=(2, 2, 1, 1, 30, 30, 32), causal=True, first=[500, 77])):
        Q, K, V, dO, kw = make(c, dtype)
        clean = [scram.dense_attend(Q, K, V, **kw), *scram.dense_attend_backward(Q, K, V, dO, **kw)]
        nk = K.shape[1] * K.shape[2]
        K, V = K.clone(), V.clone()
        for s in range(K.shape[0]):
            live = c["lengths"][s] if "lengths" in c else c["first"][s * (Q.shape[0] // K.shape[0])] + Q.shape[1] * Q.shape[2]
            K.view(K.shape[0], nk, -1)[s, live:] = math.nan
            V.view(V.shape[0], nk, -1)[s, live:] = math.inf
        for g, w in zip([scram.dense_attend(Q, K, V, **kw), *scram.dense_attend_backward(Q, K, V, dO, **kw)], clean):
            assert torch.equal(g, w)
        if "lengths" in c:
            assert not clean[2][0].reshape(nk, -1)[40:].any() and not clean[2][1].any() and not clean[3][1].any()


def test_not_a_number_is_not_hidden(scram):
    """A query of NaN gives NaN, also where the keys are split over blocks."""
    for shape in ((1, 1, 1, 1, 40, 40, 64), (2, 2, 9, 9, 9, 9, 64)):
        Q, K, V, _, kw = make(dict(shape=shape), "bf16")
        Q[0, 0, 0, 3] = math.nan
        out = scram.dense_attend(Q, K, V, **kw)
        assert out[0, 0, 0].isnan().all() and (shape[0] == 1 or out[1].isfinite().all())


def test_numbers_of_lengths_and_places_are_clamped(scram):
    c = dict(shape=(2, 2, 1, 2, 5, 6, 32), causal=True, first=[-7, 1 << 30])
    Q, K, V, dO, kw = make(c, "f32")
    at = dict(kw, first=torch.tensor([0, 28], dtype=torch.int32, device="cuda"))
    assert torch.equal(scram.dense_attend(Q, K, V, **kw), scram.dense_attend(Q, K, V, **at))
    for g, w in zip(scram.dense_attend_backward(Q, K, V, dO, **kw), scram.dense_attend_backward(Q, K, V, dO, **at)):
        assert torch.equal(g, w)
    n = torch.tensor([-1, 1 << 30], dtype=torch.int32, device="cuda")
    m = torch.tensor([0, 30], dtype=torch.int32, device="cuda")
    assert torch.equal(scram.dense_attend(Q, K, V, lengths=n), scram.dense_attend(Q, K, V, lengths=m))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_calls_give_equal_bits(scram, dtype):
    """On another stream, into given tensors, after other work, with the workspace full of NaN."""
    c = dict(shape=(6, 3, 9, 40, 9, 40, 64), heads=2, causal=True)
    Q, K, V, dO, kw = make(c, dtype)
    first = [scram.dense_attend(Q, K, V, **kw), *scram.dense_attend_backward(Q, K, V, dO, **kw)]
    torch.cuda.synchronize()
    n = scram.dense_attend_backward_workspace_bytes(6, 3, 9, 40, 9, 40, d=64, dtype=TYPES[dtype], heads=2)
    ws = torch.full((n + 4,), 0xFF, dtype=torch.uint8, device="cuda")[:n]
    m = scram.dense_attend_workspace_bytes(6, 3, 9, 40, 9, 40, d=64, dtype=TYPES[dtype], bias=True)
    wf = torch.full((m + 4,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(first[0])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = scram.dense_attend(Q, K, V, out=out, workspace=wf, **kw)
        again = [got, *scram.dense_attend_backward(Q, K, V, dO, workspace=ws, **kw)]
    torch.cuda.current_stream().wait_stream(stream)
    assert got is out
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_graph_replays(scram):
    """Captured forward and backward over one workspace, replayed with new inputs and eager work between."""
    c = dict(shape=(4, 2, 1, 300, 1, 300, 64), heads=2, causal=True)
    Q, K, V, dO, kw = make(c, "bf16")
    n = max(scram.dense_attend_backward_workspace_bytes(4, 2, 1, 300, 1, 300, d=64, dtype=torch.bfloat16, heads=2),
            scram.dense_attend_workspace_bytes(4, 2, 1, 300, 1, 300, d=64, dtype=torch.bfloat16, bias=True))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    call = lambda: [scram.dense_attend(Q, K, V, workspace=ws, **kw), *scram.dense_attend_backward(Q, K, V, dO, workspace=ws, **kw)]  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed in range(1, 4):
        q, k, v, g, _ = make(c, "bf16", seed)
        for to, x in zip((Q, K, V, dO), (q, k, v, g)):
            to.copy_(x)
        graph.replay()
        got = [t.clone() for t in held]
        for a, b in zip(got, call()):
            assert torch.equal(a, b)


def test_events_and_refusals(scram):
    Q, K, V, dO, kw = make(dict(shape=(2, 2, 4, 4, 4, 4, 32), heads=2), "f32")
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for e in ev:
        e.record()
    scram.dense_attend(Q, K, V, events=ev, **kw)
    torch.cuda.synchronize()
    assert ev[0].elapsed_time(ev[1]) >= 0.0
    scram.dense_attend_backward(Q, K, V, dO, events=ev, **kw)
    torch.cuda.synchronize()
    assert ev[0].elapsed_time(ev[1]) >= 0.0
    bad = [
        (ValueError, lambda: scram.dense_attend(Q, K[:1], V, **kw)),
        (ValueError, lambda: scram.dense_attend(Q[:, ::2], K, V)),
        (TypeError, lambda: scram.dense_attend(Q, K.bfloat16(), V)),
        (TypeError, lambda: scram.dense_attend(Q, K, V, bias=kw["bias"].bfloat16())),
        (ValueError, lambda: scram.dense_attend(Q, K, V, bias=kw["bias"][:, 1:].contiguous())),
        (ValueError, lambda: scram.dense_attend(Q, K, V, first=1)),
        (ValueError, lambda: scram.dense_attend(Q, K, V, lengths=torch.ones(3, dtype=torch.int32, device="cuda"))),
        (TypeError, lambda: scram.dense_attend(Q, K, V, lengths=torch.ones(2, device="cuda"))),
        (ValueError, lambda: scram.dense_attend(Q, K, V, out=torch.empty(2, 4, 4, 16, device="cuda"))),
        (ValueError, lambda: scram.dense_attend_backward(Q, K, V, dO[:1], **kw)),
        (scram.ScramError, lambda: scram.dense_attend(Q, K, V, out=V)),
        (scram.ScramError, lambda: scram.dense_attend(Q, K, V, scale=math.nan)),
        (scram.ScramError, lambda: scram.dense_attend(Q[:, :2, :3].contiguous(), K, V, causal=True)),
        (scram.ScramError, lambda: scram.dense_attend(Q, K, V, causal=True, first=1)),
        (scram.ScramError, lambda: scram.dense_attend_backward(Q, K, V, dO, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"), **kw)),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()
    x = torch.zeros(1, 2, 2, 256, device="cuda")
    with pytest.raises(scram.ScramError):
        scram.dense_attend(x, x, x)
