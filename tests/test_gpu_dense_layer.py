"""Group norm, dense attention and the bias by buckets together, and calls that reach the kernels' other forms."""
import math

import pytest

torch = pytest.importorskip("torch")
import dense_ref as ref  # noqa: E402
from test_gpu_dense import TYPES, check, make, near  # noqa: E402

pytestmark = pytest.mark.gpu


def layer(scram, kind, N=2, H=9, W=11, C=64, heads=2, seed=3):
    """An image model's attention layer and its gradients: state, and a call of it on the state."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(kind)  # noqa: E731
    s = dict(x=normal(N, H, W, C), dY=normal(N, H, W, C), gamma=1 + 0.2 * normal(C), beta=0.2 * normal(C), table=normal(heads, 7, 9),
             w=(normal(3, C, C).float() * C ** -0.5).to(kind), lengths=torch.tensor([H * W, 40] * (N // 2), dtype=torch.int32, device="cuda"))
    s["lengths"] = s["lengths"].repeat_interleave(heads)
    d, edges = C // heads, (scram.bias_edges(3, H - 1), scram.bias_edges(4, W - 1))
    split = lambda t: t.reshape(N, H, W, heads, d).permute(0, 3, 1, 2, 4).reshape(N * heads, H, W, d).contiguous()  # noqa: E731
    join = lambda t: t.reshape(N, heads, H, W, d).permute(0, 2, 3, 1, 4).reshape(N, H, W, C).contiguous()  # noqa: E731

    def call():
        h, mean, rstd = scram.group_norm(s["x"], 8, s["gamma"], s["beta"], activation="silu", stats=True)
        q, k, v = (split(h @ w) for w in s["w"])
        bias = scram.relative_bias(s["table"], H, W, edges=edges)
        y = join(scram.dense_attend(q, k, v, bias=bias, lengths=s["lengths"]))
        *dqkv, dbias = scram.dense_attend_backward(q, k, v, split(s["dY"]), bias=bias, lengths=s["lengths"])
        dtable = scram.relative_bias_backward(dbias, edges=edges)
        dqkv = [join(t) for t in dqkv]
        dw = torch.stack([h.reshape(-1, C).t() @ t.reshape(-1, C) for t in dqkv])
        dh = sum(t @ w.t() for t, w in zip(dqkv, s["w"]))
        dx, dgamma, dbeta = scram.group_norm_backward(dh, s["x"], mean, rstd, s["gamma"], s["beta"], activation="silu")
        return [y, dx, dgamma, dbeta, dtable, dw]

    return s, call, split, join, edges


def test_a_layer_and_its_gradients(scram):
    s, call, split, join, edges = layer(scram, torch.float32)
    got = call()
    leaves = [s[n].double().requires_grad_(True) for n in ("x", "gamma", "beta", "table", "w")]
    x, gamma, beta, table, w = leaves
    N, H, W, C = x.shape
    h = ref.group_norm(x, 8, gamma, beta, act="silu")[0]
    q, k, v = (split(h @ one).flatten(1, 2) for one in w)
    j = torch.arange(H * W, device="cuda")
    bucket = [torch.tensor([[math.copysign(sum(e <= abs(b - a) for e in edge), b - a) + len(edge) for b in range(n)] for a in range(n)],
                           device="cuda").long() for n, edge in ((H, edges[0]), (W, edges[1]))]
    by, bx = bucket[0][j // W][:, j // W], bucket[1][j % W][:, j % W]
    a = q @ k.transpose(1, 2) * q.shape[-1] ** -0.5 + table[:, by, bx].repeat(N, 1, 1)
    a = a.masked_fill(j >= s["lengths"][:, None, None], -math.inf)
    y = join((torch.softmax(a, 2) @ v).reshape(-1, H, W, q.shape[-1]))
    want = [y.detach(), *torch.autograd.grad((y * s["dY"].double()).sum(), leaves)]
    # every step is held to its own tolerance elsewhere; together they stay within a few hundred roundings of a result's size
    # (the inner derivatives are of order one: normalised rows, weights of order one)
    for i, (g, t) in enumerate(zip(got, want)):
        err = float((g.double() - t).norm() / t.norm())
        assert err < 500 * ref.U32, f"result {i}: {err:.2e}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_layer_in_a_graph(scram, dtype):
    """Captured with its gradients, replayed with other inputs and the same layer's eager work between."""
    s, call, *_ = layer(scram, TYPES[dtype])
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed in range(4, 7):
        for name, t in layer(scram, TYPES[dtype], seed=seed)[0].items():
            s[name].copy_(t)
        graph.replay()
        got = [t.clone() for t in held]
        for a, b in zip(got, call()):
            assert torch.equal(a, b)


# four and eight waves' queries to a block, two blocks a CU, other shares of the keys; keys' blocks with and without parts
FORMS = [
    dict(shape=(128, 128, 15, 17, 15, 17, 64)),
    dict(shape=(128, 64, 15, 17, 15, 17, 64), heads=4, causal=True),
    dict(shape=(64, 64, 16, 16, 16, 16, 64), heads=2),
    dict(shape=(64, 64, 1, 250, 1, 250, 32), causal=True, lengths=[250, 3, 0, 129] * 16),
    dict(shape=(128, 128, 1, 230, 1, 230, 128), heads=1),
    dict(shape=(64, 64, 13, 18, 13, 18, 128)),
    dict(shape=(256, 256, 1, 70, 1, 300, 16), heads=2, causal=True, first=230),
    dict(shape=(8, 1, 1, 4, 40, 41, 64), heads=8, causal=True, first=[3, 1636, 70, 800, 0, 1, 2, 1599]),
    dict(shape=(4, 1, 1, 8, 30, 31, 32), heads=2, first=[5, 922, 70, 800]),
    dict(shape=(2, 1, 40, 41, 2, 3, 64)),
    dict(shape=(2, 2, 2, 700, 2, 700, 64), heads=1),
    # two blocks a CU that stage one step at a time
    dict(shape=(300, 300, 1, 40, 1, 601, 64)),
    dict(shape=(260, 130, 1, 5, 1, 790, 64), lengths=[790, 0, 700, 5, 64] * 26),
    dict(shape=(264, 264, 1, 24, 1, 600, 32), causal=True, first=576),
    # causal runs of the keys' side: many and few queries behind a place of their own, shared keys
    dict(shape=(3, 1, 1, 900, 1, 1500, 32), causal=True, first=421),
    dict(shape=(2, 2, 1, 129, 1, 1100, 128), causal=True, first=971),
    dict(shape=(8, 1, 1, 640, 1, 641, 16), heads=2, causal=True, first=1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", FORMS, ids=lambda c: "x".join(map(str, c["shape"])))
def test_forms(scram, c, dtype):
    check(scram, c, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,dv", [(20, 33), (64, 16), (8, 100)])
def test_values_of_another_width(scram, d, dv, dtype):
    Q, K, V, dO, kw = make(dict(shape=(4, 2, 5, 9, 5, 9, max(d, dv)), heads=2, causal=True), dtype)
    Q, K, V, dO = (t[..., :n].contiguous() for t, n in ((Q, d), (K, d), (V, dv), (dO, dv)))
    want, tol = ref.attend_all(Q, K, V, dO, **kw)
    out = torch.full_like(dO, 7.0)
    assert scram.dense_attend(Q, K, V, out=out, **kw) is out
    got = [out, *scram.dense_attend_backward(Q, K, V, dO, **kw)]
    for name, g, w, t in zip(("out", "dQ", "dK", "dV", "dbias"), got, want, tol):
        assert g.shape == w.shape
        near(g, w, t, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 2, 10, 20, 10, 20, 64), (128, 128, 10, 20, 10, 20, 64), (2, 2, 1, 2, 30, 40, 32)])
@pytest.mark.parametrize("heads", [0, 2])
def test_far_larger_scores_behind_the_first_keys(scram, shape, heads, dtype):
    """A few late keys outdo the others by more than any fixed shift bears: by hundreds, for some queries only."""
    S, Sk, Hq, Wq, Hk, Wk, d = shape
    gen = torch.Generator(device="cuda").manual_seed(9)
    Q, K, V, dO = (torch.randn(*s, generator=gen, device="cuda") for s in ((S, Hq, Wq, d), (Sk, Hk, Wk, d), (Sk, Hk, Wk, d), (S, Hq, Wq, d)))
    K = 0.1 * K
    late = K.view(Sk, -1, d)[:, -3:]
    late += 12.0
    Q.view(S, -1, d)[:, ::2] += 3.0   # scores of some 36 d^(1/2) there; of the other queries to both sides
    kw = dict(bias=torch.randn(heads, 2 * Hk - 1, 2 * Wk - 1, generator=gen, device="cuda").to(TYPES[dtype]) if heads else None)
    Q, K, V, dO = (t.to(TYPES[dtype]) for t in (Q, K, V, dO))
    want, tol = ref.attend_all(Q, K, V, dO, **kw)
    got = [scram.dense_attend(Q, K, V, **kw), *scram.dense_attend_backward(Q, K, V, dO, **kw)]
    for name, g, w, t in zip(("out", "dQ", "dK", "dV", "dbias"), got, want, tol):
        near(g, w, t, name)


def test_two_graphs_share_a_workspace(scram):
    """Replayed in turn on one stream, in both orders."""
    cases = [dict(shape=(4, 2, 1, 300, 1, 300, 64), heads=2, causal=True), dict(shape=(2, 2, 9, 31, 9, 31, 64), heads=1)]
    sizes, calls = [], []
    for c in cases:
        S, Sk, Hq, Wq, Hk, Wk, d = c["shape"]
        sizes += [scram.dense_attend_backward_workspace_bytes(S, Sk, Hq, Wq, Hk, Wk, d=d, dtype=torch.bfloat16, heads=c["heads"]),
                  scram.dense_attend_workspace_bytes(S, Sk, Hq, Wq, Hk, Wk, d=d, dtype=torch.bfloat16, bias=True)]
    ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
    for c in cases:
        Q, K, V, dO, kw = make(c, "bf16")
        calls.append(lambda Q=Q, K=K, V=V, dO=dO, kw=kw: [scram.dense_attend(Q, K, V, workspace=ws, **kw),
                                                         *scram.dense_attend_backward(Q, K, V, dO, workspace=ws, **kw)])
    want = [call() for call in calls]
    torch.cuda.synchronize()
    graphs, held = [torch.cuda.CUDAGraph() for _ in calls], []
    for graph, call in zip(graphs, calls):
        with torch.cuda.graph(graph):
            held.append(call())
    for turn in ((0, 1), (1, 0), (1, 1), (0, 0)):
        for t in held[0] + held[1]:
            t.fill_(7.0)
        for i in turn:
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in set(turn):
            for a, b in zip(held[i], want[i]):
                assert torch.equal(a, b)


def test_places_past_32_bits(scram):
    """The last slice of a cache of more than 2^31 numbers, one query and one key block's gradients."""
    Sk, n, d = 17, 1_000_003, 128
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    gen = torch.Generator(device="cuda").manual_seed(1)
    K, V = (torch.randn(Sk, 1, n, d, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    Q, dO = (torch.randn(Sk, 1, 1, d, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    Q = 2 * Q  # (the larger weights are some thousandths)
    assert K.numel() > 2 ** 31
    out = scram.dense_attend(Q, K, V)
    dQ, dK, dV = scram.dense_attend_backward(Q, K, V, dO)
    for s in (0, Sk - 1):
        want, tol = ref.attend_all(*(t[s:s + 1] for t in (Q, K, V, dO)))
        for name, g, w, t in zip(("out", "dQ", "dK", "dV"), (out, dQ, dK, dV), want, tol):
            near(g[s:s + 1], w, t, f"{name} of slice {s}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_other_dispatch_order(scram, dtype):
    """The same bits whichever blocks take which part of the work, and in which order."""
    from paper_1905_10308_amd import binding

    runs = []
    for c in (dict(shape=(6, 3, 9, 40, 9, 40, 64), heads=2, causal=True), dict(shape=(128, 64, 15, 17, 15, 17, 64), heads=4),
              dict(shape=(1, 1, 1, 1, 40, 41, 64))):
        Q, K, V, dO, kw = make(c, dtype)
        runs.append(lambda Q=Q, K=K, V=V, dO=dO, kw=kw: [scram.dense_attend(Q, K, V, **kw), *scram.dense_attend_backward(Q, K, V, dO, **kw)])
    x = torch.randn(3, 33, 21, 60, device="cuda").to(TYPES[dtype])

    def norm():
        y, mean, rstd = scram.group_norm(x, 6, activation="silu", stats=True)
        return [y, mean, rstd, *[t for t in scram.group_norm_backward(y, x, mean, rstd, activation="silu") if t is not None]]

    runs.append(norm)
    want = [run() for run in runs]
    saved = binding.lib()
    binding._lib = binding.load(binding.ORDER_LIB_PATH)
    try:
        for run, w in zip(runs, want):
            for a, b in zip(run(), w):
                assert torch.equal(a, b)
    finally:
        binding._lib = saved
