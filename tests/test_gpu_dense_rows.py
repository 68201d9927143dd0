"""The bias by buckets and group norm against their 64-bit definitions, through the public entry points."""
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


GRIDS = [
    (1, 1, 1, (), ()),
    (3, 1, 40, (), (1, 2, 5, 11)),
    (2, 5, 7, (1, 2, 3), (2, 4)),
    (4, 9, 3, (3,), (1, 2, 3, 4, 5, 100)),     # edges past the grid: buckets without an offset
    (1, 33, 65, tuple(range(1, 40)), tuple(range(1, 65))),
    (130, 4, 6, (1,), (1, 3)),
    (2, 70, 300, (4, 9, 30), (1, 2, 3, 5, 9, 17, 33, 65, 129)),
    (1, 1, 5000, (), (1, 10, 100, 1000)),
    (1, 300, 1, (7, 70), ()),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", GRIDS, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}")
def test_relative_bias(scram, c, dtype):
    heads, H, W, ey, ex = c
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = torch.randn(heads, 2 * len(ey) + 1, 2 * len(ex) + 1, generator=gen, device="cuda").to(TYPES[dtype])
    want = ref.relative_bias(table, H, W, (ey, ex))
    got = scram.relative_bias(table, H, W, edges=(ey, ex))
    assert got.dtype == table.dtype and torch.equal(got, want)
    out = torch.full_like(got, math.nan)
    assert scram.relative_bias(table, H, W, edges=(ey, ex), out=out) is out and torch.equal(out, want)
    d = torch.randn(got.shape, generator=gen, device="cuda").to(TYPES[dtype])
    want, reach = ref.relative_bias_backward(d, (ey, ex))
    got = scram.relative_bias_backward(d, edges=(ey, ex))
    assert got.dtype == d.dtype and got.shape == table.shape
    # a cell's rows one after another, and a row's values: at most so many roundings
    near(got, want, (H + W) * ref.U32 * reach + ref.HALF[TYPES[dtype]] * want.abs())
    ws = torch.full((scram.relative_bias_backward_workspace_bytes(heads, H, W, len(ex)),), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(scram.relative_bias_backward(d, edges=(ey, ex), workspace=ws), got)


def test_default_edges(scram):
    table = torch.randn(2, 5, 9, device="cuda")
    edges = (scram.bias_edges(2, 11), scram.bias_edges(4, 19))
    assert edges == ((1, 11), (1, 2, 6, 19))
    assert torch.equal(scram.relative_bias(table, 12, 20), scram.relative_bias(table, 12, 20, edges=edges))


def test_relative_bias_refusals(scram):
    t = torch.randn(2, 5, 3, device="cuda")
    d = torch.randn(2, 7, 9, device="cuda")
    for call in (lambda: scram.relative_bias(t, 4, 5, edges=((1, 2), ())), lambda: scram.relative_bias(t, 4, 5, edges=((2, 2), (1,))),
                 lambda: scram.relative_bias(t, 4, 5, edges=((0, 2), (1,))), lambda: scram.relative_bias(t, 0, 5),
                 lambda: scram.relative_bias(t[:, :4].contiguous(), 4, 5), lambda: scram.relative_bias(t, 1 << 31, 1),
                 lambda: scram.relative_bias(t.cpu(), 4, 5), lambda: scram.relative_bias_backward(d[:, 1:].contiguous(), edges=((1,), (1,))),
                 lambda: scram.relative_bias_backward(d, edges=(tuple(range(1, 70)), ())),
                 lambda: scram.relative_bias(t, 4, 5, out=torch.empty(2, 7, 8, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        scram.relative_bias(t.half(), 4, 5)
    with pytest.raises(scram.ScramError):
        scram.relative_bias_backward(d, edges=((1,), (1,)), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


IMAGES = [  # shape, groups
    ((1, 1, 1, 1), 1),
    ((2, 8, 8, 64), 8),
    ((3, 7, 9, 100), 20),
    ((1, 5, 5, 24), 24),
    ((2, 1, 1, 32), 4),
    ((2, 33, 17, 12), 3),
    ((1, 40, 50, 7), 7),
    ((4, 3, 3, 1000), 8),
    ((1, 2, 2, 2056), 1),
    ((2, 3, 5, 2049), 3),
    ((1, 2, 3, 16384), 32),
    ((5, 128, 3), 3),
    ((2, 70, 90, 48), 4),
    ((1, 300, 5), 1),
    ((1500, 3, 4), 2),
]


def image(shape, groups, dtype, seed, by=0, at=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    n = math.prod(shape)
    store = torch.empty(n + by, dtype=TYPES[dtype], device="cuda")
    x = store[by:].view(shape)
    x.copy_(normal(*shape) * (0.5 + torch.rand(shape[-1], generator=gen, device="cuda")) + normal(shape[-1]) + at)
    C = shape[-1]
    return x, 1.0 + 0.3 * normal(C), 0.3 * normal(C), normal(*shape)


def joins(shape, kind):
    """Most steps in which the statistics of a group of these images are joined, one after another (half of them bounds what
    their roundings add up to: a step's is shrunk by the weights of those after it)."""
    return 2 * (64 + shape[-1] + math.prod(shape[1:-1]) // 2)


@pytest.mark.parametrize("act", [None, "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,groups", IMAGES, ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))
def test_group_norm(scram, shape, groups, dtype, act):
    kind = TYPES[dtype]
    x, w, b, dy = image(shape, groups, dtype, 1)
    N, C = shape[0], shape[-1]
    U = ref.U32
    for weight, bias, eps in ((w, b, 1e-5), (w.to(kind), b.to(kind), 1e-3), (None, None, 1e-5), (None, b.to(kind), 1e-5)):
        y, mean, rstd = scram.group_norm(x, groups, weight, bias, eps, activation=act, stats=True)
        want, wm, wr = ref.group_norm(x, groups, weight, bias, eps, act)
        assert y.dtype == kind and mean.shape == rstd.shape == (N, groups)
        each = x.double().reshape(N, -1, groups, C // groups)
        most = each.abs().amax((1, 3))
        spread = (each - wm[:, None, :, None]).abs().amax((1, 3))
        n = min(joins(shape, kind), 300)
        mean_tol = U * (2 * most + n * spread)
        near(mean, wm, mean_tol)
        # squares: each to a few roundings, their sum to one a step; what the means are off, against the spread
        rel = U * (n + 12) + 2 * mean_tol * wr
        near(rstd, wr, wr * (rel + (mean_tol * wr) ** 2))
        wide = lambda t: t[:, None, :, None].expand_as(each).reshape(shape)  # noqa: E731
        ws = 1.0 if weight is None else weight.double()
        z = ref.group_norm(x, groups, weight, bias, eps)[0]
        bb = 0.0 if bias is None else bias.double()
        z_tol = (ws * wide(wr * (mean_tol + U * most))).abs() + (z - bb).abs() * (wide(rel + (mean_tol * wr) ** 2) + 6 * U) + U * (4 * z.abs())
        near(y, want, 1.1 * z_tol + 8 * U * want.abs() + ref.HALF[kind] * want.abs() + 1e-37, f"{shape}")
        assert torch.equal(scram.group_norm(x, groups, weight, bias, eps, activation=act), y)
        if N * C < 3000:
            again = x.clone()
            assert scram.group_norm(again, groups, weight, bias, eps, activation=act, out=again) is again and torch.equal(again, y)
        for grad in {dtype, "f32"}:
            d = dy.to(TYPES[grad])
            got = scram.group_norm_backward(d, x, mean, rstd, weight, bias, activation=act)
            want_g, reach = ref.group_norm_backward(d, x, mean, rstd, weight, bias, act)
            count = math.prod(shape[1:-1]) * (C // groups)
            # the activation's slope to 12 roundings, products and means to one each; sums over at most `count` values
            steps = 24 + 4 * math.sqrt(count) + 300
            zr = (z.abs() + 1) if act else 1.0
            near(got[0], want_g[0], steps * U * zr * reach[0] * (3 if act else 1) + 4 * U * zr * wide(most * wr ** 2) * dy.abs().max() + ref.HALF[TYPES[grad]] * want_g[0].abs() + 1e-37, f"dX {shape}")
            assert got[0].dtype == d.dtype and got[1].dtype == got[2].dtype == torch.float32
            sums = (24 + N + math.prod(shape[1:-1])) * U * 12
            near(got[1], want_g[1], sums * reach[1] + 4 * U * (d.double().abs() * wide(most * wr)).reshape(-1, C).sum(0) + 1e-37, "dweight")
            near(got[2], want_g[2], sums * reach[2] + 1e-37, "dbias")
            if N * C < 3000:
                assert scram.group_norm_backward(d, x, mean, rstd, weight, bias, activation=act, out=d)[0] is d
                assert torch.equal(d, got[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("by", [1, 3])
def test_any_alignment(scram, dtype, by):
    """Images that start at any element of their storage give the same bits."""
    x, w, b, dy = image((2, 9, 11, 20), 5, dtype, 2, by)
    y, mean, rstd = scram.group_norm(x, 5, w, b, activation="silu", stats=True)
    want = scram.group_norm(x.clone(), 5, w, b, activation="silu", stats=True)
    assert all(torch.equal(a, c) for a, c in zip((y, mean, rstd), want))
    store = torch.empty(dy.numel() + by, dtype=x.dtype, device="cuda")
    d = store[by:].view(dy.shape).copy_(dy)
    got = scram.group_norm_backward(d, x, mean, rstd, w, b, activation="silu")
    want = scram.group_norm_backward(d.clone(), x.clone(), mean, rstd, w, b, activation="silu")
    assert all(torch.equal(a, c) for a, c in zip(got, want))


def test_an_offset_costs_no_accuracy(scram):
    """4096 +- 1: sums of squares in fp32 would leave nothing of the variance of 1."""
    x = torch.full((2, 16, 16, 32), 4096.0, device="cuda")
    x[:, ::2] += 1.0
    x[:, 1::2] -= 1.0
    x[:, 0, 0] = 0.0  # an outlier where a shift would be taken from
    x[:, 0, 0] = 4097.0
    y, mean, rstd = scram.group_norm(x, 4, eps=0.0, stats=True)
    # the means' roundings: half a step of 4096, 2^-12, each
    assert float((mean - 4096.0).abs().max()) <= 4 * 2.0 ** -12
    assert float((rstd - 1.0).abs().max()) <= 1e-4


def test_extremes(scram):
    """Values that are not finite stay in their image and group; an image of equal values gives the bias."""
    x, w, b, dy = image((3, 6, 6, 16), 4, "f32", 3)
    x[1, 2, 3, 5] = math.nan
    x[2, 0, 0, 0] = math.inf
    y = scram.group_norm(x, 4, w, b, activation="silu")
    bad = ~y.isfinite().all(1).all(1)
    want = torch.zeros(3, 16, dtype=torch.bool, device="cuda")
    want[1, 4:8] = want[2, :4] = True
    assert torch.equal(bad, want)
    same = torch.full((2, 5, 7, 16), 3.25, device="cuda")
    assert torch.equal(scram.group_norm(same, 4, w, b), b.expand(2, 5, 7, 16))
    big = scram.group_norm(torch.tensor([[[-200.0], [200.0]]], device="cuda") * 1e3, 1, torch.full((1,), 500.0, device="cuda"), activation="silu")
    assert big.flatten().tolist()[0] == 0.0 and abs(big.flatten().tolist()[1] - 500.0) < 1e-3


def test_group_norm_graph_and_refusals(scram):
    x, w, b, dy = image((2, 30, 40, 40), 5, "bf16", 4)
    dy = dy.bfloat16()
    n = max(scram.group_norm_workspace_bytes(2, 1200, 40, 5, dtype=torch.bfloat16),
            scram.group_norm_backward_workspace_bytes(2, 1200, 40, 5, dtype=torch.bfloat16))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def call():
        y, m, r = scram.group_norm(x, 5, w, b, activation="silu", stats=True, workspace=ws)
        return [y, m, r, *scram.group_norm_backward(dy, x, m, r, w, b, activation="silu", workspace=ws)]

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed in range(5, 8):
        x.copy_(image((2, 30, 40, 40), 5, "bf16", seed)[0])
        graph.replay()
        got = [t.clone() for t in held]
        assert all(torch.equal(a, c) for a, c in zip(got, call()))
    y, m, r = scram.group_norm(x, 5, w, b, stats=True)
    for kind, f in ((ValueError, lambda: scram.group_norm(x, 7)), (ValueError, lambda: scram.group_norm(x, 0)),
                    (ValueError, lambda: scram.group_norm(x, 5, activation="tanh")), (ValueError, lambda: scram.group_norm(x, 5, w[:3])),
                    (TypeError, lambda: scram.group_norm(x, 5, w.double())), (ValueError, lambda: scram.group_norm(x[..., ::2], 5)),
                    (ValueError, lambda: scram.group_norm(x[0, 0, 0], 5)), (TypeError, lambda: scram.group_norm(x.half(), 5)),
                    (ValueError, lambda: scram.group_norm_backward(dy[:1], x, m, r)), (ValueError, lambda: scram.group_norm_backward(dy, x, m[:1], r)),
                    (TypeError, lambda: scram.group_norm_backward(dy.double(), x, m, r)),
                    (scram.ScramError, lambda: scram.group_norm(x, 5, workspace=ws[:256])),
                    (scram.ScramError, lambda: scram.group_norm(x, 5, eps=-1.0))):
        with pytest.raises(kind):
            f()
