"""Rotary grid positions and layer norm against their 64-bit definitions, through the public entry points."""
import pytest

torch = pytest.importorskip("torch")
import layer_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def near(got, want, tol, what=""):
    off = (got.double() - want).abs()
    assert got.isfinite().all(), f"{what}: not finite"
    assert (off <= tol).all(), f"{what}: off by {float(off.max()):.3e}, {float((off / tol.clamp(min=1e-300)).max()):.2f} of its tolerance"


def skewed(shape, kind, gen, by):
    """A contiguous tensor that starts `by` elements into its storage."""
    n = 1
    for s in shape:
        n *= s
    store = torch.empty(n + by, dtype=kind, device="cuda")
    t = store[by:].view(shape)
    t.copy_(torch.randn(shape, generator=gen, device="cuda"))
    return t


def rotary_tolerance(x, want, P, groups, interleaved, reach):
    """Per element: cos and sin to 4 roundings (the series' first left-out terms are below 2^-27, the angle's own rounding and
    the argument's 2 together), two products and a sum; the frequencies are held to 2^-53 of their value, so an angle is off by
    `reach` times that; and the result's rounding."""
    y = x.double().abs().reshape(*x.shape[:4], groups, -1)
    pair = torch.zeros_like(y)
    for k in range(P):
        i, j = (2 * k, 2 * k + 1) if interleaved else (k, k + P)
        pair[..., i] = pair[..., j] = y[..., i] + y[..., j]
    tol = pair.reshape(x.shape) * (7 * ref.U32 + reach * 2.0 ** -51)
    return tol + ref.HALF[x.dtype] * want.abs() * (pair.reshape(x.shape) > 0) * (x.dtype == torch.bfloat16) * 1.01


ROTARY = [
    dict(shape=(2, 1, 5, 7, 16), sections=(0, 4, 4)),
    dict(shape=(3, 4, 5, 6, 64), sections=(8, 12, 12)),
    dict(shape=(2, 1, 33, 17, 128), sections=(0, 16, 16), groups=2),
    dict(shape=(1, 2, 3, 3, 100), sections=(12, 17, 17)),
    dict(shape=(2, 3, 4, 5, 46), sections=(5, 7, 8)),
    dict(shape=(2, 1, 3, 4, 42), sections=(0, 3, 4), groups=3),
    dict(shape=(1, 1, 1, 1, 2), sections=(0, 0, 1)),
    dict(shape=(7, 1, 1, 1, 64), sections=(4, 6, 6), groups=2),
    dict(shape=(1, 9, 1, 1, 8), sections=(3, 0, 0)),
    dict(shape=(1, 1, 40, 300, 256), sections=(0, 64, 64)),
    dict(shape=(130, 1, 4, 4, 32), sections=(0, 8, 8)),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("c", ROTARY, ids=lambda c: "x".join(map(str, c["shape"])))
def test_rotary(scram, c, interleaved, dtype):
    gen = torch.Generator(device="cuda").manual_seed(1)
    S, groups, P = c["shape"][0], c.get("groups", 1), sum(c["sections"])
    freqs = ref.frequencies(c["sections"])
    kw = dict(sections=c["sections"], groups=groups, interleaved=interleaved)
    for by in (0, 1, 4):
        x, y = skewed(c["shape"], TYPES[dtype], gen, by), skewed((2,) + c["shape"][1:], TYPES[dtype], gen, by)
        origins = [(5, 3, 11), torch.tensor([4000, -77, 2 ** 20], dtype=torch.int32, device="cuda"),
                   torch.randint(-2 ** 31, 2 ** 31 - 1, (S, 3), generator=gen, device="cuda").to(torch.int32)]
        for origin in origins:
            o = torch.as_tensor(origin, device="cuda").reshape(-1, 3)
            tensors = (x, y) if o.shape[0] in (1, 2) and S != 1 else (x,)
            for inverse, call in ((False, scram.rotary), (True, scram.rotary_backward)):
                got = call(*tensors, origin=origin, **kw)
                for t, g in zip(tensors, got if len(tensors) > 1 else (got,)):
                    if o.shape[0] > 1 and t.shape[0] != o.shape[0]:
                        continue
                    want = ref.rotary(t, c["sections"], freqs, o, groups, interleaved, inverse)
                    near(g, want, rotary_tolerance(t, want, P, groups, interleaved, 2.0 ** 31 if o.shape[0] > 1 else 2.0 ** 21), f"skew {by}")
        where = x.clone()
        assert scram.rotary(where, out=where, origin=origins[0], **kw) is where
        assert torch.equal(where, scram.rotary(x, origin=origins[0], **kw))


def test_rotary_defaults_own_frequencies_and_images(scram):
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(2, 6, 8, 24, generator=gen, device="cuda")
    five = x[:, None]
    assert torch.equal(scram.rotary(x), scram.rotary(five, sections=(0, 6, 6))[:, 0])
    assert torch.equal(scram.rotary(x, sections=(6, 6)), scram.rotary(x))
    f = [0.5, -0.25, 3.0]
    near(scram.rotary(x, sections=(0, 1, 2), freqs=f), ref.rotary(five, (0, 1, 2), f, torch.zeros(1, 3, device="cuda"))[:, 0], torch.full((1,), 1e-5, device="cuda", dtype=torch.float64))
    clip = torch.randn(1, 3, 4, 5, 12, generator=gen, device="cuda")
    assert torch.equal(scram.rotary(clip), scram.rotary(clip, sections=(2, 2, 2)))
    assert torch.equal(scram.rotary(x, origin=(3, 4)), scram.rotary(x, origin=(0, 3, 4)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("slices,per_slice", [((1,), False), ((70001, 5), False), ((4099, 4099), True), ((3, 300, 2047, 2049), False)])
def test_rotary_of_single_pixels(scram, slices, per_slice, dtype):
    """Many slices of one pixel: their rows share blocks."""
    gen = torch.Generator(device="cuda").manual_seed(19)
    xs = [torch.randn(s, 1, 1, 20, generator=gen, device="cuda").to(TYPES[dtype]) for s in slices]
    at = torch.randint(-3000, 3000, (slices[0] if per_slice else 1, 3), generator=gen, device="cuda", dtype=torch.int32)
    freqs = [10000.0 ** (-j / m) for m in (4, 5) for j in range(m)]
    got = scram.rotary(*xs, origin=at, sections=(4, 5))
    for x, y in zip(xs, got if len(xs) > 1 else [got]):
        want = ref.rotary(x[:, None], (0, 4, 5), freqs, at)
        near(y[:, None], want, rotary_tolerance(x[:, None], want, 9, 1, False, 3001), "pixels")


def test_rotary_of_the_most_slices(scram):
    """2^31 - 1 slices of one pixel of two channels: the last ones are turned."""
    n = (1 << 31) - 1
    x = torch.zeros(n, 1, 1, 2, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(4096, 1, 1, 2, generator=torch.Generator(device="cuda").manual_seed(20), device="cuda").bfloat16()
    x[-4096:], x[:4096] = tail, tail
    scram.rotary(x, origin=(0, 2, 0), sections=(1, 0), out=x)
    want = ref.rotary(tail[:, None], (0, 1, 0), [1.0], torch.tensor([[0, 2, 0]], device="cuda"))
    for y in (x[-4096:], x[:4096]):
        near(y[:, None], want, rotary_tolerance(tail[:, None], want, 1, 1, False, 3), "slices")


def test_rotary_replays(scram):
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(8, 1, 1, 64, generator=gen, device="cuda").bfloat16()
    at = torch.zeros(8, 3, dtype=torch.int32, device="cuda")
    scram.rotary(x, origin=at, groups=2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = scram.rotary(x, origin=at, groups=2)
    for _ in range(3):  # the next position, read on the device
        at.add_(torch.tensor([0, 1, 5], dtype=torch.int32, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, scram.rotary(x, origin=at, groups=2))


CHANNELS = [1, 2, 3, 7, 8, 31, 32, 64, 65, 100, 128, 256, 512, 520, 1000, 1024, 1026, 2047, 4096, 5000, 8192, 9001, 12004, 16384]


@pytest.mark.parametrize("kind", ["f32", "bf16", "bf16_f32"])
@pytest.mark.parametrize("C", CHANNELS)
def test_layer_norm(scram, C, kind):
    gen = torch.Generator(device="cuda").manual_seed(C)
    T, TG = TYPES[kind.split("_")[0]], TYPES[kind.split("_")[-1]]
    for rows, offset, by, weights in ((1, 0.0, 0, "own"), (5, 30.0, 0, "f32"), (67, -3.0, 1, "own"), (600 if C <= 1024 else 33, 1.0, 2, None), (1100 if C < 600 else 7, 0.5, 4, "own")):
        x = skewed((rows, C), T, gen, by)
        x.add_(offset)
        kw = {}
        w = b = None
        if weights:
            w, b = ((1.0 + torch.randn(C, generator=gen, device="cuda")).to(T if weights == "own" else torch.float32) for _ in range(2))
            kw = dict(weight=w, bias=b)
        y, mean, rstd = scram.layer_norm(x, **kw, stats=True)
        wy, wm, wr = ref.layer_norm(x, w, b, 1e-5)
        xd = x.double()
        # the mean: a sum of C terms in a tree, at most C / 64 + 16 deep; the centred values carry its error and a rounding of
        # their own, the deviation twice that; eps keeps a row of equal values bounded
        depth = C / 64 + 24
        dm = depth * ref.U32 * xd.abs().mean(1)
        near(mean, wm, dm + 1e-30, "mean")
        dx_off = (dm + ref.U32 * xd.abs().amax(1))  # of one centred value
        var = 1.0 / wr ** 2
        rel = (depth * ref.U32 + dx_off * (var - 1e-5).clamp(min=0).sqrt() * 2 / var + dx_off ** 2 / var)
        near(rstd, wr, wr * rel + 1e-30, "rstd")
        xh = (xd - wm[:, None]) * wr[:, None]
        wf = torch.ones_like(xd[0]) if w is None else w.double().abs()
        tol = wf * (dx_off[:, None] * wr[:, None] + xh.abs() * (rel[:, None] + 4 * ref.U32)) + 2 * ref.U32 * wy.abs() + 1e-30
        near(y, wy, tol + ref.HALF[T] * (wy.abs() + tol) * (T == torch.bfloat16), "rows")
        # in place (on a copy, whose alignment and so order of summation may be another)
        where = x.clone()
        apart = scram.layer_norm(where, **kw)
        assert scram.layer_norm(where, **kw, out=where) is where and torch.equal(where, apart)

        dy = skewed((rows, C), TG, gen, by)
        got = scram.layer_norm_backward(dy, x, mean, rstd, w)
        want = ref.layer_norm_backward(dy, x, mean, rstd, w)
        assert got[0].dtype == TG and got[1].dtype == got[2].dtype == torch.float32
        m, r, dyd = mean.double()[:, None], rstd.double()[:, None], dy.double().abs()
        xa = ((xd - m) * r).abs()
        g = dyd * wf
        tol = r * (3 * g + (depth + 4) * (g.mean(1, keepdim=True) + xa * (g * xa).mean(1, keepdim=True)) + 4 * xa * (g * xa).mean(1, keepdim=True)) * ref.U32 * 2 + 1e-30
        near(got[0], want[0], tol + ref.HALF[TG] * (want[0].abs() + tol) * (TG == torch.bfloat16), "dX")
        # a column: the rows of a block one after another, then the blocks
        many = (rows + 40) * ref.U32
        near(got[1], want[1], (dyd * xa).sum(0) * (many + 4 * ref.U32) + 1e-30, "dweight")
        near(got[2], want[2], dyd.sum(0) * many + 1e-30, "dbias")
        again = scram.layer_norm_backward(dy, x, mean, rstd, w)
        assert all(torch.equal(p, q) for p, q in zip(got, again))
        place = dy.clone()
        apart = scram.layer_norm_backward(place, x, mean, rstd, w)
        assert all(torch.equal(p, q) for p, q in zip(scram.layer_norm_backward(place, x, mean, rstd, w, out=place), apart))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_rows_of_equal_values_and_not_finite_ones(scram, dtype):
    x = torch.full((6, 64), 3.0, dtype=TYPES[dtype], device="cuda")
    x[1], x[3, 5], x[4, 0] = 1e4, float("nan"), float("inf")
    b = torch.arange(64, device="cuda", dtype=torch.float32)
    y = scram.layer_norm(x, None, b)
    for i in (0, 1, 2, 5):  # their deviation is 0
        assert torch.equal(y[i].float(), b.to(y.dtype).float())
    assert y[3].isnan().all() and y[4].isnan().all()
    z = scram.layer_norm(torch.ones(4, 1, device="cuda"), eps=0.0)
    assert z.isnan().all()  # 0 / 0, as the definition has it


def test_layer_norm_large(scram):
    """More rows than one pass of the grid takes, and rows past 4 GiB."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(1 << 16, 64, generator=gen, device="cuda").bfloat16().repeat(600, 1)  # 5 GB
    y, mean, rstd = scram.layer_norm(x, stats=True)
    few = slice(x.shape[0] - 5000, None)
    wy, wm, wr = ref.layer_norm(x[few], None, None, 1e-5)
    near(mean[few], wm, torch.full((1,), 1e-6, device="cuda", dtype=torch.float64))
    near(y[few], wy, 2.0 ** -8 * wy.abs() + 1e-5)
    assert torch.equal(y[:1 << 16], y[-(1 << 16):])
    dX, dw, db = scram.layer_norm_backward(y, x, mean, rstd)
    part = scram.layer_norm_backward(y[:1 << 16], x[:1 << 16], mean[:1 << 16], rstd[:1 << 16])
    assert torch.equal(dX[-(1 << 16):], part[0])
    # 600 times the same rows: sums of 39 million terms against those of a 600th
    total = (y[:1 << 16].double().abs() * 4).sum(0) * 600
    near(dw, part[1].double() * 600, total * 4e-5)
    near(db, part[2].double() * 600, total * 4e-5)


def test_norm_replays_and_streams(scram):
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(3000, 96, generator=gen, device="cuda").bfloat16()
    w = torch.randn(96, generator=gen, device="cuda").bfloat16()
    dy = torch.randn(3000, 96, generator=gen, device="cuda")

    def step():
        y, mean, rstd = scram.layer_norm(x, w, w, stats=True)
        return (y, *scram.layer_norm_backward(dy, x, mean, rstd, w))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caught = step()
    for _ in range(3):
        x.copy_(torch.randn(3000, 96, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(caught, step()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, step()))
