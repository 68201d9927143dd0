"""Differential attention and its gradients where rows lie past 4 GiB: within a slice, and in later slices."""
import pytest

torch = pytest.importorskip("torch")
import layer_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu


def check(got, want, tol, what):
    off = (got.double() - want).abs()
    assert got.isfinite().all() and (off <= tol).all(), f"{what}: off by {float(off.max()):.3e}, {float((off / tol).max()):.2f} of its tolerance"


# slices that the matrix cores must leave (over 4 GiB of key rows each), slices that they take, both types
@pytest.mark.parametrize("S,H,W,d,dtype", [(1, 4200, 8192, 64, "bf16"), (40, 1024, 1024, 64, "bf16"), (1, 8300, 16384, 16, "bf16"),
                                           (20, 1024, 1024, 64, "f32"), (1, 2100, 8192, 64, "f32")])
def test_rows_past_4_gib(scram, S, H, W, d, dtype):
    """Every query near its own place: the last corner's results are those of a small grid of its own."""
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    gen = torch.Generator(device="cuda").manual_seed(51)
    Q, K, V, dO = (torch.empty(S, H, W, d, dtype=kind, device="cuda").normal_(generator=gen) for _ in range(4))
    at = torch.arange(H * W, dtype=torch.int32, device="cuda").reshape(H, W)
    J = torch.stack([at, (at + 1).clamp(max=H * W - 1)])[:, None].expand(2, S, H, W).contiguous()
    lam = torch.rand(S, generator=gen, device="cuda")
    out = scram.differential_attend(Q, K, V, J, lam, 3)
    dQ, dK, dV, dlam = scram.differential_attend_backward(Q, K, V, J, lam, dO, 3)
    assert dlam.isfinite().all()
    # the last slice's last 8 rows of the last 14 columns; windows reach two columns and a row further, gradients twice that
    h, w = 8, 14
    corner = lambda t: t[-1:, H - h:, W - w:].contiguous()  # noqa: E731
    small = [corner(t) for t in (Q, K, V, dO)]
    own = torch.arange(h * w, device="cuda").reshape(h, w)
    mine = torch.stack([own, (own + 1).clamp(max=h * w - 1)])[:, None]
    mask = ref.key_mask(mine, h, w, h, w, 3)
    got = [corner(t) for t in (out, dQ, dK, dV)]
    want, tol, wg, tg = ref.differential(*small[:3], mask, lam[-1:], (d // 2) ** -0.5, small[3])
    tol = tol + ref.HALF[kind] * (want.abs() + tol)
    shaped = lambda t: t.reshape(1, h, w, d)  # noqa: E731
    # the last column's second window lies at the first column of the next row, elsewhere in the small grid: left out with what
    # it touches
    check(got[0][:, 3:, 4:-1], shaped(want)[:, 3:, 4:-1], shaped(tol)[:, 3:, 4:-1], "output")
    check(got[1][:, 3:, 4:-1], shaped(wg[0])[:, 3:, 4:-1], shaped(tg[0])[:, 3:, 4:-1], "dQ")
    for name, g, x, t in (("dK", got[2], wg[1], tg[1]), ("dV", got[3], wg[2], tg[2])):
        check(g[:, 4:, 6:-2], shaped(x)[:, 4:, 6:-2], shaped(t)[:, 4:, 6:-2], name)
