"""Rotary positions and layer norm at the ends of their ranges, through the public entry points."""
from fractions import Fraction

import pytest

torch = pytest.importorskip("torch")
import layer_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
PI = Fraction(314159265358979323846264338327950288419716939937510582097494459230781640628620899, 10 ** 80)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("size", [3.0, 0.25, 1e-4, 1e-6, 1e-9])
@pytest.mark.parametrize("at", [2 ** 31 - 1, -2 ** 31, 1500000001])
def test_rotary_at_the_ends_of_the_positions(scram, at, size, sign):
    """(1, 0) turned by at * freq, the angle from whole numbers.

    A frequency is off by 2^-52 of its value (the division by a turn and that constant's own rounding) and 2^-65 of a turn, an
    angle by |at| times that; cos and sin are within 7 roundings of 2^-24 (the series, its argument, the product and the sum).
    """
    P = 128
    freqs = [sign * size * (1.0 + k / 173.0) for k in range(P)]
    x = torch.zeros(1, 1, 1, 2 * P, device="cuda")
    x[..., :P] = 1.0
    for inverse, call in ((1, scram.rotary), (-1, scram.rotary_backward)):
        y = call(x, sections=(0, P), freqs=freqs, origin=(0, 0, at)).flatten().double().cpu()
        t = torch.tensor([float(inverse * at * Fraction(f) % (2 * PI)) for f in freqs], dtype=torch.float64)
        for got, want in ((y[:P], t.cos()), (y[P:], t.sin())):
            tol = 7 * ref.U32 + abs(at) * (2 * torch.tensor(freqs, dtype=torch.float64).abs() * 2.0 ** -53 + 6.3 * 2.0 ** -65)
            off = (got - want).abs()
            assert (off <= tol).all(), f"off by {float(off.max()):.3e}, {float((off / tol).max()):.2f} of its tolerance"


@pytest.mark.parametrize("C", [1, 2, 4, 8, 16, 20, 24, 100, 1026])
@pytest.mark.parametrize("eps,size", [(1e-5, 2.0 ** 120), (1e-30, 2.0 ** 90), (1e-5, 1.0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_of_rows_far_from_zero(scram, dtype, eps, size, C):
    """Rows of one large number, by their exact statistics: the channels that a row does not fill take no part.

    xh is exactly 0, so dX = rstd (g - mean g) and dweight = 0.  g's sum is rounded at most C + 6 times, the mean, the difference
    and the product 4 times: each a rounding of at most the sum of |g| / C, or |g|, times rstd.
    """
    gen = torch.Generator(device="cuda").manual_seed(41)
    rows, kind = 37, TYPES[dtype]
    X = torch.full((rows, C), size, dtype=kind, device="cuda")
    mean = torch.full((rows,), size, device="cuda")
    rstd = torch.full((rows,), eps ** -0.5, device="cuda")
    dY = torch.randn(rows, C, generator=gen, device="cuda")
    w = torch.randn(C, generator=gen, device="cuda")
    dX, dweight, dbias = scram.layer_norm_backward(dY, X, mean, rstd, w)
    g, r = dY.double() * w.double(), rstd.double()[:, None]
    want = r * (g - g.mean(1, keepdim=True))
    tol = r * ((C + 10) * g.abs().mean(1, keepdim=True) + 6 * g.abs()) * ref.U32
    assert ((dX.double() - want).abs() <= tol).all() and (dweight == 0).all()
    assert ((dbias.double() - dY.double().sum(0)).abs() <= rows * ref.U32 * dY.double().abs().sum(0)).all()
