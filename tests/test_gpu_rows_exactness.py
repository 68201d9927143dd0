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
