"""Group norm's statistics where values are not finite."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 6, 6, 16), (3, 200, 170, 40)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_statistics_of_values_that_are_not_finite(scram, value, shape, dtype):
    """A group with one has no variance: its rstd is not a number, as its results; the other groups' are as without."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(*shape, generator=gen, device="cuda").to(TYPES[dtype])
    clean = scram.group_norm(x, 4, stats=True)
    x[1, 2, 3, 5] = value
    hit = torch.zeros(shape[0], 4, dtype=torch.bool, device="cuda")
    hit[1, 5 // (shape[-1] // 4)] = True
    y, mean, rstd = scram.group_norm(x, 4, stats=True)
    assert rstd[hit].isnan().all() and not mean[hit].isfinite().any()
    assert torch.equal(mean[~hit], clean[1][~hit]) and torch.equal(rstd[~hit], clean[2][~hit])
    wide = hit.repeat_interleave(shape[-1] // 4, 1)[:, None, None, :].expand(shape)
    assert y[wide].isnan().all() and torch.equal(y[~wide], clean[0][~wide])
