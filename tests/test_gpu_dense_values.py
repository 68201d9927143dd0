"""Dense attention with values at the ends of their types."""
import math

import pytest

torch = pytest.importorskip("torch")
import dense_ref as ref  # noqa: E402
from test_gpu_dense import make, near  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [0, 2])
@pytest.mark.parametrize("shape", [(2, 2, 7, 9, 7, 9, 64), (2, 1, 1, 2, 20, 20, 16)])
def test_a_scale_of_zero(scram, shape, heads, dtype):
    """Every key counts as much, however far the products that it takes out lie apart (here by 2^120 and more)."""
    Q, K, V, dO, kw = make(dict(shape=shape, heads=heads, causal=True, first=0), dtype)
    Q, K = (Q.float() * 2.0 ** 60).to(Q.dtype), (K.float() * 2.0 ** 60).to(K.dtype)
    want, tol = ref.attend_all(Q, K, V, dO, 0.0, **kw)
    got = [scram.dense_attend(Q, K, V, 0.0, **kw), *scram.dense_attend_backward(Q, K, V, dO, 0.0, **kw)]
    for name, g, w, t in zip(("out", "dQ", "dK", "dV", "dbias"), got, want, tol):
        near(g, w, t, name)
    assert not got[1].any() and not got[2].any()
    Q[1, 0, 0, 3] = math.nan
    out = scram.dense_attend(Q, K, V, 0.0, **kw)
    assert out[1, 0, 0].isnan().all() and torch.equal(out[0], got[0][0])
