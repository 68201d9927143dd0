"""Dense attention in bf16 loses nothing beside its results' rounding: weights and score gradients keep 16 bits in their products.

The tolerance of :mod:`dense_ref` for bf16 is the one for fp32 rows of the same values, and half a step (2^-8) of what the
products with weights and score gradients add up in absolute value, and of the result.  Here the former counts 2^-16: two parts,
each rounded to half a step of what it holds, hold a number to 2^-8 * 2^-8.
"""
import pytest

torch = pytest.importorskip("torch")
import dense_ref as ref  # noqa: E402
from test_gpu_dense import make, near  # noqa: E402

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


def hold(scram, Q, K, V, dO, what="", **kw):
    want, bf16 = ref.attend_all(Q, K, V, dO, **kw)
    wide = dict(kw, bias=None if kw.get("bias") is None else kw["bias"].float())
    _, fp32 = ref.attend_all(*(t.float() for t in (Q, K, V, dO)), **wide)
    got = [scram.dense_attend(Q, K, V, **kw), *scram.dense_attend_backward(Q, K, V, dO, **kw)]
    for name, g, w, t16, t32 in zip(("out", "dQ", "dK", "dV", "dbias"), got, want, bf16, fp32):
        reach = (t16 - t32 - (HALF - ref.U32) * w.abs()).clamp(min=0) / HALF  # what the products add up
        off = t32 - ref.U32 * w.abs() + HALF * HALF * reach
        near(g, w, (1 + HALF) * off + HALF * w.abs(), f"{name} {what}")


CASES = [
    dict(shape=(2, 2, 7, 9, 7, 9, 16), heads=1, causal=True),
    dict(shape=(6, 3, 9, 7, 4, 11, 64), lengths=[44, 0, 17]),
    dict(shape=(2, 1, 16, 16, 16, 16, 128), heads=2),
    dict(shape=(4, 2, 12, 17, 12, 17, 64), heads=4, causal=True),
    dict(shape=(2, 2, 1, 300, 1, 300, 32), causal=True),
    dict(shape=(64, 64, 16, 16, 16, 16, 64), heads=2),
    dict(shape=(128, 128, 15, 17, 15, 17, 64)),
    dict(shape=(64, 64, 13, 18, 13, 18, 128)),
    dict(shape=(4, 4, 1, 1, 30, 31, 64), heads=4, causal=True, first=[929, 0, 463, 64]),
    dict(shape=(2, 2, 40, 40, 40, 40, 64), heads=2, lean=2.0),
    dict(shape=(3, 1, 4, 5, 4, 5, 20), heads=3),
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "x".join(map(str, c["shape"])))
def test_weights_keep_their_bits(scram, c):
    Q, K, V, dO, kw = make(c, "bf16")
    hold(scram, Q, K, V, dO, str(c), **kw)


@pytest.mark.parametrize("d", [16, 64, 128])
def test_opposite_values(scram, d):
    """Pairs of keys of opposite values and nearly equal scores: the output is what their weights differ by."""
    S, n = 2, 32
    gen = torch.Generator(device="cuda").manual_seed(4)
    V = torch.randn(S, 1, n, d, generator=gen, device="cuda").bfloat16()
    V[:, :, 1::2] = -V[:, :, ::2]
    K = torch.zeros(S, 1, n, d, device="cuda", dtype=torch.bfloat16)
    K[..., 0] = torch.tensor([1.0, -1.0], device="cuda").repeat(n // 2)
    Q = torch.zeros(S, 1, 8, d, device="cuda", dtype=torch.bfloat16)
    Q[..., 0] = 2.0 ** -torch.arange(8, device="cuda")  # scores of the two sides that lie 2^-1 .. 2^-8 d^(-1/2) 4 apart
    dO = torch.randn(S, 1, 8, d, generator=gen, device="cuda").bfloat16()
    hold(scram, Q, K, V, dO)
