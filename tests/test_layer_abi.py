"""Refusals of the operators around the attention: on the host, before any HIP call, so these run without a GPU.

Every call through the C ABI below has at least one argument out of place; none reaches a launch.
"""
import ctypes
import os

import pytest
import torch

OK, ENULL, ESHAPE, EUNSUP, EALIGN, EALIAS, EWS = 0, -1, -2, -3, -4, -5, -7
F32, BF16 = 0, 1
# fake, well-aligned "device" addresses far apart (never read)
A = [0x10000000 * (i + 1) for i in range(14)]
CAUSAL = 4


@pytest.fixture(scope="module")
def L():
    from paper_1905_10308_amd import binding

    if not os.path.exists(binding.LIB_PATH):
        from paper_1905_10308_amd import build

        build.build()
    return binding.lib()


def diff(L, backward=False, **kw):
    a = dict(Q=A[0], K=A[1], V=A[2], dtype=BF16, J=A[3], kappa=2, lam=A[4], S=2, Hq=8, Wq=8, Hk=8, Wk=8, d=16, dv=16, window=3,
             scale=0.25, flags=0, first=0, origin=None, out=A[5], dO=A[6], dQ=A[7], dK=A[8], dV=A[9], dlam=A[10], ws=A[11],
             ws_bytes=1 << 24)
    a.update(kw)
    head = [a[k] for k in ("Q", "K", "V", "dtype", "J", "kappa", "lam", "S", "Hq", "Wq", "Hk", "Wk", "d", "dv", "window", "scale", "flags",
                           "first", "origin")]
    if backward:
        return L.scram_differential_attend_backward(*head, *[a[k] for k in ("dO", "dQ", "dK", "dV", "dlam", "ws", "ws_bytes")], None, None)
    return L.scram_differential_attend(*head, a["out"], None, None)


SHARED = [
    (dict(Q=None), ENULL), (dict(J=None), ENULL), (dict(lam=None), ENULL),
    (dict(S=0), ESHAPE), (dict(Wq=0), ESHAPE), (dict(Hk=-1), ESHAPE), (dict(window=2), ESHAPE), (dict(window=0), ESHAPE),
    (dict(window=32769), ESHAPE), (dict(kappa=0), ESHAPE), (dict(kappa=9), ESHAPE), (dict(scale=float("nan")), ESHAPE),
    (dict(scale=float("inf")), ESHAPE), (dict(S=1 << 16, Hq=1 << 8, Wq=1 << 7), ESHAPE),
    (dict(d=48, dv=48), EUNSUP), (dict(dv=32), EUNSUP), (dict(dtype=2), EUNSUP), (dict(flags=1), EUNSUP), (dict(flags=8), EUNSUP),
    # a place among the keys without the mask, before the first key, past the last, rows of another width
    (dict(first=1), ESHAPE), (dict(origin=A[12]), ESHAPE), (dict(flags=CAUSAL, first=-1), ESHAPE), (dict(flags=CAUSAL, first=1), ESHAPE),
    (dict(flags=CAUSAL, Hq=1, Wq=5, first=60), ESHAPE), (dict(flags=CAUSAL, Hq=2, Wq=5), ESHAPE), (dict(flags=CAUSAL, Hk=4), ESHAPE),
    (dict(flags=CAUSAL, Hq=1, Wq=1, first=3, origin=A[12]), ESHAPE),
    (dict(Q=A[0] + 8), EALIGN), (dict(V=A[2] + 2), EALIGN), (dict(lam=A[4] + 2), EALIGN), (dict(J=A[3] + 1), EALIGN),
    (dict(flags=CAUSAL, Hq=1, Wq=1, origin=A[12] + 2), EALIGN),
]


@pytest.mark.parametrize("kw,code", SHARED + [(dict(out=None), ENULL), (dict(out=A[5] + 8), EALIGN), (dict(out=A[0]), EALIAS),
                                              (dict(out=A[2] + 64), EALIAS), (dict(lam=A[5] + 16), EALIAS),
                                              (dict(flags=CAUSAL, Hq=1, Wq=1, origin=A[5]), EALIAS)])
def test_differential_attend_rejects(L, kw, code):
    assert diff(L, **kw) == code


@pytest.mark.parametrize("kw,code", SHARED + [
    (dict(dO=None), ENULL), (dict(dQ=None), ENULL), (dict(dlam=None), ENULL), (dict(ws=None), EWS), (dict(ws_bytes=64), EWS),
    (dict(dK=A[8] + 4), EALIGN), (dict(ws=A[11] + 16), EALIGN), (dict(dO=A[6] + 8), EALIGN),
    (dict(dQ=A[0]), EALIAS), (dict(dV=A[8]), EALIAS), (dict(dlam=A[7]), EALIAS), (dict(ws=A[9]), EALIAS), (dict(dK=A[6]), EALIAS),
    (dict(dlam=A[4]), EALIAS),
    # 2^31 entries of the inverse map, 2^31 keys in all
    (dict(S=1, Hq=1 << 14, Wq=1 << 14, kappa=8), ESHAPE), (dict(S=1 << 11, Hk=1 << 10, Wk=1 << 10), ESHAPE),
])
def test_differential_attend_backward_rejects(L, kw, code):
    assert diff(L, True, **kw) == code


def test_differential_workspace(L):
    size = L.scram_differential_attend_backward_workspace_bytes
    assert size(2, 8, 8, 8, 8, 16, BF16, 2) > 0
    assert size(4, 256, 256, 256, 256, 64, BF16, 2) > size(4, 256, 256, 256, 256, 64, BF16, 1) >= 4 * 256 * 256 * 32
    for bad in ((0, 8, 8, 8, 8, 16, BF16, 2), (2, 8, 8, 8, 8, 20, BF16, 2), (2, 8, 8, 8, 8, 16, 5, 2), (2, 8, 8, 8, 8, 16, BF16, 9)):
        assert size(*bad) == 0


def rot(L, **kw):
    a = dict(count=2, src=[A[0], A[1]], dst=[A[2], A[3]], slices=[2, 3], dtype=F32, T=2, H=4, W=5, d=16, groups=1, sections=(2, 3, 3),
             freqs=[1.0] * 200, first=(0, 0, 0), origin=None, rows=0, flags=0)
    a.update(kw)
    P, n = ctypes.c_void_p, len(a["src"])
    arr = lambda t, v: None if v is None else (t * len(v))(*v)  # noqa: E731
    return L.scram_rotary(a["count"], arr(P, a["src"]), arr(P, a["dst"]), arr(ctypes.c_int, a["slices"]), a["dtype"], a["T"], a["H"],
                          a["W"], a["d"], a["groups"], arr(ctypes.c_int, a["sections"]), arr(ctypes.c_double, a["freqs"]),
                          arr(ctypes.c_int, a["first"]), a["origin"], a["rows"], a["flags"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(freqs=None), ENULL), (dict(sections=None), ENULL), (dict(first=None), ENULL), (dict(src=[A[0], None]), ENULL),
    (dict(origin=A[4], rows=0), ENULL),
    (dict(count=0), ESHAPE), (dict(count=5), ESHAPE), (dict(T=0), ESHAPE), (dict(H=-3), ESHAPE), (dict(W=(1 << 30) + 1), ESHAPE),
    (dict(T=1 << 12, H=1 << 12, W=1 << 12), ESHAPE), (dict(groups=3), ESHAPE), (dict(groups=0), ESHAPE), (dict(d=1), ESHAPE),
    (dict(sections=(0, 0, 0)), ESHAPE), (dict(sections=(-1, 4, 4)), ESHAPE), (dict(sections=(3, 3, 3)), ESHAPE),
    (dict(d=512, sections=(43, 43, 43)), ESHAPE), (dict(groups=2, sections=(2, 2, 2)), ESHAPE),
    (dict(freqs=[1.0, float("nan")] + [1.0] * 6), ESHAPE), (dict(freqs=[float("inf")] * 8), ESHAPE), (dict(slices=[2, 0]), ESHAPE),
    (dict(origin=A[4], rows=3), ESHAPE),  # the first tensor has two slices
    # 2^33 work items
    (dict(count=1, src=[A[0]], dst=[1 << 50], slices=[1], T=1, H=1 << 15, W=1 << 15, d=64, sections=(8, 12, 12)), ESHAPE),
    (dict(dtype=3), EUNSUP), (dict(flags=4), EUNSUP),
    (dict(src=[A[0] + 2, A[1]]), EALIGN), (dict(dst=[A[2] + 1, A[3]]), EALIGN), (dict(origin=A[4] + 2, rows=1), EALIGN),
    (dict(dst=[A[2], A[2]]), EALIAS), (dict(dst=[A[2], A[0]]), EALIAS), (dict(dst=[A[0] + 64, A[3]]), EALIAS),
    (dict(dst=[A[1], A[0]]), EALIAS), (dict(origin=A[2] + 8, rows=1), EALIAS),
])
def test_rotary_rejects(L, kw, code):
    assert rot(L, **kw) == code


def norm(L, backward=False, **kw):
    a = dict(X=A[0], dtype=BF16, w=A[1], b=A[2], wtype=BF16, rows=100, C=64, eps=1e-5, Y=A[3], mean=A[4], rstd=A[5], dY=A[6], gtype=F32,
             dX=A[7], dw=A[8], db=A[9], ws=A[10], ws_bytes=1 << 24)
    a.update(kw)
    if backward:
        return L.scram_layer_norm_backward(a["dY"], a["gtype"], a["X"], a["dtype"], a["mean"], a["rstd"], a["w"], a["wtype"], a["rows"],
                                           a["C"], a["dX"], a["dw"], a["db"], a["ws"], a["ws_bytes"], None)
    return L.scram_layer_norm(a["X"], a["dtype"], a["w"], a["b"], a["wtype"], a["rows"], a["C"], a["eps"], a["Y"], a["mean"], a["rstd"], None)


NORM = [(dict(X=None), ENULL), (dict(rows=0), ESHAPE), (dict(rows=-1), ESHAPE), (dict(C=0), ESHAPE), (dict(C=16385), ESHAPE),
        (dict(dtype=2), EUNSUP), (dict(wtype=2), EUNSUP), (dict(dtype=F32), EUNSUP), (dict(X=A[0] + 1), EALIGN), (dict(w=A[1] + 1), EALIGN),
        (dict(mean=A[4] + 2), EALIGN)]


@pytest.mark.parametrize("kw,code", NORM + [
    (dict(Y=None), ENULL), (dict(mean=None), ENULL), (dict(eps=-1.0), ESHAPE), (dict(eps=float("nan")), ESHAPE),
    (dict(eps=float("inf")), ESHAPE), (dict(Y=A[0] + 128), EALIAS), (dict(mean=A[0]), EALIAS), (dict(rstd=A[4]), EALIAS), (dict(Y=A[1]), EALIAS)])
def test_layer_norm_rejects(L, kw, code):
    assert norm(L, **kw) == code


@pytest.mark.parametrize("kw,code", NORM + [
    (dict(dY=None), ENULL), (dict(mean=None), ENULL), (dict(dw=None), ENULL), (dict(ws=None), EWS), (dict(ws_bytes=256), EWS),
    (dict(dtype=F32, wtype=F32, gtype=BF16), EUNSUP), (dict(ws=A[10] + 4), EALIGN), (dict(dX=A[0]), EALIAS), (dict(dX=A[6] + 256), EALIAS),
    (dict(db=A[8]), EALIAS), (dict(dw=A[6]), EALIAS), (dict(ws=A[7]), EALIAS)])
def test_layer_norm_backward_rejects(L, kw, code):
    assert norm(L, True, **kw) == code


def test_binding_rejects():
    """The checks of the Python entry points, on tensors of the CPU (none is a device tensor, which is said first)."""
    import paper_1905_10308_amd as scram

    x = torch.zeros(1, 4, 4, 16)
    for call in (lambda: scram.rotary(x), lambda: scram.layer_norm(x), lambda: scram.rotary_backward(x, x),
                 lambda: scram.layer_norm_backward(x, x, x, x),
                 lambda: scram.differential_attend(x, x, x, torch.zeros(1, 4, 4, dtype=torch.int32), torch.ones(1), 3)):
        with pytest.raises(ValueError, match="device"):
            call()
    with pytest.raises(ValueError):
        scram.rotary()


def test_numbers_that_no_c_int_holds():
    """They are refused, not cut to 32 bits."""
    from paper_1905_10308_amd import binding, rows

    assert binding._int32("first", (1 << 31) - 1) == (1 << 31) - 1 and binding._int32("origin", -(1 << 31)) == -(1 << 31)
    for x in (1 << 31, -(1 << 31) - 1, 1 << 32):
        with pytest.raises(ValueError, match="int32"):
            binding._int32("first", x)
    with pytest.raises(ValueError, match="pairs"):
        rows._pairs((1 << 40, 0, 0), None, 10000.0, 8, 3)
    with pytest.raises(ValueError, match="sections"):
        rows._pairs((1, 1, 1, 1), None, 10000.0, 8, 3)
