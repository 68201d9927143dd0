"""Refusals of the dense attention, its bias and group norm: on the host, before any HIP call, so these run without a GPU.

Every call through the C ABI below has at least one argument out of place; none reaches a launch.
"""
import ctypes
import os

import pytest
import torch

OK, ENULL, ESHAPE, EUNSUP, EALIGN, EALIAS, EWS = 0, -1, -2, -3, -4, -5, -7
F32, BF16 = 0, 1
# fake, well-aligned "device" addresses far apart (never read)
A = [0x10000000 * (i + 1) for i in range(16)]
CAUSAL = 4


@pytest.fixture(scope="module")
def L():
    from paper_1905_10308_amd import binding

    if not os.path.exists(binding.LIB_PATH):
        from paper_1905_10308_amd import build

        build.build()
    return binding.lib()


def dense(L, backward=False, **kw):
    a = dict(Q=A[0], K=A[1], V=A[2], dtype=BF16, bias=None, heads=0, lengths=None, S=4, Sk=2, Hq=8, Wq=8, Hk=8, Wk=8, d=16, dv=16,
             scale=0.25, flags=0, first=0, origin=None, out=A[3], dO=A[4], dQ=A[5], dK=A[6], dV=A[7], dB=None, ws=A[8], ws_bytes=1 << 24)
    a.update(kw)
    head = [a[k] for k in ("Q", "K", "V", "dtype", "bias", "heads", "lengths", "S", "Sk", "Hq", "Wq", "Hk", "Wk", "d", "dv", "scale",
                           "flags", "first", "origin")]
    if backward:
        return L.scram_dense_attend_backward(*head, *[a[k] for k in ("dO", "dQ", "dK", "dV", "dB", "ws", "ws_bytes")], None, None)
    return L.scram_dense_attend(*head, a["out"], a["ws"], a["ws_bytes"], None, None)


B = dict(bias=A[9], heads=2)
SHARED = [
    (dict(Q=None), ENULL), (dict(K=None), ENULL), (dict(V=None), ENULL),
    (dict(S=0), ESHAPE), (dict(Sk=0), ESHAPE), (dict(Sk=3), ESHAPE), (dict(Sk=8), ESHAPE), (dict(Wq=0), ESHAPE), (dict(Hk=-1), ESHAPE),
    (dict(scale=float("nan")), ESHAPE), (dict(scale=float("-inf")), ESHAPE), (dict(S=1 << 16, Sk=1, Hq=1 << 8, Wq=1 << 7), ESHAPE),
    (dict(d=48, dv=48), EUNSUP), (dict(dv=32), EUNSUP), (dict(d=256, dv=256), EUNSUP), (dict(dtype=2), EUNSUP), (dict(flags=1), EUNSUP),
    # places without the mask or a bias, before the first key, past the last, rows of another width
    (dict(first=1), ESHAPE), (dict(origin=A[10]), ESHAPE), (dict(flags=CAUSAL, first=-1), ESHAPE), (dict(flags=CAUSAL, first=1), ESHAPE),
    (dict(flags=CAUSAL, Hq=1, Wq=5, first=60), ESHAPE), (dict(flags=CAUSAL, Hq=2, Wq=5), ESHAPE), (dict(B, Hq=2, Wq=5), ESHAPE),
    (dict(B, Hk=4), ESHAPE), (dict(flags=CAUSAL, Hq=1, Wq=1, first=3, origin=A[10]), ESHAPE),
    # a bias whose heads do not divide the slices, planes of 2^31 places, windows that no block holds
    (dict(bias=A[9], heads=0), ESHAPE), (dict(bias=A[9], heads=3), ESHAPE), (dict(B, S=2, Hq=1, Wq=1, Hk=1 << 15, Wk=1 << 14), ESHAPE),
    (dict(B, Hq=1, Wq=1, Hk=2, Wk=7000), ESHAPE),
    # so many rows that a step behind the last is no number
    (dict(S=2, Sk=2, Hq=1, Wq=1, Hk=2, Wk=(1 << 30) - 1), ESHAPE), (dict(S=2, Sk=1, Hq=1, Wq=(1 << 30) - 1), ESHAPE),
    (dict(Q=A[0] + 8), EALIGN), (dict(V=A[2] + 2), EALIGN), (dict(B, bias=A[9] + 1), EALIGN), (dict(lengths=A[10] + 2), EALIGN),
    (dict(flags=CAUSAL, Hq=1, Wq=1, origin=A[10] + 2), EALIGN),
]


@pytest.mark.parametrize("kw,code", SHARED + [
    (dict(out=None), ENULL), (dict(out=A[3] + 8), EALIGN), (dict(out=A[0]), EALIAS), (dict(out=A[2] + 64), EALIAS),
    (dict(B, bias=A[3] + 32), EALIAS), (dict(lengths=A[3]), EALIAS), (dict(flags=CAUSAL, Hq=1, Wq=1, origin=A[3]), EALIAS),
    # few queries of many keys: parts to join
    (dict(Hq=1, Wq=1, Hk=64, Wk=64, ws=None), EWS), (dict(Hq=1, Wq=1, Hk=64, Wk=64, ws_bytes=64), EWS),
    (dict(Hq=1, Wq=1, Hk=64, Wk=64, ws=A[8] + 16), EALIGN), (dict(Hq=1, Wq=1, Hk=64, Wk=64, ws=A[3]), EALIAS),
    (dict(Hq=1, Wq=1, Hk=64, Wk=64, ws=A[1]), EALIAS)])
def test_dense_attend_rejects(L, kw, code):
    assert dense(L, **kw) == code


@pytest.mark.parametrize("kw,code", SHARED + [
    (dict(dO=None), ENULL), (dict(dQ=None), ENULL), (dict(dV=None), ENULL), (dict(dB=A[9]), ENULL), (dict(ws=None), EWS),
    (dict(ws_bytes=64), EWS), (dict(dK=A[6] + 4), EALIGN), (dict(ws=A[8] + 16), EALIGN), (dict(dO=A[4] + 8), EALIGN),
    (dict(B, dB=A[10] + 1), EALIGN), (dict(dQ=A[0]), EALIAS), (dict(dV=A[6]), EALIAS), (dict(ws=A[7]), EALIAS), (dict(dK=A[4]), EALIAS),
    (dict(B, dB=A[9]), EALIAS), (dict(B, dB=A[5]), EALIAS), (dict(B, dB=A[8] + 512), EALIAS)])
def test_dense_attend_backward_rejects(L, kw, code):
    assert dense(L, True, **kw) == code


def test_dense_workspace(L):
    size, back = L.scram_dense_attend_workspace_bytes, L.scram_dense_attend_backward_workspace_bytes
    assert size(32, 32, 1, 1, 64, 64, 64, BF16, 0) > 0 and size(64, 64, 128, 128, 128, 128, 64, BF16, 1) == 0
    assert back(4, 2, 8, 8, 8, 8, 16, BF16, 2) > back(4, 2, 8, 8, 8, 8, 16, BF16, 0) > 0
    for bad in ((0, 1, 8, 8, 8, 8, 16, BF16, 0), (4, 3, 8, 8, 8, 8, 16, BF16, 0), (4, 2, 8, 8, 8, 8, 20, BF16, 0), (4, 2, 8, 8, 8, 8, 16, 5, 0)):
        assert size(*bad) == 0 and back(*bad) == 0
    assert back(4, 2, 8, 8, 8, 8, 16, BF16, 3) == 0


def relative(L, backward=False, **kw):
    a = dict(table=A[0], dtype=F32, heads=4, H=6, W=9, ey=(1, 3), ex=(1, 2, 4), my=None, mx=None, bias=A[1], ws=A[2], ws_bytes=1 << 20)
    a.update(kw)
    arr = lambda v: None if v is None else (ctypes.c_int * max(len(v), 1))(*v)  # noqa: E731
    n = lambda m, v: m if m is not None else len(v)  # noqa: E731
    edges = (arr(a["ey"]), n(a["my"], a["ey"]), arr(a["ex"]), n(a["mx"], a["ex"]))
    if backward:
        return L.scram_relative_bias_backward(a["bias"], a["dtype"], a["heads"], a["H"], a["W"], *edges, a["table"], a["ws"], a["ws_bytes"], None)
    return L.scram_relative_bias(a["table"], a["dtype"], a["heads"], a["H"], a["W"], *edges, a["bias"], None)


RELATIVE = [
    (dict(table=None), ENULL), (dict(bias=None), ENULL), (dict(ey=None, my=2), ENULL), (dict(heads=0), ESHAPE), (dict(H=0), ESHAPE),
    (dict(W=-4), ESHAPE), (dict(W=(1 << 30) + 1), ESHAPE), (dict(H=1 << 15, W=1 << 15), ESHAPE), (dict(heads=1 << 30, H=64, W=64), ESHAPE),
    (dict(ey=(0, 1)), ESHAPE), (dict(ex=(2, 2)), ESHAPE), (dict(ex=(3, 2)), ESHAPE), (dict(ey=(-1,)), ESHAPE), (dict(my=-1), ESHAPE),
    (dict(ey=tuple(range(1, 66))), ESHAPE), (dict(dtype=2), EUNSUP), (dict(table=A[0] + 2), EALIGN), (dict(bias=A[1] + 1), EALIGN),
    (dict(table=A[1] + 64), EALIAS)]


@pytest.mark.parametrize("kw,code", RELATIVE)
def test_relative_bias_rejects(L, kw, code):
    assert relative(L, **kw) == code


@pytest.mark.parametrize("kw,code", RELATIVE + [(dict(ws=None), EWS), (dict(ws_bytes=64), EWS), (dict(ws=A[2] + 4), EALIGN),
                                                (dict(ws=A[1]), EALIAS), (dict(ws=A[0]), EALIAS)])
def test_relative_bias_backward_rejects(L, kw, code):
    assert relative(L, True, **kw) == code


def group(L, backward=False, **kw):
    a = dict(X=A[0], dtype=BF16, w=A[1], b=A[2], wtype=BF16, N=2, P=3000, C=64, G=8, eps=1e-5, act=1, Y=A[3], mean=A[4], rstd=A[5], dY=A[6],
             gtype=F32, dX=A[7], dw=A[8], db=A[9], ws=A[10], ws_bytes=1 << 24)
    a.update(kw)
    size = (a["N"], a["P"], a["C"], a["G"])
    if backward:
        return L.scram_group_norm_backward(a["dY"], a["gtype"], a["X"], a["dtype"], a["mean"], a["rstd"], a["w"], a["b"], a["wtype"], *size,
                                           a["act"], a["dX"], a["dw"], a["db"], a["ws"], a["ws_bytes"], None)
    return L.scram_group_norm(a["X"], a["dtype"], a["w"], a["b"], a["wtype"], *size, a["eps"], a["act"], a["Y"], a["mean"], a["rstd"],
                              a["ws"], a["ws_bytes"], None)


GROUP = [
    (dict(X=None), ENULL), (dict(N=0), ESHAPE), (dict(P=0), ESHAPE), (dict(P=-1), ESHAPE), (dict(C=0), ESHAPE), (dict(C=16392), ESHAPE),
    (dict(G=0), ESHAPE), (dict(G=7), ESHAPE), (dict(N=1 << 20, P=1 << 20), ESHAPE), (dict(N=1 << 28, P=1), ESHAPE), (dict(dtype=2), EUNSUP),
    (dict(wtype=2), EUNSUP), (dict(dtype=F32), EUNSUP), (dict(act=2), EUNSUP), (dict(act=-1), EUNSUP), (dict(X=A[0] + 1), EALIGN),
    (dict(w=A[1] + 1), EALIGN), (dict(mean=A[4] + 2), EALIGN), (dict(ws=None), EWS), (dict(ws_bytes=256), EWS), (dict(ws=A[10] + 4), EALIGN)]


@pytest.mark.parametrize("kw,code", GROUP + [
    (dict(Y=None), ENULL), (dict(mean=None), ENULL), (dict(eps=-1.0), ESHAPE), (dict(eps=float("nan")), ESHAPE), (dict(Y=A[0] + 128), EALIAS),
    (dict(mean=A[0]), EALIAS), (dict(rstd=A[4]), EALIAS), (dict(Y=A[1]), EALIAS), (dict(ws=A[3]), EALIAS)])
def test_group_norm_rejects(L, kw, code):
    assert group(L, **kw) == code


@pytest.mark.parametrize("kw,code", GROUP + [
    (dict(dY=None), ENULL), (dict(mean=None), ENULL), (dict(dw=None), ENULL), (dict(dtype=F32, wtype=F32, gtype=BF16), EUNSUP),
    (dict(dX=A[0]), EALIAS), (dict(dX=A[6] + 256), EALIAS), (dict(db=A[8]), EALIAS), (dict(dw=A[6]), EALIAS), (dict(ws=A[7]), EALIAS),
    (dict(dw=A[2]), EALIAS)])
def test_group_norm_backward_rejects(L, kw, code):
    assert group(L, True, **kw) == code


def test_binding_rejects():
    """The checks of the Python entry points, on tensors of the CPU (none is a device tensor, which is said first)."""
    import paper_1905_10308_amd as scram

    x = torch.zeros(1, 4, 4, 16)
    for call in (lambda: scram.dense_attend(x, x, x), lambda: scram.dense_attend_backward(x, x, x, x), lambda: scram.relative_bias(x[0], 4, 5),
                 lambda: scram.relative_bias_backward(x[0], edges=((), ())), lambda: scram.group_norm(x, 4),
                 lambda: scram.group_norm_backward(x, x, x, x)):
        with pytest.raises(ValueError, match="device"):
            call()


def test_bias_edges():
    from paper_1905_10308_amd import bias_edges

    assert bias_edges(0, 5) == () and bias_edges(1, 0) == (1,) and bias_edges(4, 64) == (1, 2, 11, 64)
    for count in range(65):
        for furthest in (0, 1, 7, 100, 4096):
            e = bias_edges(count, furthest)
            assert len(e) == count and all(b > a for a, b in zip((0,) + e, e))
    with pytest.raises(ValueError):
        bias_edges(65, 100)
