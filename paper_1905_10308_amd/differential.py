"""Differential attention over the match windows: the difference of two softmax maps, and its gradients.

Argument marshalling only, as in :mod:`.binding`.  A row of Q and K holds the channels of two maps, the first
half and the last.  The kernels take d in {16, 32, 64, 128} with dv == d; other even widths up to 128 are
zero-padded here, each half by itself, and results are cut back.
"""
from __future__ import annotations

from . import binding as _b


def _rows(Q, K, V, argmax, lam, first, causal, dO=None):
    """Checks of the arguments that the call and its gradients share: (grid, d, dv, kappa, first, origin)."""
    torch = _b._torch()
    kind, index = Q.dtype, Q.get_device()
    _b._plain("Q", Q, 4, kind, index)
    S, Hq, Wq, d = Q.shape
    _, Hk, Wk, dv = _b._plain("V", V, 4, kind, index).shape
    if _b._plain("K", K, 4, kind, index).shape != (S, Hk, Wk, d) or V.shape[0] != S:
        raise ValueError("K and V must share the key grid; K must match Q's slices and channels")
    if d < 2 or d % 2:
        raise ValueError(f"the channels of Q and K are two maps' halves: {d} is not even")
    maps = argmax.dim()
    _b._plain("argmax", argmax, maps, torch.int32, index)
    if argmax.shape[-3:] != (S, Hq, Wq) or maps not in (3, 4):
        raise ValueError("argmax must be int32 [S, Hq, Wq] or [kappa, S, Hq, Wq]")
    if _b._plain("lam", lam, 1, torch.float32, index).shape[0] != S:
        raise ValueError(f"lam must have {S} weights, one per slice")
    if dO is not None and _b._plain("dO", dO, 4, kind, index).shape != (S, Hq, Wq, dv):
        raise ValueError("dO must be [S, Hq, Wq, dv]")
    origin = None
    if isinstance(first, torch.Tensor):
        first, origin = 0, _b._plain("first", first, 1, torch.int32, index)
        if origin.shape[0] != S:
            raise ValueError(f"first must be a place for each of {S} slices")
    first = _b._int32("first", first)
    if not causal and (first or origin is not None):
        raise ValueError("first is the queries' place under the causal mask: it needs causal=True")
    return (S, Hq, Wq, Hk, Wk), d, dv, argmax.shape[0] if maps == 4 else 1, int(first), origin


def _width(d: int, dv: int) -> int:
    """The channel count of the kernels that holds rows of two halves of d / 2 and values of dv."""
    w = _b._native_width(max(d, dv))
    return w if w == d else max(w, 32)  # (padded halves are 16 wide at least)


def _halves(width: int, *tensors):
    """The tensors [..., d] with each half of their rows zero-padded to width / 2."""
    if tensors[0].shape[-1] == width or width not in _b.NATIVE_WIDTHS:
        return tensors
    two = [t.view(*t.shape[:-1], 2, t.shape[-1] // 2) for t in tensors]
    return tuple(p.view(*t.shape[:-1], width) for t, p in zip(tensors, _b._pad_channels(width // 2, *two)))


def differential_attend(Q, K, V, argmax, lam, window: int, scale: float | None = None, *, causal: bool = False, first=0,
                        out=None, events=None):
    """Window softmaxes of two maps and their difference's value sum around ``argmax`` (``scram_differential_attend``).

    Q ``[S, Hq, Wq, d]``, K ``[S, Hk, Wk, d]``: rows of two maps, d / 2 channels each; V ``[S, Hk, Wk, dv]``; ``argmax``
    int32 ``[S, Hq, Wq]`` or ``[kappa, S, Hq, Wq]`` (union of the kappa windows, the key set of both maps); ``lam`` fp32
    ``[S]``.  Returns ``sum_j (p1_j - lam p2_j) v_j``, ``[S, Hq, Wq, dv]`` in Q's dtype.  ``scale`` defaults to
    1/sqrt(d / 2).

    ``causal`` keeps keys at or before the query in raster order.  The queries then may be a part of the key grid -- whole
    rows, or one row of any length, down to a single new pixel: ``first`` is the raster index of a slice's first query, a
    number or an int32 ``[S]`` tensor (a position for each slice, read on the device).
    ``events``: optional 2 timing-enabled torch.cuda.Event objects stamped with the kernel's start and end.
    """
    torch = _b._torch()
    grid, d, dv, kappa, first, origin = _rows(Q, K, V, argmax, lam, first, causal)
    dev = Q.device
    S, Hq, Wq, _, _ = grid
    if out is not None and _b._plain("out", out, 4, Q.dtype, Q.get_device()).shape != (S, Hq, Wq, dv):
        raise ValueError(f"out must be {(S, Hq, Wq, dv)}, got {tuple(out.shape)}")
    code = _b._dtype_code(Q)
    if scale is None:
        scale = (d // 2) ** -0.5
    w = _width(d, dv)
    if w != d or w != dv:
        Q, K = _halves(w, Q, K)
        V, = _b._pad_channels(w, V)
    res = out if out is not None and w == dv else torch.empty((S, Hq, Wq, w), dtype=Q.dtype, device=dev)
    ev = None if events is None else _b._event_array(events, 2)
    _b._call(_b.lib().scram_differential_attend, "scram_differential_attend", dev,
             (Q.data_ptr(), K.data_ptr(), V.data_ptr(), code, argmax.data_ptr(), kappa, lam.data_ptr(), *grid, w, w, int(window),
              float(scale), _b.CAUSAL if causal else 0, first, _b._ptr(origin), res.data_ptr(), ev))
    return res if w == dv else _b._unpad_into(res, dv, out)


def differential_attend_backward(Q, K, V, argmax, lam, dO, window: int, scale: float | None = None, *, causal: bool = False,
                                 first=0, workspace=None, events=None):
    """Gradients of :func:`differential_attend` with the maps held fixed (``scram_differential_attend_backward``).

    Returns fp32 ``(dQ [S,Hq,Wq,d], dK [S,Hk,Wk,d], dV [S,Hk,Wk,dv], dlam [S])``.
    ``workspace``: optional uint8 device tensor of at least ``differential_attend_backward_workspace_bytes(...)`` bytes.
    ``events``: optional 2 timing-enabled events (start and end of the whole call).
    """
    torch = _b._torch()
    grid, d, dv, kappa, first, origin = _rows(Q, K, V, argmax, lam, first, causal, dO)
    dev = Q.device
    _b._same_device(dev, workspace=workspace)
    code = _b._dtype_code(Q)
    if scale is None:
        scale = (d // 2) ** -0.5
    w = _width(d, dv)
    S, Hq, Wq, Hk, Wk = grid
    dQ = torch.empty((S, Hq, Wq, w), dtype=torch.float32, device=dev)
    dK = torch.empty((S, Hk, Wk, w), dtype=torch.float32, device=dev)
    dV = torch.empty((S, Hk, Wk, w), dtype=torch.float32, device=dev)
    dlam = torch.empty((S,), dtype=torch.float32, device=dev)
    kind = Q.dtype
    if w != d or w != dv:
        Q, K = _halves(w, Q, K)
        V, dO = _b._pad_channels(w, V, dO)
    workspace = _b._workspace(workspace, differential_attend_backward_workspace_bytes(*grid, kappa, d=w, dtype=kind), dev)
    ev = None if events is None else _b._event_array(events, 2)
    _b._call(_b.lib().scram_differential_attend_backward, "scram_differential_attend_backward", dev,
             (Q.data_ptr(), K.data_ptr(), V.data_ptr(), code, argmax.data_ptr(), kappa, lam.data_ptr(), *grid, w, w, int(window),
              float(scale), _b.CAUSAL if causal else 0, first, _b._ptr(origin), dO.data_ptr(), dQ.data_ptr(), dK.data_ptr(),
              dV.data_ptr(), dlam.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(), ev))
    if w != d:
        two = [t.view(*t.shape[:-1], 2, w // 2) for t in (dQ, dK)]
        dQ, dK = (t.view(*t.shape[:-2], d) for t in _b._unpad(w // 2, *((t, d // 2) for t in two)))
    dV, = _b._unpad(w, (dV, dv))
    return dQ, dK, dV, dlam


def differential_attend_backward_workspace_bytes(S: int, Hq: int, Wq: int, Hk: int, Wk: int, kappa: int = 1, *, d: int,
                                                 dtype) -> int:
    """Bytes of device workspace ``differential_attend_backward`` needs (``d``: the width of the kernels that holds the
    call's rows; ``dtype``: torch dtype of Q, K, V)."""
    return int(_b.lib().scram_differential_attend_backward_workspace_bytes(S, Hq, Wq, Hk, Wk, d, _b._dtype_code_of(dtype),
                                                                          kappa))
