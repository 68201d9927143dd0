"""Attention over every key with a learned bias by relative position, that bias by buckets of distance, and their gradients.

Argument marshalling only, as in :mod:`.binding`.  The kernels take d in {16, 32, 64, 128} with dv == d; other widths up to
128 are zero-padded here and results are cut back.
"""
from __future__ import annotations

import ctypes
import functools

from . import binding as _b

BIAS_MAX_EDGES = 64


def _rows(Q, K, V, bias, causal, first, lengths, dO=None):
    """Checks of the arguments that the call and its gradients share: (grid, key slices, d, dv, bias rows, first, origin)."""
    torch = _b._torch()
    kind, index = Q.dtype, Q.get_device()
    _b._plain("Q", Q, 4, kind, index)
    S, Hq, Wq, d = Q.shape
    Sk, Hk, Wk, dv = _b._plain("V", V, 4, kind, index).shape
    if _b._plain("K", K, 4, kind, index).shape != (Sk, Hk, Wk, d):
        raise ValueError("K and V must share their slices and the key grid; K must match Q's channels")
    if Sk < 1 or S % Sk:
        raise ValueError(f"{S} slices of queries do not share {Sk} slices of keys evenly")
    heads = 0
    if bias is not None:
        heads = _b._plain("bias", bias, 3, kind, index).shape[0]
        if bias.shape[1:] != (2 * Hk - 1, 2 * Wk - 1) or heads < 1 or S % heads:
            raise ValueError(f"bias must be [heads, {2 * Hk - 1}, {2 * Wk - 1}] with a number of heads that divides {S}, got "
                             f"{tuple(bias.shape)}")
    if lengths is not None and _b._plain("lengths", lengths, 1, torch.int32, index).shape[0] != Sk:
        raise ValueError(f"lengths must have a count for each of {Sk} slices of keys")
    if dO is not None and _b._plain("dO", dO, 4, kind, index).shape != (S, Hq, Wq, dv):
        raise ValueError("dO must be [S, Hq, Wq, dv]")
    origin = None
    if isinstance(first, torch.Tensor):
        first, origin = 0, _b._plain("first", first, 1, torch.int32, index)
        if origin.shape[0] != S:
            raise ValueError(f"first must be a place for each of {S} slices")
    first = _b._int32("first", first)
    if not causal and bias is None and (first or origin is not None):
        raise ValueError("first is the queries' place among the keys: it needs causal=True or a bias")
    return (Hq, Wq, Hk, Wk), S, Sk, d, dv, heads, first, origin


def dense_attend(Q, K, V, scale: float | None = None, *, bias=None, causal: bool = False, first=0, lengths=None, out=None,
                 workspace=None, events=None):
    """Softmax over every key and the values' sum (``scram_dense_attend``).

    Q ``[S, Hq, Wq, d]``, K ``[Sk, Hk, Wk, d]``, V ``[Sk, Hk, Wk, dv]`` with Sk a divisor of S: slice s reads slice
    ``s // (S // Sk)`` of the keys.  Returns ``[S, Hq, Wq, dv]`` in Q's dtype.  ``scale`` defaults to 1/sqrt(d).

    ``bias``: ``[heads, 2 Hk - 1, 2 Wk - 1]`` in Q's dtype, heads a divisor of S (slice s has head ``s % heads``), added to the
    score of a key dy rows below and dx columns right of its query at ``[dy + Hk - 1, dx + Wk - 1]``; :func:`relative_bias`
    makes one of a table by buckets.  ``causal`` keeps keys at or before the query in raster order.  With either the queries
    stand on the key grid, and may be a part of it -- whole rows, or one row of any length, down to a single new pixel:
    ``first`` is the raster index of a slice's first query, a number or an int32 ``[S]`` tensor.
    ``lengths``: int32 ``[Sk]``, the keys of each slice that count, in raster order; a query that sees none gets zeros.
    ``workspace``: optional uint8 device tensor of at least ``dense_attend_workspace_bytes(...)`` bytes.
    ``events``: optional 2 timing-enabled torch.cuda.Event objects stamped with the start and end.
    """
    torch = _b._torch()
    (Hq, Wq, Hk, Wk), S, Sk, d, dv, heads, first, origin = _rows(Q, K, V, bias, causal, first, lengths)
    dev = Q.device
    if out is not None and _b._plain("out", out, 4, Q.dtype, Q.get_device()).shape != (S, Hq, Wq, dv):
        raise ValueError(f"out must be {(S, Hq, Wq, dv)}, got {tuple(out.shape)}")
    code = _b._dtype_code(Q)
    if scale is None:
        scale = d ** -0.5
    w = _b._native_width(max(d, dv))
    if w != d or w != dv:
        Q, K, V = _b._pad_channels(w, Q, K, V)
    res = out if out is not None and w == dv else torch.empty((S, Hq, Wq, w), dtype=Q.dtype, device=dev)
    size = 0
    if workspace is not None:
        size = _b._workspace(workspace, 0, dev).numel() * workspace.element_size()
    else:
        size = int(_b.lib().scram_dense_attend_workspace_bytes(S, Sk, Hq, Wq, Hk, Wk, w, code, int(heads > 0)))
        if size:
            workspace = torch.empty(size, dtype=torch.uint8, device=dev)
    ev = None if events is None else _b._event_array(events, 2)
    _b._call(_b.lib().scram_dense_attend, "scram_dense_attend", dev,
             (Q.data_ptr(), K.data_ptr(), V.data_ptr(), code, _b._ptr(bias), heads, _b._ptr(lengths), S, Sk, Hq, Wq, Hk, Wk, w, w,
              float(scale), _b.CAUSAL if causal else 0, first, _b._ptr(origin), res.data_ptr(), _b._ptr(workspace), size, ev))
    return res if w == dv else _b._unpad_into(res, dv, out)


def dense_attend_backward(Q, K, V, dO, scale: float | None = None, *, bias=None, causal: bool = False, first=0, lengths=None,
                          workspace=None, events=None):
    """Gradients of :func:`dense_attend` (``scram_dense_attend_backward``).

    Returns ``(dQ, dK, dV)`` of the shapes of Q, K and V, with a ``bias`` ``(dQ, dK, dV, dbias)``, in Q's dtype.  The forward
    pass's output is not needed.
    ``workspace``: optional uint8 device tensor of at least ``dense_attend_backward_workspace_bytes(...)`` bytes.
    ``events``: optional 2 timing-enabled events (start and end of the whole call).
    """
    torch = _b._torch()
    (Hq, Wq, Hk, Wk), S, Sk, d, dv, heads, first, origin = _rows(Q, K, V, bias, causal, first, lengths, dO)
    dev = Q.device
    code = _b._dtype_code(Q)
    if scale is None:
        scale = d ** -0.5
    w = _b._native_width(max(d, dv))
    if w != d or w != dv:
        Q, K, V, dO = _b._pad_channels(w, Q, K, V, dO)
    dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
    dbias = None if bias is None else torch.empty_like(bias)
    if workspace is None:
        size = int(_b.lib().scram_dense_attend_backward_workspace_bytes(S, Sk, Hq, Wq, Hk, Wk, w, code, heads))
        workspace = torch.empty(max(size, 1), dtype=torch.uint8, device=dev)
    else:
        _b._workspace(workspace, 0, dev)
    ev = None if events is None else _b._event_array(events, 2)
    _b._call(_b.lib().scram_dense_attend_backward, "scram_dense_attend_backward", dev,
             (Q.data_ptr(), K.data_ptr(), V.data_ptr(), code, _b._ptr(bias), heads, _b._ptr(lengths), S, Sk, Hq, Wq, Hk, Wk, w, w,
              float(scale), _b.CAUSAL if causal else 0, first, _b._ptr(origin), dO.data_ptr(), dQ.data_ptr(), dK.data_ptr(),
              dV.data_ptr(), _b._ptr(dbias), workspace.data_ptr(), workspace.numel() * workspace.element_size(), ev))
    if w != d or w != dv:
        dQ, dK, dV = _b._unpad(w, (dQ, d), (dK, d), (dV, dv))
    return (dQ, dK, dV) if bias is None else (dQ, dK, dV, dbias)


def dense_attend_workspace_bytes(S: int, Sk: int, Hq: int, Wq: int, Hk: int, Wk: int, *, d: int, dtype, bias: bool = False) -> int:
    """Bytes of device workspace ``dense_attend`` needs (``d``: the width of the kernels that holds the call's rows)."""
    return int(_b.lib().scram_dense_attend_workspace_bytes(S, Sk, Hq, Wq, Hk, Wk, d, _b._dtype_code_of(dtype), int(bias)))


def dense_attend_backward_workspace_bytes(S: int, Sk: int, Hq: int, Wq: int, Hk: int, Wk: int, *, d: int, dtype,
                                          heads: int = 0) -> int:
    """Bytes of device workspace ``dense_attend_backward`` needs (``heads`` of the bias, 0: none)."""
    return int(_b.lib().scram_dense_attend_backward_workspace_bytes(S, Sk, Hq, Wq, Hk, Wk, d, _b._dtype_code_of(dtype), heads))


def bias_edges(count: int, furthest: int):
    """``count`` distances at which the buckets of one side of an axis begin: the nearer half 1, 2, 3, .., the others in about
    equal ratios up to ``furthest``."""
    if not 0 <= count <= BIAS_MAX_EDGES:
        raise ValueError(f"0 to {BIAS_MAX_EDGES} edges, got {count}")
    near = (count + 1) // 2
    edges = list(range(1, near + 1))
    for j in range(1, count - near + 1):
        edges.append(max(int(near * max(1.0, furthest / near) ** (j / (count - near))), edges[-1] + 1))
    return tuple(edges)


@functools.lru_cache(maxsize=256)
def _axes(y, x):
    """The host arrays of two axes' edges, as the library's calls take them: (edges, count, edges, count)."""
    got = []
    for axis in (y, x):
        axis = tuple(_b._int32("edge", e) for e in axis)
        if len(axis) > BIAS_MAX_EDGES:
            raise ValueError(f"at most {BIAS_MAX_EDGES} edges an axis, got {len(axis)}")
        if any(b <= a for a, b in zip((0,) + axis, axis)):
            raise ValueError(f"edges must rise from 1 on, got {axis}")
        got += [(ctypes.c_int * max(len(axis), 1))(*axis), len(axis)]
    return tuple(got)


def relative_bias(table, H: int, W: int, *, edges=None, out=None):
    """The bias of every offset on an H x W grid from a table by buckets of distance (``scram_relative_bias``).

    ``table`` ``[heads, 2 my + 1, 2 mx + 1]``; ``edges``: the rising distances, from 1 on, at which the buckets of a side of the
    height (my of them) and of the width (mx) begin; an offset of t has bucket ``m + sign(t) * (edges up to |t|)``.  Default:
    ``bias_edges(my, H - 1), bias_edges(mx, W - 1)``.  Returns ``[heads, 2 H - 1, 2 W - 1]`` in the table's dtype, for
    :func:`dense_attend`.
    """
    _b._plain("table", table, 3, table.dtype, table.get_device())
    code, (heads, ny, nx) = _b._dtype_code(table), table.shape
    if ny % 2 == 0 or nx % 2 == 0:
        raise ValueError(f"table must be [heads, 2 my + 1, 2 mx + 1], got {tuple(table.shape)}")
    H, W = _b._int32("H", H), _b._int32("W", W)
    if H < 1 or W < 1:
        raise ValueError(f"a grid of {H} x {W}")
    y, x = edges if edges is not None else (bias_edges(ny // 2, H - 1), bias_edges(nx // 2, W - 1))
    axes = _axes(tuple(y), tuple(x))
    if (2 * axes[1] + 1, 2 * axes[3] + 1) != (ny, nx):
        raise ValueError(f"{axes[1]} and {axes[3]} edges need a table of {2 * axes[1] + 1} x {2 * axes[3] + 1} a head, got {ny} x {nx}")
    shape = (heads, 2 * H - 1, 2 * W - 1)
    if out is None:
        out = table.new_empty(shape)
    elif _b._plain("out", out, 3, table.dtype, table.get_device()).shape != shape:
        raise ValueError(f"out must be {shape}, got {tuple(out.shape)}")
    _b._call(_b.lib().scram_relative_bias, "scram_relative_bias", table.device,
             (table.data_ptr(), code, heads, H, W, *axes, out.data_ptr()))
    return out


def relative_bias_backward(dbias, *, edges, workspace=None):
    """Gradient of :func:`relative_bias`'s table (``scram_relative_bias_backward``): ``[heads, 2 my + 1, 2 mx + 1]`` in dbias'
    dtype, from ``dbias`` ``[heads, 2 H - 1, 2 W - 1]``.  ``edges``: those of the call (:func:`bias_edges` gives the defaults).
    ``workspace``: optional uint8 device tensor of at least ``relative_bias_backward_workspace_bytes(...)`` bytes.
    """
    torch = _b._torch()
    _b._plain("dbias", dbias, 3, dbias.dtype, dbias.get_device())
    code, (heads, hh, ww), dev = _b._dtype_code(dbias), dbias.shape, dbias.device
    if hh % 2 == 0 or ww % 2 == 0:
        raise ValueError(f"dbias must be [heads, 2 H - 1, 2 W - 1], got {tuple(dbias.shape)}")
    axes = _axes(*map(tuple, edges))
    H, W = (hh + 1) // 2, (ww + 1) // 2
    dtable = dbias.new_empty((heads, 2 * axes[1] + 1, 2 * axes[3] + 1))
    if workspace is None:
        workspace = torch.empty(max(relative_bias_backward_workspace_bytes(heads, H, W, axes[3]), 1), dtype=torch.uint8, device=dev)
    else:
        _b._workspace(workspace, 0, dev)
    _b._call(_b.lib().scram_relative_bias_backward, "scram_relative_bias_backward", dev,
             (dbias.data_ptr(), code, heads, H, W, *axes, dtable.data_ptr(), workspace.data_ptr(),
              workspace.numel() * workspace.element_size()))
    return dtable


@functools.lru_cache(maxsize=256)
def relative_bias_backward_workspace_bytes(heads: int, H: int, W: int, mx: int) -> int:
    """Bytes of device workspace ``relative_bias_backward`` needs (``mx``: edges of the width)."""
    return int(_b.lib().scram_relative_bias_backward_workspace_bytes(heads, H, W, mx))
