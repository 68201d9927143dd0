"""Operators on channel rows around the attention: rotary grid positions, layer norm and group norm, with their gradients.

Argument marshalling only, as in :mod:`.binding`; rows of any width, no padding.
"""
from __future__ import annotations

import ctypes
import functools

from . import binding as _b

ROTARY_INTERLEAVED = 1
ROTARY_INVERSE = 2
MAX_PAIRS = 128


@functools.lru_cache(maxsize=256)
def _pairs(sections, freqs, base, pairs, axes):
    """The host arrays of a rotation's channel pairs: (sections, freqs).  ``sections`` None: all ``pairs``, shared among the
    grid's ``axes``; ``freqs`` None: base ** (-j / m) for pair j of an axis with m."""
    if sections is None:
        nh = pairs // axes
        nw = pairs - nh if axes == 2 else nh
        sections = (pairs - nh - nw, nh, nw)
    if len(sections) == 2:
        sections = (0,) + sections
    if len(sections) != 3 or min(sections) < 0:
        raise ValueError(f"sections must be the pairs of (time,) height and width, got {sections}")
    if sum(sections) > MAX_PAIRS:
        raise ValueError(f"at most {MAX_PAIRS} pairs are turned, got {sections}")
    if freqs is None:
        if not base > 0:
            raise ValueError("base must be positive")
        freqs = tuple(base ** (-j / m) for m in sections for j in range(m))
    if len(freqs) != sum(sections):
        raise ValueError(f"{sum(sections)} pairs need as many freqs, got {len(freqs)}")
    return (ctypes.c_int * 3)(*sections), (ctypes.c_double * max(len(freqs), 1))(*freqs)


_POINTERS = [ctypes.c_void_p * n for n in range(5)]
_INTS = [ctypes.c_int * n for n in range(5)]


def _rotate(tensors, sections, base, freqs, origin, groups, interleaved, out, inverse):
    torch = _b._torch()
    n = len(tensors)
    if not 1 <= n <= 4:
        raise ValueError(f"one to four tensors, got {n}")
    x = tensors[0]
    kind, index, ndim, grid = x.dtype, x.get_device(), x.dim(), x.shape[1:]
    for i, t in enumerate(tensors):
        _b._plain(f"tensor {i}", t, ndim, kind, index)
        if ndim not in (4, 5) or t.shape[1:] != grid:
            raise ValueError("tensors must be [S, H, W, d] or [S, T, H, W, d] of one grid and width, got "
                             f"{tuple(t.shape)} and {tuple(x.shape)}")
    code = _b._dtype_code(x)
    T, H, W, d = grid if ndim == 5 else (1, *grid)
    groups = int(groups)
    if groups < 1 or d % groups:
        raise ValueError(f"{d} channels do not split into {groups} groups")
    parts, turns = _pairs(None if sections is None else tuple(map(int, sections)), None if freqs is None else tuple(map(float, freqs)),
                          float(base), d // groups // 2, ndim - 2)
    rows, at = 0, None
    if isinstance(origin, torch.Tensor):
        _b._plain("origin", origin, origin.dim(), torch.int32, index)
        if origin.dim() not in (1, 2) or origin.shape[-1] != 3:
            raise ValueError("origin must be int32 [3], [1, 3] or [S, 3]: time, height, width")
        rows = origin.numel() // 3
    else:
        at = tuple(_b._int32("origin", a) for a in origin)
        if len(at) > 3:
            raise ValueError(f"origin is time, height, width, got {at}")
        at = _INTS[3](*((0,) * (3 - len(at)) + at))
        origin = None
    if out is None:
        out = [torch.empty_like(t) for t in tensors]
    else:
        out = [out] if isinstance(out, torch.Tensor) else list(out)
        if len(out) != n:
            raise ValueError(f"{n} tensors need as many outputs, got {len(out)}")
        for i, (o, t) in enumerate(zip(out, tensors)):
            if _b._plain(f"out {i}", o, ndim, kind, index).shape != t.shape:
                raise ValueError(f"out {i} must be {tuple(t.shape)}, got {tuple(o.shape)}")
    _b._call(_b.lib().scram_rotary, "scram_rotary", x.device,
             (n, _POINTERS[n](*[t.data_ptr() for t in tensors]), _POINTERS[n](*[t.data_ptr() for t in out]),
              _INTS[n](*[t.shape[0] for t in tensors]), code, T, H, W, d, groups, parts, turns, at, _b._ptr(origin), rows,
              (ROTARY_INTERLEAVED if interleaved else 0) | (ROTARY_INVERSE if inverse else 0)))
    return tuple(out) if n > 1 else out[0]


def rotary(*tensors, sections=None, base: float = 10000.0, freqs=None, origin=(0, 0, 0), groups: int = 1,
           interleaved: bool = False, out=None):
    """Rotary positions with the axes time, height and width (``scram_rotary``).

    ``tensors``: one to four of ``[S, H, W, d]`` or ``[S, T, H, W, d]`` (slices may differ), turned in one launch.  Each row
    is ``groups`` groups of channels turned alike (2 for the rows of :func:`differential_attend`).  ``sections``: channel
    pairs of a group that turn with (time,) height and width; the channels after them are left as they are.  Default: all
    pairs, shared among the grid's axes.  Pair j of an axis with m pairs turns by ``base ** (-j / m)`` radians a step, or
    ``freqs`` gives the radians of every pair.  A pair is channels (k, k + all pairs) of a group, ``interleaved``:
    (2k, 2k + 1).
    ``origin``: the position (time, height, width) of the grid's first pixel -- numbers, or an int32 device tensor ``[3]``
    or ``[S, 3]`` (a position for each slice, as single new pixels have).
    ``out``: tensors like ``tensors`` to write (the same ones: in place).  Returns a tensor, or a tuple of several.
    """
    return _rotate(tensors, sections, base, freqs, origin, groups, interleaved, out, False)


def rotary_backward(*grads, sections=None, base: float = 10000.0, freqs=None, origin=(0, 0, 0), groups: int = 1,
                    interleaved: bool = False, out=None):
    """Gradients of :func:`rotary`'s tensors from those of its results: the rotation back, in the gradients' dtype."""
    return _rotate(grads, sections, base, freqs, origin, groups, interleaved, out, True)


def _norm_rows(X, weight, bias, out):
    """Checks of a norm's tensors: (rows, channels, dtype code, weights' dtype code, device index)."""
    torch = _b._torch()
    index, kind, shape = X.get_device(), X.dtype, X.shape
    _b._plain("X", X, X.dim(), kind, index)
    if not shape:
        raise ValueError("X must have channels")
    C = shape[-1]
    code = wcode = _b._dtype_code_of(kind)
    if weight is not None or bias is not None:
        wkind = bias.dtype if weight is None else weight.dtype
        if wkind != kind and wkind != torch.float32:
            raise TypeError("weight and bias must be float32 or of X's dtype")
        wcode = _b._dtype_code_of(wkind)
        for name, t in (("weight", weight), ("bias", bias)):
            if t is not None and _b._plain(name, t, 1, wkind, index).shape[0] != C:
                raise ValueError(f"{name} must have {C} channels, got {t.shape[0]}")
    if out is not None and out.shape != shape:
        raise ValueError(f"out must be {tuple(shape)}, got {tuple(out.shape)}")
    return X.numel() // C if C else 0, C, code, wcode, index


def layer_norm(X, weight=None, bias=None, eps: float = 1e-5, *, out=None, stats: bool = False):
    """Layer norm of the rows (last dimension) of ``X`` (``scram_layer_norm``).

    ``weight``, ``bias``: [channels] in X's dtype or float32, or None.  Returns the normalised rows in X's dtype, with
    ``stats`` ``(rows, mean, rstd)``: fp32 of ``X.shape[:-1]``, for :func:`layer_norm_backward`.  ``out`` may be ``X``.
    """
    torch = _b._torch()
    rows, C, code, wcode, index = _norm_rows(X, weight, bias, out)
    if out is None:
        out = torch.empty_like(X)
    else:
        _b._plain("out", out, X.dim(), X.dtype, index)
    mean = rstd = None
    if stats:
        mean = torch.empty(X.shape[:-1], dtype=torch.float32, device=X.device)
        rstd = torch.empty_like(mean)
    _b._call(_b.lib().scram_layer_norm, "scram_layer_norm", X.device,
             (X.data_ptr(), code, _b._ptr(weight), _b._ptr(bias), wcode, rows, C, float(eps), out.data_ptr(), _b._ptr(mean),
              _b._ptr(rstd)))
    return (out, mean, rstd) if stats else out


def layer_norm_backward(dY, X, mean, rstd, weight=None, *, out=None, workspace=None):
    """Gradients of :func:`layer_norm` (``scram_layer_norm_backward``): ``(dX, dweight, dbias)``.

    ``dY`` is in X's dtype or float32 and dX in dY's (``out`` may be ``dY``); dweight and dbias are fp32 [channels], also
    where the call had no weights.  ``mean``, ``rstd``: what the call gave with ``stats``.
    ``workspace``: optional uint8 device tensor of at least ``layer_norm_backward_workspace_bytes(rows, channels)`` bytes.
    """
    torch = _b._torch()
    rows, C, code, wcode, index = _norm_rows(X, weight, None, out)
    kind, gkind, dev = X.dtype, dY.dtype, X.device
    if gkind != kind and gkind != torch.float32:
        raise TypeError("dY must be float32 or of X's dtype")
    if _b._plain("dY", dY, X.dim(), gkind, index).shape != X.shape:
        raise ValueError(f"dY must be {tuple(X.shape)}, got {tuple(dY.shape)}")
    for name, t in (("mean", mean), ("rstd", rstd)):
        if _b._plain(name, t, X.dim() - 1, torch.float32, index).shape != X.shape[:-1]:
            raise ValueError(f"{name} must be {tuple(X.shape[:-1])}, got {tuple(t.shape)}")
    if out is None:
        out = torch.empty_like(dY)
    else:
        _b._plain("out", out, X.dim(), gkind, index)
    dweight = torch.empty(C, dtype=torch.float32, device=dev)
    dbias = torch.empty_like(dweight)
    if workspace is None:
        workspace = torch.empty(layer_norm_backward_workspace_bytes(rows, C), dtype=torch.uint8, device=dev)
    else:
        _b._workspace(workspace, 0, dev)
    _b._call(_b.lib().scram_layer_norm_backward, "scram_layer_norm_backward", dev,
             (dY.data_ptr(), _b._dtype_code_of(gkind), X.data_ptr(), code, mean.data_ptr(), rstd.data_ptr(), _b._ptr(weight), wcode, rows,
              C, out.data_ptr(), dweight.data_ptr(), dbias.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size()))
    return out, dweight, dbias


def layer_norm_backward_workspace_bytes(rows: int, channels: int) -> int:
    """Bytes of device workspace ``layer_norm_backward`` needs."""
    return int(_b.lib().scram_layer_norm_backward_workspace_bytes(rows, channels))


ACTIVATIONS = {None: 0, "silu": 1}


def _group(X, groups, weight, bias, activation, out):
    """Checks of a group norm's tensors: (images, pixels, channels, groups, dtype code, weights' dtype code, activation,
    device index)."""
    if X.dim() < 2:
        raise ValueError(f"X must be [images, ..., channels], got {tuple(X.shape)}")
    _, C, code, wcode, index = _norm_rows(X, weight, bias, out)
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {tuple(ACTIVATIONS)}, got {activation!r}")
    groups = int(groups)
    if groups < 1 or C % groups:
        raise ValueError(f"{C} channels do not split into {groups} groups")
    N = X.shape[0]
    return N, X.numel() // (N * C) if N * C else 0, C, groups, code, wcode, ACTIVATIONS[activation], index


@functools.lru_cache(maxsize=1024)
def _group_bytes(backward, *sizes):
    L = _b.lib()
    return int((L.scram_group_norm_backward_workspace_bytes if backward else L.scram_group_norm_workspace_bytes)(*sizes))


def group_norm(X, groups: int, weight=None, bias=None, eps: float = 1e-5, *, activation=None, out=None, stats: bool = False,
               workspace=None):
    """Group norm of images, channels last, and an activation (``scram_group_norm``).

    ``X`` ``[images, ..., channels]``, normalised over an image's pixels and each of ``groups`` groups of neighbouring
    channels; ``weight``, ``bias``: [channels] in X's dtype or float32, or None; ``activation``: None or "silu".  Returns
    the result in X's dtype, with ``stats`` ``(result, mean, rstd)``: fp32 ``[images, groups]``, for
    :func:`group_norm_backward`.  ``out`` may be ``X``.
    ``workspace``: optional uint8 device tensor of at least ``group_norm_workspace_bytes(...)`` bytes.
    """
    torch = _b._torch()
    N, pixels, C, groups, code, wcode, act, index = _group(X, groups, weight, bias, activation, out)
    dev = X.device
    if out is None:
        out = torch.empty_like(X)
    else:
        _b._plain("out", out, X.dim(), X.dtype, index)
    mean = rstd = None
    if stats:
        mean, rstd = torch.empty((2, N, groups), dtype=torch.float32, device=dev)
    if workspace is None:
        size = _group_bytes(False, N, pixels, C, groups, code)
        if size:
            workspace = torch.empty(size, dtype=torch.uint8, device=dev)
    else:
        size = _b._workspace(workspace, 0, dev).numel() * workspace.element_size()
    _b._call(_b.lib().scram_group_norm, "scram_group_norm", dev,
             (X.data_ptr(), code, _b._ptr(weight), _b._ptr(bias), wcode, N, pixels, C, groups, float(eps), act, out.data_ptr(),
              _b._ptr(mean), _b._ptr(rstd), _b._ptr(workspace), size))
    return (out, mean, rstd) if stats else out


def group_norm_backward(dY, X, mean, rstd, weight=None, bias=None, *, activation=None, out=None, workspace=None):
    """Gradients of :func:`group_norm` (``scram_group_norm_backward``): ``(dX, dweight, dbias)``.

    ``dY`` is in X's dtype or float32 and dX in dY's (``out`` may be ``dY``); dweight and dbias are fp32 [channels], also
    where the call had no weights.  ``mean``, ``rstd`` ``[images, groups]``: what the call gave with ``stats``.
    ``workspace``: optional uint8 device tensor of at least ``group_norm_backward_workspace_bytes(...)`` bytes.
    """
    torch = _b._torch()
    index = X.get_device()
    _b._plain("mean", mean, 2, torch.float32, index)
    N, pixels, C, groups, code, wcode, act, index = _group(X, mean.shape[1], weight, bias, activation, out)
    kind, gkind, dev = X.dtype, dY.dtype, X.device
    if gkind != kind and gkind != torch.float32:
        raise TypeError("dY must be float32 or of X's dtype")
    if _b._plain("dY", dY, X.dim(), gkind, index).shape != X.shape:
        raise ValueError(f"dY must be {tuple(X.shape)}, got {tuple(dY.shape)}")
    for name, t in (("mean", mean), ("rstd", rstd)):
        if _b._plain(name, t, 2, torch.float32, index).shape != (N, groups):
            raise ValueError(f"{name} must be {(N, groups)}, got {tuple(t.shape)}")
    if out is None:
        out = torch.empty_like(dY)
    else:
        _b._plain("out", out, X.dim(), gkind, index)
    dweight, dbias = torch.empty((2, C), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = torch.empty(max(_group_bytes(True, N, pixels, C, groups, code), 1), dtype=torch.uint8, device=dev)
    else:
        _b._workspace(workspace, 0, dev)
    _b._call(_b.lib().scram_group_norm_backward, "scram_group_norm_backward", dev,
             (dY.data_ptr(), _b._dtype_code_of(gkind), X.data_ptr(), code, mean.data_ptr(), rstd.data_ptr(), _b._ptr(weight),
              _b._ptr(bias), wcode, N, pixels, C, groups, act, out.data_ptr(), dweight.data_ptr(), dbias.data_ptr(),
              workspace.data_ptr(), workspace.numel() * workspace.element_size()))
    return out, dweight, dbias


def group_norm_workspace_bytes(images: int, pixels: int, channels: int, groups: int, *, dtype) -> int:
    """Bytes of device workspace ``group_norm`` needs (``dtype``: torch dtype of X)."""
    return _group_bytes(False, images, pixels, channels, groups, _b._dtype_code_of(dtype))


def group_norm_backward_workspace_bytes(images: int, pixels: int, channels: int, groups: int, *, dtype) -> int:
    """Bytes of device workspace ``group_norm_backward`` needs (``dtype``: torch dtype of X)."""
    return _group_bytes(True, images, pixels, channels, groups, _b._dtype_code_of(dtype))
