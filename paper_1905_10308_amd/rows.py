"""Operators on channel rows around the attention: rotary grid positions and layer norm, with their gradients.

Argument marshalling only, as in :mod:`.binding`; rows of any width, no padding.
"""
from __future__ import annotations

import ctypes
import functools

from . import binding as _b

ROTARY_INTERLEAVED = 1
ROTARY_INVERSE = 2


@functools.lru_cache(maxsize=64)
def _frequencies(sections, base: float):
    """base ** (-j / m) for pair j of an axis with m pairs, as a ctypes array."""
    f = [base ** (-j / m) for m in sections for j in range(m)]
    return (ctypes.c_double * max(len(f), 1))(*f)


def _rotate(tensors, sections, base, freqs, origin, groups, interleaved, out, inverse):
    torch = _b._torch()
    if not 1 <= len(tensors) <= 4:
        raise ValueError(f"one to four tensors, got {len(tensors)}")
    x = tensors[0]
    for i, t in enumerate(tensors):
        _b._dev_tensor(t, f"tensor {i}")
        if t.dim() not in (4, 5) or t.shape[1:] != x.shape[1:]:
            raise ValueError("tensors must be [S, H, W, d] or [S, T, H, W, d] of one grid and width, got "
                             f"{tuple(t.shape)} and {tuple(x.shape)}")
        if t.dtype != x.dtype:
            raise TypeError("tensors must share a dtype")
    dev, code = x.device, _b._dtype_code(x)
    T, H, W, d = (1,) * (5 - x.dim()) + tuple(x.shape[1:])
    groups = int(groups)
    if groups < 1 or d % groups:
        raise ValueError(f"{d} channels do not split into {groups} groups")
    if sections is None:  # all pairs; an axis each for height and width, or for time, height and width
        pairs = d // groups // 2
        nh = pairs // (2 if x.dim() == 4 else 3)
        nw = pairs - nh if x.dim() == 4 else nh
        sections = (pairs - nh - nw, nh, nw)
    sections = tuple(int(n) for n in sections)
    if len(sections) == 2:
        sections = (0,) + sections
    if len(sections) != 3 or min(sections) < 0:
        raise ValueError(f"sections must be the pairs of (time,) height and width, got {sections}")
    if freqs is None:
        if not base > 0:
            raise ValueError("base must be positive")
        freqs = _frequencies(sections, float(base))
    else:
        freqs = [float(f) for f in freqs]
        if len(freqs) != sum(sections):
            raise ValueError(f"{sum(sections)} pairs need as many freqs, got {len(freqs)}")
        freqs = (ctypes.c_double * max(len(freqs), 1))(*freqs)
    rows, at = 0, None
    if isinstance(origin, torch.Tensor):
        _b._dev_tensor(origin, "origin")
        if origin.dtype != torch.int32 or origin.dim() > 2 or origin.shape[-1:] != (3,):
            raise ValueError("origin must be int32 [3], [1, 3] or [S, 3]: time, height, width")
        rows = origin.numel() // 3
    else:
        at = tuple(int(n) for n in origin)
        at = (ctypes.c_int * 3)(*((0,) * (3 - len(at)) + at))
        origin = None
    if out is None:
        out = [torch.empty_like(t) for t in tensors]
    else:
        out = [out] if isinstance(out, torch.Tensor) else list(out)
        if len(out) != len(tensors):
            raise ValueError(f"{len(tensors)} tensors need as many outputs, got {len(out)}")
        for i, (o, t) in enumerate(zip(out, tensors)):
            _b._check_buffer(o, f"out {i}", t.shape, t.dtype)
    for i, (t, o) in enumerate(zip(tensors, out)):
        _b._same_device(dev, **{f"tensor {i}": t, f"out {i}": o, "origin": origin})
    n = len(tensors)
    _b._call(_b.lib().scram_rotary, "scram_rotary", dev,
             (n, (ctypes.c_void_p * n)(*(t.data_ptr() for t in tensors)), (ctypes.c_void_p * n)(*(t.data_ptr() for t in out)),
              (ctypes.c_int * n)(*(t.shape[0] for t in tensors)), code, T, H, W, d, groups, (ctypes.c_int * 3)(*sections), freqs,
              at, _b._ptr(origin), rows, (ROTARY_INTERLEAVED if interleaved else 0) | (ROTARY_INVERSE if inverse else 0)))
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


def _norm_rows(X, weight, bias, **more):
    torch = _b._torch()
    _b._dev_tensor(X, "X")
    if X.dim() < 1:
        raise ValueError("X must have channels")
    C = X.shape[-1]
    code = _b._dtype_code(X)
    wcode = code
    for name, t in (("weight", weight), ("bias", bias)):
        if t is not None:
            _b._dev_tensor(t, name, 1)
            if t.shape[0] != C:
                raise ValueError(f"{name} must have {C} channels, got {t.shape[0]}")
            if t.dtype not in (X.dtype, torch.float32):
                raise TypeError(f"{name} must be float32 or of X's dtype")
            if weight is not None and t.dtype != weight.dtype:
                raise TypeError("weight and bias must share a dtype")
            wcode = _b._dtype_code(t)
    _b._same_device(X.device, weight=weight, bias=bias, **more)
    return X.numel() // C if C else 0, C, code, wcode


def layer_norm(X, weight=None, bias=None, eps: float = 1e-5, *, out=None, stats: bool = False):
    """Layer norm of the rows (last dimension) of ``X`` (``scram_layer_norm``).

    ``weight``, ``bias``: [channels] in X's dtype or float32, or None.  Returns the normalised rows in X's dtype, with
    ``stats`` ``(rows, mean, rstd)``: fp32 of ``X.shape[:-1]``, for :func:`layer_norm_backward`.  ``out`` may be ``X``.
    """
    torch = _b._torch()
    rows, C, code, wcode = _norm_rows(X, weight, bias, out=out)
    if out is None:
        out = torch.empty_like(X)
    else:
        _b._check_buffer(out, "out", X.shape, X.dtype)
    mean = rstd = None
    if stats:
        mean, rstd = (torch.empty(X.shape[:-1], dtype=torch.float32, device=X.device) for _ in range(2))
    _b._call(_b.lib().scram_layer_norm, "scram_layer_norm", X.device,
             (_b._ptr(X), code, _b._ptr(weight), _b._ptr(bias), wcode, rows, C, float(eps), _b._ptr(out), _b._ptr(mean), _b._ptr(rstd)))
    return (out, mean, rstd) if stats else out


def layer_norm_backward(dY, X, mean, rstd, weight=None, *, out=None, workspace=None):
    """Gradients of :func:`layer_norm` (``scram_layer_norm_backward``): ``(dX, dweight, dbias)``.

    ``dY`` is in X's dtype or float32 and dX in dY's (``out`` may be ``dY``); dweight and dbias are fp32 [channels], also
    where the call had no weights.  ``mean``, ``rstd``: what the call gave with ``stats``.
    ``workspace``: optional uint8 device tensor of at least ``layer_norm_backward_workspace_bytes(rows, channels)`` bytes.
    """
    torch = _b._torch()
    rows, C, code, wcode = _norm_rows(X, weight, None, dY=dY, mean=mean, rstd=rstd, out=out, workspace=workspace)
    _b._dev_tensor(dY, "dY")
    if dY.shape != X.shape:
        raise ValueError(f"dY must be {tuple(X.shape)}, got {tuple(dY.shape)}")
    if dY.dtype not in (X.dtype, torch.float32):
        raise TypeError("dY must be float32 or of X's dtype")
    for name, t in (("mean", mean), ("rstd", rstd)):
        _b._check_buffer(t, name, X.shape[:-1], torch.float32)
    if out is None:
        out = torch.empty_like(dY)
    else:
        _b._check_buffer(out, "out", dY.shape, dY.dtype)
    dweight, dbias = (torch.empty(C, dtype=torch.float32, device=X.device) for _ in range(2))
    workspace = _b._workspace(workspace, layer_norm_backward_workspace_bytes(rows, C), X.device)
    _b._call(_b.lib().scram_layer_norm_backward, "scram_layer_norm_backward", X.device,
             (_b._ptr(dY), _b._dtype_code(dY), _b._ptr(X), code, _b._ptr(mean), _b._ptr(rstd), _b._ptr(weight), wcode, rows, C,
              _b._ptr(out), _b._ptr(dweight), _b._ptr(dbias), _b._ptr(workspace), workspace.numel() * workspace.element_size()))
    return out, dweight, dbias


def layer_norm_backward_workspace_bytes(rows: int, channels: int) -> int:
    """Bytes of device workspace ``layer_norm_backward`` needs."""
    return int(_b.lib().scram_layer_norm_backward_workspace_bytes(rows, channels))
