"""A table of embeddings on torch tensors: rows by id, and the table's gradient
(``pp_embed_*`` of ``include/pp.h``).

``embed_fwd``   features of ids, a row of the table times a scale each
``embed_bwd``   the table's gradient from that of the features

The features are what ``linear_xent_*`` takes as token rows.  As there, no call
records an autograd graph.
"""
from __future__ import annotations

import ctypes
import functools
import struct

from . import _check, _dtype_code, _torch, load_library
from .train import _changed, _empty, _entry, _native, _p, _stream_of

_DESC = struct.Struct("@2i6qf4x")     # pp_embed_desc as the library lays it out


def bind(lib):
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    for name, at in {"pp_embed_fwd": [vp, vp, vp, vp, vp], "pp_embed_workspace": [vp, ctypes.POINTER(sz)],
                     "pp_embed_bwd": [vp, vp, vp, vp, vp, vp, sz, vp]}.items():
        if hasattr(lib, name):
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = at, ctypes.c_int32


def _dtype_of(dtype, name):
    torch = _torch()
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"{name} must be float32 or bfloat16, got {dtype}")
    return 1 if dtype == torch.bfloat16 else 0


def _ids(ids):
    torch = _torch()
    if ids.dtype != torch.int64 or not ids.is_contiguous():
        raise ValueError("ids must be contiguous int64")
    if not ids.is_cuda:
        raise ValueError("the tensors must be on a GPU")


def _rows(t, name, shape, device):
    """Elements from one row to the next of [.., d], whose leading axes lie as one
    in memory."""
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must be of shape {shape}, got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} must be on the ids' device")
    d = shape[-1]
    if t.numel() == 0 or t.is_contiguous():
        return d
    if d > 1 and t.stride(-1) != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    ld, n = None, 1
    for size, step in zip(reversed(shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if ld is None:
            ld = step
        elif step != ld * n:
            raise ValueError(f"the leading axes of {name} do not lie as one axis in memory (call contiguous())")
        n *= size
    if ld is None:
        return d
    if ld < d:
        raise ValueError(f"the rows of {name} overlap")
    return ld


def _done(got, name):
    """What a native call gave, unless it is a status."""
    if type(got) is int:
        _check(got, name)
    return got


def embed_fwd(ids, w, scale=1.0, ignore_index=-100, dtype=None, out=None, stream=None):
    """pp_embed_fwd: ``scale * w[ids]``, features [*ids.shape, d].

    ids: contiguous int64 of any shape; w: [v, d] float32 or bfloat16 with
    contiguous rows; ``dtype``: of the features (w's if None).  Fills ``out``, if
    given, whose rows may lie apart.  ``ignore_index`` gives zeros, another id
    outside of 0..v-1 NaN."""
    torch = _torch()
    if out is None and stream is None and ids.is_cuda:
        with _stream_of(None, ids.device) as sp:
            y = _native().embed_fwd(ids, w, dtype, scale, ignore_index, _entry("pp_embed_fwd"), sp)
        if y is not None:
            return _done(y, "pp_embed_fwd")
    code = _dtype_code(w)
    if w.dim() != 2 or w.shape[0] < 1 or w.shape[1] < 1:
        raise ValueError(f"w must be [v, d], got {tuple(w.shape)}")
    _ids(ids)
    v, d = w.shape
    w_ld = _rows(w, "w", (v, d), ids.device)
    shape = (*ids.shape, d)
    if out is None:
        y_ld = d
        yc = code if dtype is None else _dtype_of(dtype, "dtype")
    else:
        if dtype is not None and out.dtype != dtype:
            raise TypeError(f"out must be of dtype {dtype}, got {out.dtype}")
        yc = _dtype_of(out.dtype, "out")
        y_ld = _rows(out, "out", shape, ids.device)
        if out.numel() and out.data_ptr() in (w.data_ptr(), ids.data_ptr()):
            raise ValueError("out is another tensor of the call")
    desc = _DESC.pack(code, yc, ids.numel(), v, d, w_ld, y_ld, ignore_index, scale)
    given = out is not None
    with _stream_of(stream, ids.device) as sp:
        if not given:
            out = _empty(shape, torch.bfloat16 if yc else torch.float32, ids.device, stream)
        _check(load_library().pp_embed_fwd(desc, ids.data_ptr(), w.data_ptr(), out.data_ptr(), sp),
               "pp_embed_fwd")
    if given:
        _changed([out])
    return out


@functools.lru_cache(maxsize=256)
def _bytes(desc):
    """pp_embed_workspace of a description: a function of it alone."""
    nb = ctypes.c_size_t(0)
    _check(load_library().pp_embed_workspace(desc, ctypes.byref(nb)), "pp_embed_workspace")
    return nb.value


def embed_bwd(ids, dy, v, scale=1.0, ignore_index=-100, dtype=None, add=None, out=None, stream=None):
    """pp_embed_bwd: the gradient [v, d] of a table from its features' gradient
    ``dy`` [*ids.shape, d], whose rows may lie apart.

    ``dtype``: of the result (dy's if None; ``add``'s or ``out``'s where given).
    ``add``: a gradient of the same table to add to (a table whose rows are a
    head's weights too).  Fills ``out``, if given; it may be ``add``, and then only
    the rows that ids reach are touched."""
    torch = _torch()
    if out is None and stream is None and ids.is_cuda:
        with _stream_of(None, ids.device) as sp:
            dw = _native().embed_bwd(ids, dy, v, dtype, scale, ignore_index, add, _entry("pp_embed_workspace"), _entry("pp_embed_bwd"), sp)
        if dw is not None:
            return _done(dw, "pp_embed_bwd")
    yc = _dtype_code(dy)
    _ids(ids)
    if dy.dim() < 1 or dy.shape[-1] < 1 or int(v) < 1:
        raise ValueError("dy must be [..., d] and v at least 1")
    d = dy.shape[-1]
    y_ld = _rows(dy, "dy", (*ids.shape, d), ids.device)
    shape, w_ld, kind = (int(v), d), None, dtype
    for name, t in (("add", add), ("out", out)):
        if t is not None:
            if kind is not None and t.dtype != kind:
                raise TypeError(f"{name} must be of dtype {kind}, got {t.dtype}")
            kind = t.dtype
            ld = _rows(t, name, shape, ids.device)
            if w_ld is not None and ld != w_ld:
                raise ValueError("add and out must have the same strides")
            w_ld = ld
    wc = yc if kind is None else _dtype_of(kind, "dtype")
    if out is None and add is not None and w_ld != d:
        raise ValueError("add must be contiguous where out is not given")
    if out is not None and out.data_ptr() in (ids.data_ptr(), dy.data_ptr()):
        raise ValueError("out is another tensor of the call")
    desc = _DESC.pack(wc, yc, ids.numel(), int(v), d, w_ld or d, y_ld, ignore_index, scale)
    given = out is not None
    with _stream_of(stream, ids.device) as sp:
        if not given:
            out = _empty(shape, torch.bfloat16 if wc else torch.float32, ids.device, stream)
        nb = _bytes(desc)
        ws = _empty(nb, torch.uint8, ids.device, stream)
        _check(load_library().pp_embed_bwd(desc, ids.data_ptr(), dy.data_ptr(), _p(add), out.data_ptr(),
                                           ws.data_ptr(), nb, sp), "pp_embed_bwd")
    if given:
        _changed([out])
    return out
