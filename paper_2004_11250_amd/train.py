"""Training operators: the loss of a linear head with its gradient, and the
orthogonalised weight step of pruned layers (the calls of ``include/pp.h``'s
training section, on torch tensors).

``linear_xent_fwd`` / ``linear_xent_bwd`` / ``linear_xent_step``
    softmax cross entropy of a 1x1 convolution or fully connected layer over
    any number of classes, and its gradients, without keeping the logits.
``orthogonalize``
    a list of updates, each replaced by its Newton-Schulz iterate (singular
    values taken towards 1).
``muon_step``
    momentum, orthogonalised update and weight step of a list of layers; a
    pruned 3x3 layer (``keep_masks``) stays on its kept taps.

As elsewhere in this package every computation runs in the library's kernels;
this module checks and marshals arguments, and allocates outputs and scratch
on the stream of the call.

No call records an autograd graph.  Tensors that require a gradient are read as
they are, and no result requires one: the gradients that ``linear_xent_bwd`` and
``linear_xent_step`` return are passed on by hand (``features.backward(dx)``).
Tensors that a call writes in place count as changed: a graph that has saved one
refuses its backward pass.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools

import numpy as np

from . import _check, _dtype_code, _stream_ptr, _torch, load_library

PP_MEAN, PP_SUM, PP_NONE = 0, 1, 2
PP_XENT_FWD, PP_XENT_BWD = 1, 2
_REDUCTION = {"mean": PP_MEAN, "sum": PP_SUM, "none": PP_NONE}


class XentDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("reduction", ctypes.c_int32), ("n", ctypes.c_int64), ("d", ctypes.c_int64),
                ("hw", ctypes.c_int64), ("v", ctypes.c_int64), ("x_sn", ctypes.c_int64), ("x_sc", ctypes.c_int64),
                ("x_sp", ctypes.c_int64), ("dx_sn", ctypes.c_int64), ("dx_sc", ctypes.c_int64),
                ("dx_sp", ctypes.c_int64), ("w_ld", ctypes.c_int64), ("ignore_index", ctypes.c_int64)]


class OrthoMat(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("u", ctypes.c_void_p), ("u_rs", ctypes.c_int64),
                ("u_cs", ctypes.c_int64), ("o", ctypes.c_void_p), ("o_rs", ctypes.c_int64), ("o_cs", ctypes.c_int64)]


class MuonLayer(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("w", ctypes.c_void_p), ("g", ctypes.c_void_p),
                ("momentum", ctypes.c_void_p), ("w_out", ctypes.c_void_p), ("momentum_out", ctypes.c_void_p),
                ("keep", ctypes.c_void_p)]


class MuonDesc(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("momentum", ctypes.c_float), ("weight_decay", ctypes.c_float),
                ("nesterov", ctypes.c_int32), ("steps", ctypes.c_int32), ("coeffs", ctypes.c_float * 3),
                ("eps", ctypes.c_float)]


def bind(lib):
    """Argument types of the training calls (a library without them, the
    host-only one, is left as it is)."""
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    desc = ctypes.POINTER(XentDesc)
    argtypes = {
        "pp_xent_workspace": [desc, i32, ctypes.POINTER(sz)],
        "pp_xent_fwd": [desc, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
        "pp_xent_bwd": [desc, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
        "pp_xent_step": [desc, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
        "pp_ortho_workspace": [vp, i32, i32, ctypes.POINTER(sz)],
        "pp_ortho": [vp, i32, i32, i32, ctypes.POINTER(ctypes.c_float), ctypes.c_float, vp, sz, vp],
        "pp_muon_workspace": [vp, i32, i32, ctypes.POINTER(sz)],
        "pp_muon_step": [vp, i32, i32, ctypes.POINTER(MuonDesc), vp, sz, vp],
    }
    for name, at in argtypes.items():
        if hasattr(lib, name):
            fn = getattr(lib, name)
            fn.argtypes = at
            fn.restype = i32


def _p(t):
    return None if t is None else t.data_ptr()


def _on(stream, device):
    """Context in which tensors belong to the call's stream."""
    if stream is None:
        return contextlib.nullcontext()
    torch = _torch()
    return torch.cuda.stream(torch.cuda.ExternalStream(int(stream.cuda_stream), device))


def _changed(tensors):
    """Tell autograd that a call has written these."""
    _torch().autograd.graph.increment_version(tensors)


def _flat_pixels(x):
    """(n, d, hw, strides) of features [n, d, ...]; the pixel axes have to be
    one axis in memory."""
    n, d = x.shape[0], x.shape[1]
    sizes, strides = list(x.shape[2:]), list(x.stride()[2:])
    hw, sp = 1, 1
    for size, step in zip(reversed(sizes), reversed(strides)):   # from the innermost axis out
        if size != 1 and hw != 1 and step != hw * sp and 0 not in x.shape:
            raise ValueError("the pixel axes of x do not lie as one axis in memory (call contiguous())")
        if size != 1 and hw == 1:
            sp = step
        hw *= size
    return n, d, hw, (x.stride(0), x.stride(1), sp)


def _xent_args(x, w, target, bias, class_weight, ignore_index, reduction):
    torch = _torch()
    if reduction not in _REDUCTION:
        raise ValueError(f"reduction must be one of {sorted(_REDUCTION)}, got {reduction!r}")
    if x.dim() < 2 or w.dim() < 2 or any(k != 1 for k in w.shape[2:]):
        raise ValueError("x must be [n, d, ...] and w [v, d] (or [v, d, 1, 1])")
    dt = _dtype_code(x)
    if w.dtype != x.dtype:
        raise TypeError(f"w must be of x's dtype {x.dtype}, got {w.dtype}")
    if w.dim() > 2:
        w = w.reshape(w.shape[0], w.shape[1])
    if w.shape[1] != x.shape[1] or w.shape[0] < 1 or w.shape[1] < 1:
        raise ValueError(f"w {tuple(w.shape)} does not fit features {tuple(x.shape)}")
    if w.stride(1) != 1 and w.shape[1] != 1 or w.shape[0] > 1 and w.stride(0) < w.shape[1]:
        raise ValueError("the rows of w must be contiguous")
    if tuple(target.shape) != (x.shape[0],) + tuple(x.shape[2:]) or target.dtype != torch.int64:
        raise ValueError(f"target must be int64 of shape {(x.shape[0],) + tuple(x.shape[2:])}")
    if not target.is_contiguous():
        raise ValueError("target must be contiguous")
    for name, t in (("bias", bias), ("class_weight", class_weight)):
        if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (w.shape[0],) or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous float32 [{w.shape[0]}]")
    for t in (w, target, bias, class_weight):
        if t is not None and t.device != x.device:
            raise ValueError("all tensors must be on x's device")
    if not x.is_cuda:
        raise ValueError("the tensors must be on a GPU")
    n, d, hw, (sn, sc, sp) = _flat_pixels(x)
    v = w.shape[0]
    ld = w.stride(0) if v > 1 else d
    desc = XentDesc(dt, _REDUCTION[reduction], n, d, hw, v, sn, sc, sp, d * hw, hw, 1, ld, int(ignore_index))
    return desc, w


def _xent_grad_arg(grad, target, reduction):
    torch = _torch()
    if grad is None:
        return
    want = tuple(target.shape) if reduction == "none" else ()
    if grad.dtype != torch.float32 or (tuple(grad.shape) != want and grad.numel() != (target.numel() if want else 1)) \
            or not grad.is_contiguous() or grad.device != target.device:
        raise ValueError(f"grad must be contiguous float32 of shape {want} on the targets' device")


@functools.lru_cache(maxsize=256)
def _xent_bytes(desc, parts):
    """pp_xent_workspace of a description (as bytes): a function of it alone."""
    nb = ctypes.c_size_t(0)
    _check(load_library().pp_xent_workspace(ctypes.byref(XentDesc.from_buffer_copy(desc)), parts, ctypes.byref(nb)),
           "pp_xent_workspace")
    return max(nb.value, 256)


def _xent_workspace(desc, parts, device):
    return _torch().empty(_xent_bytes(bytes(desc), parts), dtype=_torch().uint8, device=device)


def linear_xent_fwd(x, w, target, bias=None, class_weight=None, ignore_index=-100, reduction="mean", stream=None):
    """pp_xent_fwd: softmax cross entropy of the logits ``w x + bias``.

    x: features [n, d, ...] (float32 or bfloat16; channels first or last, or
    token rows [t, d]); w: [v, d] or a 1x1 convolution's [v, d, 1, 1]; target:
    int64 [n, ...].  Returns (loss, stats): loss a float32 scalar, or [n, ...]
    with reduction="none"; stats, float32 [tokens + 1], each token's
    log-sum-exp (0 where ignored) and the loss's divisor, for
    linear_xent_bwd."""
    torch = _torch()
    desc, w = _xent_args(x, w, target, bias, class_weight, ignore_index, reduction)
    with _on(stream, x.device):
        loss = torch.empty(target.shape if reduction == "none" else (), dtype=torch.float32, device=x.device)
        stats = torch.empty(desc.n * desc.hw + 1, dtype=torch.float32, device=x.device)
        ws = _xent_workspace(desc, PP_XENT_FWD, x.device)
    _check(load_library().pp_xent_fwd(ctypes.byref(desc), _p(x), _p(w), _p(bias), _p(class_weight), _p(target), _p(loss),
                                      _p(stats), _p(ws), ws.numel(), _stream_ptr(stream)), "pp_xent_fwd")
    return loss, stats


def _xent_outputs(desc, x, w, bias, need):
    torch = _torch()
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if need[0] else None
    dw = torch.empty(w.shape, dtype=w.dtype, device=x.device) if need[1] else None
    db = torch.empty(desc.v, dtype=torch.float32, device=x.device) if need[2] and bias is not None else None
    return dx, dw, db


def linear_xent_bwd(x, w, target, stats, grad=None, bias=None, class_weight=None, ignore_index=-100, reduction="mean",
                    need=(True, True, True), stream=None):
    """pp_xent_bwd: (dx, dw, db) of the loss that linear_xent_fwd returned with
    ``stats``, times ``grad`` (a scalar tensor, or one value a token with
    reduction="none"; None: ones).  dx is contiguous in x's shape, dw in w's;
    db is None without a bias.  need: which of the three to compute."""
    torch = _torch()
    shape = w
    desc, w = _xent_args(x, w, target, bias, class_weight, ignore_index, reduction)
    _xent_grad_arg(grad, target, reduction)
    if stats.dtype != torch.float32 or stats.numel() != desc.n * desc.hw + 1 or not stats.is_contiguous() \
            or stats.device != x.device:
        raise ValueError("stats must be what linear_xent_fwd returned for these features")
    with _on(stream, x.device):
        dx, dw, db = _xent_outputs(desc, x, shape, bias, need)
        ws = _xent_workspace(desc, PP_XENT_BWD, x.device)
    _check(load_library().pp_xent_bwd(ctypes.byref(desc), _p(x), _p(w), _p(bias), _p(class_weight), _p(target), _p(stats),
                                      _p(grad), _p(dx), _p(dw), _p(db), _p(ws), ws.numel(), _stream_ptr(stream)),
           "pp_xent_bwd")
    return dx, dw, db


def linear_xent_step(x, w, target, grad=None, bias=None, class_weight=None, ignore_index=-100, reduction="mean",
                     need=(True, True, True), stream=None):
    """pp_xent_step: (loss, dx, dw, db), forward and backward in one call."""
    torch = _torch()
    shape = w
    desc, w = _xent_args(x, w, target, bias, class_weight, ignore_index, reduction)
    _xent_grad_arg(grad, target, reduction)
    with _on(stream, x.device):
        loss = torch.empty(target.shape if reduction == "none" else (), dtype=torch.float32, device=x.device)
        stats = torch.empty(desc.n * desc.hw + 1, dtype=torch.float32, device=x.device)
        dx, dw, db = _xent_outputs(desc, x, shape, bias, need)
        ws = _xent_workspace(desc, PP_XENT_FWD | PP_XENT_BWD, x.device)
    _check(load_library().pp_xent_step(ctypes.byref(desc), _p(x), _p(w), _p(bias), _p(class_weight), _p(target), _p(grad),
                                       _p(loss), _p(stats), _p(dx), _p(dw), _p(db), _p(ws), ws.numel(),
                                       _stream_ptr(stream)), "pp_xent_step")
    return loss, dx, dw, db


# ---------------------------------------------------------------------------
# orthogonalised updates
# ---------------------------------------------------------------------------

COEFFS = (3.4445, -4.7750, 2.0315)


def _matrix(t, name):
    """(rows, cols, row stride, column stride) of [rows, ...] taken as a matrix."""
    if t.dim() < 2:
        raise ValueError(f"{name} must have two axes or more, got {tuple(t.shape)}")
    if t.numel() == 0:
        return t.shape[0], 0, 0, 1
    if t.dim() > 2:
        try:
            t = t.view(t.shape[0], -1)
        except RuntimeError:
            raise ValueError(f"the trailing axes of {name} do not lie as one axis in memory (call contiguous())") from None
    return t.shape[0], t.shape[1], t.stride(0), t.stride(1)


def _one_dtype(tensors, name):
    if not tensors:
        raise ValueError(f"{name} is empty")
    dt, dev = tensors[0].dtype, tensors[0].device
    code = _dtype_code(tensors[0])
    for t in tensors:
        if t.dtype != dt or t.device != dev:
            raise ValueError(f"{name} must be of one dtype and on one device")
    return code, dev


def _own_places(outs, ins, more=()):
    """outs[i] may be ins[i] and no other tensor of a call: the matrices of a list
    are read and written in no order.  (By where they begin.)"""
    at = {}
    for i, t in enumerate(outs):
        if any(step == 0 and size > 1 for step, size in zip(t.stride(), t.shape)):
            raise ValueError("elements of an output share their memory")
        if t.numel() and at.setdefault(t.data_ptr(), i) != i:
            raise ValueError("two outputs are the same tensor")
    for i, t in enumerate(ins):
        if t.numel() and at.get(t.data_ptr(), i) != i:
            raise ValueError("an output is another matrix's input")
    for t in more:
        if t.numel() and t.data_ptr() in at:
            raise ValueError("an output is another tensor of the call")


def _coeffs(coeffs):
    if len(coeffs) != 3:
        raise ValueError("coeffs must be three numbers")
    return (ctypes.c_float * 3)(*(float(c) for c in coeffs))


def orthogonalize(mats, steps=5, coeffs=COEFFS, eps=1e-7, out=None, stream=None):
    """pp_ortho: the Newton-Schulz iterate of each update, a tensor or a list of
    them ([rows, ...], trailing axes taken together; float32 or bfloat16, any
    strides), all in one call.  Returns contiguous tensors of the same shapes,
    or fills ``out``, each of which may be its own input."""
    torch = _torch()
    single = torch.is_tensor(mats)
    mats = [mats] if single else list(mats)
    code, dev = _one_dtype(mats, "mats")
    k = _coeffs(coeffs)
    if out is not None:
        out = [out] if torch.is_tensor(out) else list(out)
        if len(out) != len(mats) or any(o.shape != t.shape or o.dtype != t.dtype or o.device != dev
                                        for o, t in zip(out, mats)):
            raise ValueError("out must match mats")
        _own_places(out, mats)
    shapes = [_matrix(t, "a matrix of mats") for t in mats]
    if dev.type != "cuda":
        raise ValueError("the tensors must be on a GPU")
    lib = load_library()
    given = out is not None
    with _on(stream, dev):
        if not given:
            out = [torch.empty(t.shape, dtype=t.dtype, device=dev) for t in mats]
        arr = (OrthoMat * len(mats))()
        for e, t, o, (r, c, rs, cs) in zip(arr, mats, out, shapes):
            _, _, ors, ocs = _matrix(o, "a matrix of out")
            e.rows, e.cols, e.u, e.u_rs, e.u_cs, e.o, e.o_rs, e.o_cs = r, c, t.data_ptr(), rs, cs, o.data_ptr(), ors, ocs
        nb = ctypes.c_size_t(0)
        _check(lib.pp_ortho_workspace(arr, len(mats), code, ctypes.byref(nb)), "pp_ortho_workspace")
        ws = torch.empty(max(nb.value, 256), dtype=torch.uint8, device=dev)
    _check(lib.pp_ortho(arr, len(mats), code, int(steps), k, float(eps), ws.data_ptr(), ws.numel(), _stream_ptr(stream)),
           "pp_ortho")
    if given:
        _changed(out)
    return out[0] if single else out


def keep_masks(pattern_id, conn, lib_masks):
    """int16 [c_out][c_in]: the tap mask of each kernel of a pruned layer (0 where
    it is removed), for muon_step's ``keep`` (as a tensor on the GPU)."""
    pid = np.asarray(pattern_id, dtype=np.int64)
    on = np.asarray(conn)
    masks = np.asarray(lib_masks, dtype=np.int64)
    if pid.shape != on.shape or pid.ndim != 2:
        raise ValueError("pattern_id and conn must be [c_out][c_in]")
    if np.any((on != 0) & ((pid < 0) | (pid >= len(masks)))):
        raise ValueError("a kept kernel's pattern is not in the library")
    return np.where(on != 0, masks[np.clip(pid, 0, len(masks) - 1)], 0).astype(np.int16)


def muon_step(weights, grads, momenta, lr, momentum=0.95, nesterov=True, weight_decay=0.0, keep=None, steps=5,
              coeffs=COEFFS, eps=1e-7, out=None, stream=None):
    """pp_muon_step on lists of tensors (or single ones): weights and grads
    [rows, ...] of one dtype (float32 or bfloat16), momenta float32 of the same
    shapes, all contiguous.  ``keep``: None, or for each layer None or the int16
    tap masks [c_out][c_in] of a pruned 3x3 layer (keep_masks).  Updates weights
    and momenta in place, or fills ``out`` = (weights, momenta), and returns
    them.  What is written is each layer's own: a weight may be listed once."""
    torch = _torch()
    single = torch.is_tensor(weights)
    if single:
        weights, grads, momenta, keep = [weights], [grads], [momenta], [keep]
        out = None if out is None else ([out[0]], [out[1]])
    weights, grads, momenta = list(weights), list(grads), list(momenta)
    keep = [None] * len(weights) if keep is None else list(keep)
    code, dev = _one_dtype(weights, "weights")
    k = _coeffs(coeffs)
    wo, mo = (weights, momenta) if out is None else (list(out[0]), list(out[1]))
    if not len(weights) == len(grads) == len(momenta) == len(keep) == len(wo) == len(mo):
        raise ValueError("weights, grads, momenta, keep and out must be of one length")
    arr = (MuonLayer * len(weights))()
    for e, w, g, m, kp, w2, m2 in zip(arr, weights, grads, momenta, keep, wo, mo):
        for name, t, dt in (("grads", g, w.dtype), ("momenta", m, torch.float32), ("out weights", w2, w.dtype),
                            ("out momenta", m2, torch.float32), ("weights", w, w.dtype)):
            if t.shape != w.shape or t.dtype != dt or t.device != dev or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous {dt} of its weights' shape {tuple(w.shape)} and device")
        r, c, _, _ = _matrix(w, "a weight")
        if kp is not None and (kp.dtype != torch.int16 or tuple(kp.shape) != tuple(w.shape[:2]) or c != 9 * kp.shape[1]
                               or not kp.is_contiguous() or kp.device != dev):
            raise ValueError("keep must be contiguous int16 [c_out][c_in] of a 3x3 layer's weights, on their device")
        e.rows, e.cols, e.w, e.g, e.momentum = r, c, w.data_ptr(), g.data_ptr(), m.data_ptr()
        e.w_out, e.momentum_out, e.keep = w2.data_ptr(), m2.data_ptr(), _p(kp)
    _own_places(wo + mo, weights + momenta, grads)
    if dev.type != "cuda":
        raise ValueError("the tensors must be on a GPU")
    lib = load_library()
    nb = ctypes.c_size_t(0)
    _check(lib.pp_muon_workspace(arr, len(weights), code, ctypes.byref(nb)), "pp_muon_workspace")
    with _on(stream, dev):
        ws = torch.empty(max(nb.value, 256), dtype=torch.uint8, device=dev)
    d = MuonDesc(float(lr), float(momentum), float(weight_decay), int(bool(nesterov)), int(steps), k, float(eps))
    _check(lib.pp_muon_step(arr, len(weights), code, ctypes.byref(d), ws.data_ptr(), ws.numel(), _stream_ptr(stream)),
           "pp_muon_step")
    _changed(wo + mo)
    return (wo[0], mo[0]) if single else (wo, mo)
