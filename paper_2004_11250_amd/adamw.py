"""AdamW steps of lists of tensors, and the norm of their gradients, on torch
tensors (``pp_adamw_*`` and ``pp_grad_norm`` of ``include/pp.h``).

``AdamWState``   the moments of a list, in 32 bits or in 8
``adamw_step``   one step of all tensors of the list
``grad_norm``    the norm of a list of gradients and the factor that clips it

For what ``muon_step`` is not for (biases, tables, heads), or in its place.  Step
count, learning rate and gradient scale may be tensors on the GPU, so that a
recorded graph can be replayed with others.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import struct

import numpy as np

from . import _check, _torch, load_library
from .train import _empty, _entry, _native, _on, _stream_of

BLOCK = 128     # PP_ADAMW_BLOCK

# pp_adamw_tensor (as eight words), pp_adamw_desc and pp_grad as the library lays them out
_TENSOR = ("n", "w", "g", "w_out", "copy", "keep", "at", "weight_decay")
_N, _AT, _DECAY = (_TENSOR.index(name) for name in ("n", "at", "weight_decay"))
_DESC = struct.Struct("@3i4dq3Q64x")     # (the moments' addresses: the native module's)


def bind(lib):
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    for name, at in {"pp_adamw_step": [vp, i32, vp, vp],
                     "pp_adamw_values": [vp, vp, vp, vp, i64, i32, vp, vp, vp],
                     "pp_grad_norm_workspace": [vp, i32, i32, ctypes.POINTER(sz)],
                     "pp_grad_norm": [vp, i32, i32, ctypes.c_float, vp, vp, sz, vp]}.items():
        if hasattr(lib, name):
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = at, i32


class AdamWState:
    """The moments of a list of tensors: zeros, before the first step.

    m, v             flat tensors of all moments.  Tensor i's are the elements from
                     ``places[i]`` on (a multiple of 128), 0 up to the next tensor.
                     float32 with bits=32; with bits=8 float8_e4m3fn, and float16
                     whose whole part is a code of 8 bits and whose fraction what the
                     code leaves out, in sixths of one (pp.h has the format)
    m_scale, v_scale with bits=8: float32, for each block of 128 codes (else None)

    Saving these four and copying them into a new state continues a run.
    ``tensors``: the list, or its shapes (then ``device`` says where)."""

    def __init__(self, tensors, bits=32, device=None):
        torch = _torch()
        if bits not in (32, 8):
            raise ValueError(f"bits must be 32 or 8, got {bits}")
        tensors = [tensors] if torch.is_tensor(tensors) else list(tensors)
        if not tensors:
            raise ValueError("tensors is empty")
        if device is None:
            device = tensors[0].device if torch.is_tensor(tensors[0]) else torch.device("cuda", torch.cuda.current_device())
        self.bits = bits
        self.shapes = [torch.Size(t.shape if torch.is_tensor(t) else t) for t in tensors]
        self.sizes = [math.prod(s) for s in self.shapes]
        self.places, at = [], 0
        for n in self.sizes:
            self.places.append(at)
            at += -(-n // BLOCK) * BLOCK
        self.elements = at
        # the list as the library takes it, without addresses
        self._table = np.zeros((len(self.sizes), len(_TENSOR)), np.int64)
        self._table[:, _N], self._table[:, _AT] = self.sizes, self.places
        self._dims = np.array([n for s in self.shapes for n in (len(s), *s)] or [0], np.int64)

        def zeros(n, dtype):
            return torch.zeros(n, dtype=torch.uint8, device=device).view(dtype)

        if bits == 32:
            self.m, self.v = zeros(4 * at, torch.float32), zeros(4 * at, torch.float32)
            self.m_scale = self.v_scale = None
        else:
            self.m, self.v = zeros(at, torch.float8_e4m3fn), zeros(2 * at, torch.float16)
            self.m_scale, self.v_scale = (zeros(4 * (at // BLOCK), torch.float32) for _ in range(2))

    def _buffers(self):
        return self.m, self.v, self.m_scale, self.v_scale

    def buffers(self):
        """(m, v, m_scale, v_scale), checked: whoever holds a state may have put others in their places."""
        torch, n, blocks = _torch(), self.elements, self.elements // BLOCK
        got = self._buffers()
        if self.bits == 32:
            want = ((torch.float32, n), (torch.float32, n))
        else:
            want = ((torch.float8_e4m3fn, n), (torch.float16, n), (torch.float32, blocks), (torch.float32, blocks))
        device = self.m.device
        for t, (dtype, n) in zip(got, want):
            if t.dtype != dtype or t.numel() != n or not t.is_contiguous() or t.device != device:
                raise ValueError(f"the state's buffers must be contiguous, of {n} {dtype} and on one device")
        return got

    def split(self, flat):
        """Views of a flat tensor of the moments' layout, one in each tensor's shape."""
        return [flat[a:a + n].view(s) for a, n, s in zip(self.places, self.sizes, self.shapes)]

    def values(self, dtype=None, stream=None):
        """pp_adamw_values: the moments (m, v) as flat tensors of ``dtype`` (float32
        if None, or bfloat16): what the codes stand for with bits=8, without their
        fractions.  With bits=32 and float32 they are the state's own."""
        torch = _torch()
        dtype = torch.float32 if dtype is None else dtype
        if dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"dtype must be float32 or bfloat16, got {dtype}")
        m, v, ms, vs = self.buffers()
        if not m.is_cuda:
            raise ValueError("the tensors must be on a GPU")
        if self.bits == 32:
            with _on(stream, m.device):
                return m.to(dtype), v.to(dtype)
        with _stream_of(stream, m.device) as sp:
            out = [_empty(self.elements, dtype, m.device, stream) for _ in range(2)]
            _check(load_library().pp_adamw_values(m.data_ptr(), v.data_ptr(), ms.data_ptr(), vs.data_ptr(), self.elements,
                                                  int(dtype == torch.bfloat16), out[0].data_ptr(), out[1].data_ptr(), sp),
                   "pp_adamw_values")
        return tuple(out)


def _list(t):
    return [t] if _torch().is_tensor(t) else list(t)


def _fit(name, tensors, dtype, device, shapes=None):
    """Refuses a list whose tensors are not contiguous, of a dtype and device, and of
    the shapes."""
    if shapes is not None and [t.shape for t in tensors] != shapes:
        raise ValueError(f"{name} must be of the state's shapes")
    if any(t.device != device or t.dtype != dtype or not t.is_contiguous() for t in tensors):
        raise ValueError(f"{name} must be contiguous {dtype} on one device, {device}")


def _scalar(name, t, dtype, device):
    if t.dtype != dtype or t.numel() != 1 or t.device != device:
        raise ValueError(f"{name} must be one {dtype} on the state's device")
    return t.data_ptr()


# outputs are each their own, but a weight may be written in place (by where tensors begin)
_NAMES = ("weights", "grads", "out weights", "copies")
_OWN = (None, "two outputs are the same tensor", "an output is another tensor of the call", "an output is another tensor's input")


def adamw_step(weights, grads, state, lr, step, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, keep=None, copies=None,
               grad_scale=None, out=None, stream=None):
    """pp_adamw_step on a list of tensors (or a single one) and its AdamWState.

    weights and grads: contiguous, of the state's shapes, each list float32 or
    bfloat16.  ``step`` counts from 1; ``weight_decay``: one number or one a tensor;
    ``keep``: None, or for each tensor None or the int16 tap masks [c_out][c_in] of
    a pruned 3x3 layer (keep_masks); ``copies``: bfloat16 tensors that get the new
    weights, rounded.  ``lr``, ``step`` and ``grad_scale`` (that ``grad_norm``
    returns) may be tensors of one float32, int64 and float32 on the GPU.  Where
    grad_scale is not finite no step is taken, and ``step`` must not count it: a
    count on the GPU goes on by ``torch.isfinite(grad_scale)``.

    Updates weights and state in place, or fills ``out`` = (weights, state), and
    returns them."""
    torch = _torch()
    single = torch.is_tensor(weights)
    weights, grads = _list(weights), _list(grads)
    if single and keep is not None and torch.is_tensor(keep):
        keep = [keep]
    shapes, count = state.shapes, len(state.shapes)
    if len(weights) != count or len(grads) != count:
        raise ValueError(f"weights and grads must be of the state's length {count}")
    dev, wt, gt = state.m.device, weights[0].dtype, grads[0].dtype
    for name, dt in (("weights", wt), ("grads", gt)):
        if dt not in (torch.float32, torch.bfloat16):
            raise TypeError(f"{name} must be float32 or bfloat16, got {dt}")
    new, state_out = weights, state
    if out is not None:
        new, state_out = _list(out[0]), out[1]
        if len(new) != count or state_out.bits != state.bits or state_out.shapes != shapes:
            raise ValueError("out must be weights and a state of the same shapes and bits")
        if state_out.m.device != dev:
            raise ValueError("out must be on the state's device")
    if copies is not None:
        copies = _list(copies)
        if len(copies) != count:
            raise ValueError(f"copies must be of the state's length {count}")
    if keep is not None:
        keep = list(keep)
        if len(keep) != count:
            raise ValueError(f"keep must be of the state's length {count}")
    table, decay = state._table, weight_decay
    if type(decay) not in (float, int):
        table, decay = table.copy(), None
        table.view(np.float64)[:, _DECAY] = weight_decay
    d_lr = _scalar("lr", lr, torch.float32, dev) if torch.is_tensor(lr) else 0
    d_step = _scalar("step", step, torch.int64, dev) if torch.is_tensor(step) else 0
    d_scale = 0 if grad_scale is None else _scalar("grad_scale", grad_scale, torch.float32, dev)
    desc = _DESC.pack(int(wt == torch.bfloat16), int(gt == torch.bfloat16), state.bits, 0.0 if d_lr else lr, betas[0], betas[1], eps,
                      0 if d_step else int(step), d_lr, d_step, d_scale)
    lists = (weights, grads, None if out is None else new, copies, keep)
    with _stream_of(stream, dev) if dev.type == "cuda" else contextlib.nullcontext(0) as sp:
        got = _native().adamw(lists, (wt, gt), dev.index if dev.type == "cuda" else -1, state._dims, table, decay,
                              state.elements, (*state._buffers(), *state_out._buffers()), desc, _entry("pp_adamw_step"), sp)
    if got:
        if got >= 10:
            for s in (state, state_out):
                s.buffers()
            for name, t, dt in zip(_NAMES, lists, (wt, gt, wt, torch.bfloat16)):
                if t is not None:
                    _fit(name, t, dt, dev, shapes)
            for k, shape, n in zip(keep or (), shapes, state.sizes):
                if k is not None and (len(shape) < 2 or k.dtype != torch.int16 or k.shape != shape[:2] or n != 9 * k.numel() or
                                      not k.is_contiguous() or k.device != dev):
                    raise ValueError("keep must be contiguous int16 [c_out][c_in] of a 3x3 layer's weights, on their device")
            raise ValueError("the tensors must be on a GPU")
        if got > 0:
            raise ValueError(_OWN[got])
        _check(got, "pp_adamw_step")
    return (new[0], state_out) if single else (new, state_out)


def grad_norm(grads, max_norm=None, stream=None):
    """pp_grad_norm: (norm, scale) of a list of gradients (or one), float32 or
    bfloat16 and contiguous: the square root of the sum of all squares, and the
    factor that brings it to ``max_norm`` at most (1 if None; NaN where a gradient
    is not finite), for adamw_step's ``grad_scale``.  Both stay on the GPU."""
    torch = _torch()
    grads = _list(grads)
    if not grads:
        raise ValueError("grads is empty")
    dt, dev = grads[0].dtype, grads[0].device
    if dt not in (torch.float32, torch.bfloat16):
        raise TypeError(f"grads must be float32 or bfloat16, got {dt}")
    most = math.inf if max_norm is None else float(max_norm)
    if not most > 0:
        raise ValueError(f"max_norm must be above 0, got {max_norm}")
    if dev.type == "cuda":
        native = _native()
        with _stream_of(stream, dev) as sp, _on(stream, dev):
            got = native.grad_norm(grads, dt, dev.index, most, _entry("pp_grad_norm_workspace"), _entry("pp_grad_norm"), sp)
        if type(got) is tuple:
            return got
        if got < 0:
            _check(got, "pp_grad_norm")
    _fit("grads", grads, dt, dev)
    raise ValueError("the tensors must be on a GPU")
