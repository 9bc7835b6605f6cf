"""Refusals of the embedding and AdamW calls, on the host before any device work."""
import ctypes
import math

import numpy as np
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from paper_2004_11250_amd import adamw, embed   # noqa: E402

A = 1 << 20   # an address that is never used: every call here is refused


@pytest.fixture(scope="module")
def lib():
    return pp.load_library()


class EmbedDesc(ctypes.Structure):
    _fields_ = [("w_dtype", ctypes.c_int32), ("y_dtype", ctypes.c_int32), ("t", ctypes.c_int64), ("v", ctypes.c_int64),
                ("d", ctypes.c_int64), ("w_ld", ctypes.c_int64), ("y_ld", ctypes.c_int64), ("ignore_index", ctypes.c_int64),
                ("scale", ctypes.c_float)]


def desc(**kw):
    d = dict(w_dtype=0, y_dtype=0, t=100, v=7, d=8, w_ld=8, y_ld=8, ignore_index=-100, scale=1.0)
    d.update(kw)
    return EmbedDesc(**d)


def test_embed_descriptions(lib):
    nb = ctypes.c_size_t(0)
    assert lib.pp_embed_workspace(ctypes.byref(desc()), ctypes.byref(nb)) == pp.PP_OK and nb.value >= 4 * 107
    for bad in (dict(w_dtype=2), dict(y_dtype=-1), dict(t=-1), dict(v=0), dict(d=0), dict(w_ld=7), dict(y_ld=7)):
        assert lib.pp_embed_workspace(ctypes.byref(desc(**bad)), ctypes.byref(nb)) == pp.PP_EINVAL, bad
        assert lib.pp_embed_fwd(ctypes.byref(desc(**bad)), A, A, A, None) == pp.PP_EINVAL, bad
    for bad in (dict(t=1 << 30), dict(v=1 << 30), dict(d=1 << 23, w_ld=1 << 23, y_ld=1 << 23), dict(w_ld=1 << 32), dict(y_ld=1 << 32)):
        assert lib.pp_embed_workspace(ctypes.byref(desc(**bad)), ctypes.byref(nb)) == pp.PP_EUNSUPPORTED, bad
        assert lib.pp_embed_bwd(ctypes.byref(desc(**bad)), A, A, None, A, A, 1 << 50, None) == pp.PP_EUNSUPPORTED, bad
    # launches of 2^32 threads or more: 256 a row of 1025 features and above
    long = dict(d=2000, w_ld=2000, y_ld=2000)
    assert lib.pp_embed_fwd(ctypes.byref(desc(t=1 << 24, **long)), A, A, A, None) == pp.PP_EUNSUPPORTED
    assert lib.pp_embed_workspace(ctypes.byref(desc(t=1 << 24, **long)), ctypes.byref(nb)) == pp.PP_OK
    assert lib.pp_embed_workspace(ctypes.byref(desc(v=(1 << 26) - 4200, **long)), ctypes.byref(nb)) == pp.PP_OK
    assert lib.pp_embed_workspace(ctypes.byref(desc(v=1 << 26, **long)), ctypes.byref(nb)) == pp.PP_EUNSUPPORTED
    assert lib.pp_embed_bwd(ctypes.byref(desc(v=1 << 26, **long)), A, A, None, A, A, 1 << 50, None) == pp.PP_EUNSUPPORTED
    assert lib.pp_embed_workspace(None, ctypes.byref(nb)) == pp.PP_EINVAL
    assert lib.pp_embed_workspace(ctypes.byref(desc()), None) == pp.PP_EINVAL
    # the workspace goes with the tokens and the rows, not with their product with d
    for t, v, d in ((1 << 20, 1 << 20, 4096), (1 << 29, 7, 64), (33, 5, 1 << 20)):
        assert lib.pp_embed_workspace(ctypes.byref(desc(t=t, v=v, d=d, w_ld=d, y_ld=d)), ctypes.byref(nb)) == pp.PP_OK
        assert nb.value <= 8 * v + 16 * t + 2048 * 4 * (d + 8) + 4 * 256 * 128 + 4 * 128 * 1024 + 4 * 4096


def test_rows_of_a_gradient_are_limited_as_pp_h_says(lib):
    nb = ctypes.c_size_t(0)
    status = lambda v, d: lib.pp_embed_workspace(ctypes.byref(desc(v=v, d=d, w_ld=d, y_ld=d)), ctypes.byref(nb))   # noqa: E731
    for d, most in ((129, 29), (256, 29), (257, 28), (512, 28), (513, 27), (1024, 27), (1025, 26), (5000, 26)):
        assert status((1 << most) - (1 << most - 13), d) == pp.PP_OK, d          # (1024 of the 2^24 workgroups are left to the tokens)
        assert status(1 << most, d) == pp.PP_EUNSUPPORTED, d
    for d in (1, 8, 32, 64, 128):
        assert status((1 << 30) - 1, d) == (pp.PP_OK if d <= 64 else pp.PP_EUNSUPPORTED), d
        assert status((1 << 30) - (1 << 17), d) == pp.PP_OK, d


def test_embed_calls(lib):
    d = ctypes.byref(desc())
    for i in range(3):
        a = [A, A, A]
        a[i] = None
        assert lib.pp_embed_fwd(d, *a, None) == pp.PP_EINVAL
        a[i] = A + 2
        assert lib.pp_embed_fwd(d, *a, None) == pp.PP_EINVAL
    good = [A, A, A, A, A, 1 << 30, None]      # ids dy add dw workspace bytes stream
    for i in (0, 1, 3, 4):
        a = list(good)
        a[i] = None
        assert lib.pp_embed_bwd(d, *a) == pp.PP_EINVAL, i
    for i, by in ((0, 4), (1, 2), (2, 1), (3, 2), (4, 128)):
        a = list(good)
        a[i] = A + by
        assert lib.pp_embed_bwd(d, *a) == pp.PP_EINVAL, i
    a = list(good)
    a[5] = 300
    assert lib.pp_embed_bwd(d, *a) == pp.PP_ESIZE and b"workspace" in lib.pp_last_error()
    assert lib.pp_embed_fwd(None, A, A, A, None) == pp.PP_EINVAL
    # no token: nothing to look up
    assert lib.pp_embed_fwd(ctypes.byref(desc(t=0)), None, None, None, None) == pp.PP_OK


TENSOR = np.dtype([("n", "i8"), ("w", "u8"), ("g", "u8"), ("w_out", "u8"), ("copy", "u8"), ("keep", "u8"), ("at", "i8"),
                   ("weight_decay", "f8")])
GRAD = np.dtype([("g", "u8"), ("n", "i8")])


class AdamWDesc(ctypes.Structure):
    _fields_ = [("w_dtype", ctypes.c_int32), ("g_dtype", ctypes.c_int32), ("bits", ctypes.c_int32), ("lr", ctypes.c_double),
                ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("step", ctypes.c_int64),
                ("d_lr", ctypes.c_void_p), ("d_step", ctypes.c_void_p), ("d_grad_scale", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("m_out", ctypes.c_void_p), ("v_out", ctypes.c_void_p), ("m_scale_out", ctypes.c_void_p),
                ("v_scale_out", ctypes.c_void_p)]


def test_layouts():
    assert ctypes.sizeof(EmbedDesc) == embed._DESC.size and ctypes.sizeof(AdamWDesc) == adamw._DESC.size
    assert TENSOR.itemsize == 8 * len(adamw._TENSOR)
    assert TENSOR.names == adamw._TENSOR


def table(count=1, **kw):
    t = np.zeros(count, TENSOR)
    t["n"], t["w"], t["g"], t["w_out"] = 100, A, A, A
    for k, v in kw.items():
        t[k] = v
    return t


def step(lib, t, count=None, **kw):
    d = AdamWDesc(w_dtype=0, g_dtype=0, bits=32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, m=A, v=A, m_out=A, v_out=A,
                  m_scale=A, v_scale=A, m_scale_out=A, v_scale_out=A)
    for k, v in kw.items():
        setattr(d, k, v)
    return lib.pp_adamw_step(None if t is None else t.ctypes.data, len(t) if count is None else count, ctypes.byref(d), None)


def test_adamw_calls(lib):
    for kw in (dict(n=-1), dict(at=-128), dict(at=64), dict(w=0), dict(g=0), dict(w_out=0), dict(w=A + 2), dict(g=A + 1), dict(w_out=A + 2),
               dict(copy=A + 1), dict(keep=A + 1), dict(keep=A), dict(weight_decay=math.nan), dict(weight_decay=math.inf)):
        assert step(lib, table(2, **kw)) == pp.PP_EINVAL, kw
    for kw in (dict(n=1 << 34), dict(at=1 << 40)):
        assert step(lib, table(**kw)) == pp.PP_EUNSUPPORTED, kw
    for kw in (dict(w_dtype=2), dict(g_dtype=-1), dict(bits=16), dict(bits=0), dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0),
               dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=-1.0), dict(eps=math.inf), dict(step=0), dict(step=-3),
               dict(d_lr=A + 2), dict(d_step=A + 4), dict(d_grad_scale=A + 1), dict(m=None), dict(v=A + 8), dict(m_out=None),
               dict(v_out=A + 4), dict(bits=8, m_scale=None), dict(bits=8, v_scale_out=A + 2)):
        assert step(lib, table(), **kw) == pp.PP_EINVAL, kw
    assert step(lib, None, count=1) == pp.PP_EINVAL and step(lib, table(), count=-1) == pp.PP_EINVAL
    assert lib.pp_adamw_step(table().ctypes.data, 1, None, None) == pp.PP_EINVAL
    # nothing to do is no error
    assert step(lib, table(3, n=0, w=0, g=0, w_out=0), m=None, v=None) == pp.PP_OK and step(lib, None, count=0) == pp.PP_OK


def test_values_calls(lib):
    good = [A, A, A, A, 256, 0, A, A, None]
    for i, bad in ((0, None), (1, None), (2, None), (3, None), (0, A + 8), (3, A + 2), (4, -128), (4, 100), (5, 2), (6, A + 8), (7, A + 2)):
        a = list(good)
        a[i] = bad
        assert lib.pp_adamw_values(*a) == pp.PP_EINVAL, (i, bad)
    a = list(good)
    a[4] = 1 << 40
    assert lib.pp_adamw_values(*a) == pp.PP_EUNSUPPORTED
    assert lib.pp_adamw_values(None, None, None, None, 0, 0, None, None, None) == pp.PP_OK
    assert lib.pp_adamw_values(A, A, A, A, 128, 0, None, None, None) == pp.PP_OK


def test_norm_calls(lib):
    t = np.zeros(2, GRAD)
    t["g"], t["n"] = A, 1000
    nb = ctypes.c_size_t(0)
    assert lib.pp_grad_norm_workspace(t.ctypes.data, 2, 0, ctypes.byref(nb)) == pp.PP_OK and nb.value >= 16
    assert lib.pp_grad_norm_workspace(t.ctypes.data, 2, 0, None) == pp.PP_EINVAL
    assert lib.pp_grad_norm_workspace(None, 2, 0, ctypes.byref(nb)) == pp.PP_EINVAL
    norm = lambda t=t, n=2, dt=0, most=1.0, out=A, ws=A, b=1 << 20: lib.pp_grad_norm(   # noqa: E731
        t.ctypes.data, n, dt, most, out, ws, b, None)
    for kw in (dict(n=-1), dict(dt=5), dict(most=0.0), dict(most=-1.0), dict(most=math.nan), dict(out=None), dict(out=A + 2), dict(ws=None),
               dict(ws=A + 8)):
        assert norm(**kw) == pp.PP_EINVAL, kw
    assert norm(b=8) == pp.PP_ESIZE
    for k, v, want in (("g", 0, pp.PP_EINVAL), ("g", A + 2, pp.PP_EINVAL), ("n", -1, pp.PP_EINVAL), ("n", 1 << 34, pp.PP_EUNSUPPORTED)):
        bad = t.copy()
        bad[k][1] = v
        assert norm(t=bad) == want, k


# the binding: tensors here are on the CPU, so a well-formed call is refused last, for that

def refused(match, kind=ValueError):
    return pytest.raises(kind, match=match)


def test_state():
    s = pp.AdamWState([(3, 5), (0,), (200,), ()], bits=8, device="cpu")
    assert s.places == [0, 128, 128, 384] and s.elements == 512 and [len(t) for t in s.buffers()] == [512, 512, 4, 4]
    assert [tuple(t.shape) for t in s.split(s.v)] == [(3, 5), (0,), (200,), ()]
    assert not any(t.view(torch.uint8).any() for t in s.buffers())
    with refused("bits"):
        pp.AdamWState([(3,)], bits=16, device="cpu")
    with refused("empty"):
        pp.AdamWState([])
    with refused("GPU"):
        s.values()
    with refused("dtype", TypeError):
        s.values(torch.float16)
    s.v = torch.zeros(511, dtype=torch.uint8)
    with refused("buffers"):
        s.buffers()


def test_adamw_tensors():
    w, g = [torch.zeros(4, 6), torch.zeros(9)], [torch.zeros(4, 6), torch.zeros(9)]
    s = pp.AdamWState(w)
    go = lambda w=w, g=g, s=s, lr=1e-3, step=1, **kw: pp.adamw_step(w, g, s, lr=lr, step=step, **kw)   # noqa: E731
    with refused("GPU"):
        go()
    with refused("length"):
        go(w=w[:1])
    with refused("length"):
        go(g=g + g)
    with refused("shapes"):
        go(w=[torch.zeros(6, 4), w[1]])
    with refused("contiguous"):
        go(g=[torch.zeros(6, 4).t(), g[1]])
    with refused("contiguous"):
        go(g=[g[0], g[1].bfloat16()])
    with refused("must be float32 or bfloat16", TypeError):
        go(g=[t.double() for t in g])
    with refused("one device"):
        go(w=[t.to("meta") for t in w])
    with refused("same tensor"):
        go(w=[w[0], w[1]], s=pp.AdamWState(w), out=([w[0], w[0].view(-1)[:9]], pp.AdamWState(w)))
    with refused("another tensor"):
        go(out=([g[0], w[1]], s))
    with refused("another tensor's input"):
        go(w=[w[0], w[0].view(-1)[:9]], out=([w[0], torch.zeros(9)], s))
    with refused("same shapes and bits"):
        go(out=(w, pp.AdamWState(w, bits=8)))
    with refused("copies"):
        go(copies=[torch.zeros(4, 6), torch.zeros(9)])
    with refused("length"):
        go(copies=[torch.zeros(4, 6, dtype=torch.bfloat16)])
    with refused("GPU"):
        go(copies=[torch.zeros(4, 6, dtype=torch.bfloat16), torch.zeros(9, dtype=torch.bfloat16)])
    for name, bad in (("lr", torch.zeros(2)), ("lr", torch.zeros(1, dtype=torch.float64)), ("step", torch.zeros(1)),
                      ("grad_scale", torch.zeros(1, dtype=torch.int64))):
        with refused(name):
            go(**{name: bad})
    with refused("keep"):
        go(keep=[torch.zeros(4, 6, dtype=torch.int16), None])
    with refused("length"):
        go(keep=[None])
    layer = torch.zeros(2, 3, 3, 3)
    pruned = lambda keep: pp.adamw_step(layer, layer.clone(), pp.AdamWState(layer), lr=1e-3, step=1, keep=keep)   # noqa: E731
    with refused("GPU"):
        pruned(torch.zeros(2, 3, dtype=torch.int16))
    for bad in (torch.zeros(2, 3), torch.zeros(3, 2, dtype=torch.int16), torch.zeros(3, 2, dtype=torch.int16).t(), torch.zeros(6, dtype=torch.int16)):
        with refused("keep"):
            pruned(bad)


def test_a_state_is_copied_whole():
    import copy
    import gc
    import io
    w = [torch.zeros(3, 4), torch.zeros(5)]

    def saved(state):
        at = io.BytesIO()
        torch.save(state, at)
        return torch.load(io.BytesIO(at.getvalue()), weights_only=False)

    for again in (copy.deepcopy, saved):
        state = pp.AdamWState([t.shape for t in w], bits=8, device="cpu")
        new = again(state)
        state._dims[:], state._table[:] = -7, -7        # (nothing of the first is looked at any more)
        del state
        gc.collect()
        with refused("GPU"):
            pp.adamw_step(w, [t.clone() for t in w], new, lr=1e-3, step=1)
        with refused("shapes"):
            pp.adamw_step(w[::-1], [t.clone() for t in w], new, lr=1e-3, step=1)


def test_norm_tensors():
    with refused("empty"):
        pp.grad_norm([])
    with refused("float32 or bfloat16", TypeError):
        pp.grad_norm([torch.zeros(3, dtype=torch.float16)])
    with refused("contiguous"):
        pp.grad_norm([torch.zeros(3, 4).t()])
    with refused("contiguous"):
        pp.grad_norm([torch.zeros(3), torch.zeros(3).bfloat16()])
    with refused("max_norm"):
        pp.grad_norm([torch.zeros(3)], max_norm=0.0)
    with refused("GPU"):
        pp.grad_norm(torch.zeros(3))


def test_embed_tensors():
    ids, w = torch.zeros(5, dtype=torch.int64), torch.zeros(7, 4)
    with refused("GPU"):
        pp.embed_fwd(ids, w)
    with refused("int64"):
        pp.embed_fwd(ids.int(), w)
    with refused("int64"):
        pp.embed_fwd(torch.zeros(5, 2, dtype=torch.int64)[:, 0], w)
    with refused("v, d"):
        pp.embed_fwd(ids, torch.zeros(7))
    with refused("float32 or bfloat16", TypeError):
        pp.embed_fwd(ids, w.half())
    with refused("int64"):
        pp.embed_bwd(ids.float(), torch.zeros(5, 4), 7)
    with refused("GPU"):
        pp.embed_bwd(ids, torch.zeros(5, 4), 7)
    # (row layouts, as the calls check them)
    rows = lambda t, shape: embed._rows(t, "x", shape, t.device)   # noqa: E731
    assert rows(torch.zeros(5, 9)[:, 2:6], (5, 4)) == 9 and rows(torch.zeros(2, 3, 4), (2, 3, 4)) == 4
    assert rows(torch.zeros(4), (4,)) == 4 and rows(torch.zeros(1, 1, 4), (1, 1, 4)) == 4 and rows(torch.zeros(3, 1), (3, 1)) == 1
    for t, shape in ((torch.zeros(4, 5).t(), (5, 4)), (torch.zeros(2, 3, 4).transpose(0, 1), (3, 2, 4)), (torch.zeros(1, 4).expand(5, 4), (5, 4)),
                     (torch.zeros(5, 4), (5, 3)), (torch.zeros(9).as_strided((5, 4), (1, 1)), (5, 4))):
        with pytest.raises(ValueError):
            rows(t, shape)


# the binding's native module for lists

def test_outputs_of_their_own():
    x = [torch.zeros(4) for _ in range(8)]
    table, dims = np.zeros((2, 8), np.int64), np.array([1, 4] * 2, np.int64)
    desc = AdamWDesc(bits=32)
    moments = [torch.zeros(256) for _ in range(2)]

    def code(w, g, new=None, copies=None, n=(4, 4)):
        """Of two tensors: indices into x."""
        table[:, 0] = n
        pick = lambda t, dt=torch.float32: None if t is None else [x[i].view(dt)[:4] for i in t]   # noqa: E731
        return adamw._native().adamw((pick(w), pick(g), pick(new), pick(copies, torch.bfloat16), None), (torch.float32, torch.float32), -1, dims,
                                     table, None, 256, (*moments, None, None) * 2, bytes(desc), 1, 0)

    assert code((0, 1), (2, 2)) == 30 and code((0, 1), (2, 3), (4, 5)) == 30 and code((0, 1), (2, 3), None, (4, 5)) == 30
    assert code((0, 0), (2, 3)) == 1 and code((0, 0), (2, 3), n=(4, 0)) == 30
    assert code((0, 1), (2, 3), (0, 0)) == 1 and code((0, 1), (2, 3), None, (0, 4)) == 1
    assert code((0, 1), (0, 3)) == 2 and code((0, 1), (2, 3), (4, 2)) == 2 and code((0, 1), (2, 3), None, (4, 3)) == 2
    assert code((0, 1), (2, 3), (1, 4)) == 3 and code((0, 1), (2, 3), (4, 5), (0, 6)) == 3


def test_native_calls_take_tensors_on_a_gpu_only():
    lists, f32 = adamw._native(), torch.float32
    t, dims = np.zeros((2, 8), np.int64), np.array([1, 3, 1, 3], np.int64)
    x = [torch.zeros(3), torch.zeros(3)]
    bufs, desc = [torch.zeros(256), torch.zeros(256), None, None], bytes(AdamWDesc(bits=32))
    go = lambda w=x, g=x, new=None, copies=None, keep=None, dt=(f32, f32), at=-1, b=bufs, d=desc, n=256, rows=None, sizes=None: lists.adamw(   # noqa: E731
        (w, g, new, copies, keep), dt, at, dims if sizes is None else sizes, t if rows is None else rows, 0.5, n, (*b, *b), d, 1, 0)
    assert go() == 30 and not t.any()
    assert go(at=0) == 20 and go(n=128) == 20 and go(b=bufs[:3] + bufs[:1]) == 20 and go(d=bytes(AdamWDesc(bits=8))) == 20
    assert go(b=[torch.zeros(256).bfloat16(), *bufs[1:]]) == 20 and go(b=[torch.zeros(512)[::2], *bufs[1:]]) == 20
    assert go(w=[None, None]) == 10 and go(w=["a", 3]) == 10 and go(g=[x[0], x[1].double()]) == 11 and go(new=[x[0], torch.zeros(4)]) == 12
    assert go(copies=x) == 13 and go(keep=[None, torch.zeros(1, 1, dtype=torch.int16)]) == 14 and go(keep=[None, None]) == 30
    for bad in (dict(w=None), dict(g=x[:1]), dict(new=x[:1]), dict(copies=(1, 2)), dict(keep=[None]), dict(dt=("f", f32)), dict(dt=f32), dict(b=bufs[:3]),
                dict(d=desc[1:]), dict(d="x"), dict(n=0.5), dict(rows=t[:1]), dict(rows=3), dict(sizes=dims[:3]), dict(sizes=dims[1:]),
                dict(sizes="x")):
        with pytest.raises(TypeError):
            go(**bad)
    assert lists.grad_norm(x, f32, 0, 1.0, 1, 1, 0) == 10 and lists.grad_norm([3], f32, 0, 1.0, 1, 1, 0) == 10
    for bad in ((), (x, f32, 0, 1.0, 1, 1), (tuple(x), f32, 0, 1.0, 1, 1, 0), (x, "f", 0, 1.0, 1, 1, 0), (x, f32, "0", 1.0, 1, 1, 0)):
        with pytest.raises(TypeError):
            lists.grad_norm(*bad)
    ids, w = torch.zeros(3, dtype=torch.int64), torch.zeros(2, 4)
    assert lists.embed_fwd(ids, w, None, 1.0, -100, 1, 0) is None and lists.embed_fwd([0], w, None, 1.0, -100, 1, 0) is None
    assert lists.embed_bwd(ids, torch.zeros(3, 4), 2, None, 1.0, -100, None, 1, 1, 0) is None
    for bad in ((), (ids, w, None, 1.0, -100, 1), (ids, w, None, 1.0, -100, "1", 0)):
        with pytest.raises(TypeError):
            lists.embed_fwd(*bad)
    for bad in ((), (ids, w, 2, None, 1.0, -100, None, 1, 1), (ids, w, 2, None, 1.0, -100, None, 1, 1, "0")):
        with pytest.raises(TypeError):
            lists.embed_bwd(*bad)
