"""Refusals of the training operators, on the host before any device work:
bad descriptions, pointers, sizes and tensors."""
import ctypes

import numpy as np
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from paper_2004_11250_amd import train   # noqa: E402

A = 1 << 20   # an address that is never used: every call here is refused


@pytest.fixture(scope="module")
def lib():
    return pp.load_library()


def desc(**kw):
    d = dict(dtype=pp.PP_F32, reduction=train.PP_MEAN, n=4, d=8, hw=1, v=5, x_sn=8, x_sc=1, x_sp=8, dx_sn=8, dx_sc=1,
             dx_sp=8, w_ld=8, ignore_index=-100)
    d.update(kw)
    return train.XentDesc(**d)


def test_xent_descriptions(lib):
    nb = ctypes.c_size_t(0)
    ok = lib.pp_xent_workspace(ctypes.byref(desc()), 3, ctypes.byref(nb))
    assert ok == pp.PP_OK and nb.value > 0
    for bad in (dict(dtype=7), dict(reduction=3), dict(n=-1), dict(hw=-1), dict(d=0), dict(v=0), dict(w_ld=7), dict(x_sn=-1),
                dict(x_sc=-1), dict(dx_sp=-2)):
        assert lib.pp_xent_workspace(ctypes.byref(desc(**bad)), 3, ctypes.byref(nb)) == pp.PP_EINVAL, bad
    for bad in (dict(d=1 << 22, w_ld=1 << 22), dict(v=1 << 22), dict(n=1 << 22), dict(n=1 << 11, hw=1 << 11), dict(n=1 << 40),
                dict(n=1 << 20, d=1 << 17, w_ld=1 << 17)):
        assert lib.pp_xent_workspace(ctypes.byref(desc(**bad)), 3, ctypes.byref(nb)) == pp.PP_EUNSUPPORTED, bad
    for parts in (0, 4, -1):
        assert lib.pp_xent_workspace(ctypes.byref(desc()), parts, ctypes.byref(nb)) == pp.PP_EINVAL
    assert lib.pp_xent_workspace(None, 3, ctypes.byref(nb)) == pp.PP_EINVAL
    assert lib.pp_xent_workspace(ctypes.byref(desc()), 3, None) == pp.PP_EINVAL
    assert lib.pp_xent_workspace(ctypes.byref(desc(n=0)), 3, ctypes.byref(nb)) == pp.PP_OK and nb.value == 0


def test_xent_workspace_is_bounded(lib):
    # what it holds of tokens times classes stays below 0.6 GB; the rest goes with the inputs
    for t, v in ((1 << 13, 50000), (1 << 20, 1 << 20), (1 << 16, 1 << 21), (1 << 21, 1 << 14)):
        for dt in (pp.PP_F32, pp.PP_BF16):
            nb = ctypes.c_size_t(0)
            d = desc(dtype=dt, n=t, d=64, v=v, w_ld=64, x_sn=64, x_sp=64)
            assert lib.pp_xent_workspace(ctypes.byref(d), 3, ctypes.byref(nb)) == pp.PP_OK
            inputs = 64 * (t + v) * (6 if dt == pp.PP_F32 else 2)
            sums = 4 * 64 * (t + max(t, v)) * 64          # partial sums of the products
            assert nb.value <= inputs + sums + 700e6 + 64 * (t + v), (t, v, nb.value)


def test_xent_calls(lib):
    d = desc()
    big = 1 << 30
    fwd = lambda *a: lib.pp_xent_fwd(ctypes.byref(d), *a)   # noqa: E731
    good = [A, A, A, A, A, A, A, A, big, None]              # x w bias class_weight target loss stats workspace bytes stream
    for i, st in ((0, "x"), (1, "w"), (4, "target"), (5, "loss"), (6, "stats"), (7, "workspace")):
        a = list(good)
        a[i] = None
        assert fwd(*a) == pp.PP_EINVAL, st
    for i, off in ((0, 2), (1, 1), (2, 2), (3, 1), (4, 4), (5, 2), (6, 3), (7, 128)):
        a = list(good)
        a[i] = A + off
        assert fwd(*a) == pp.PP_EINVAL, (i, off)
    a = list(good)
    a[8] = 100
    assert fwd(*a) == pp.PP_ESIZE
    assert b"workspace" in lib.pp_last_error()
    assert lib.pp_xent_fwd(None, *good) == pp.PP_EINVAL
    bwd = [A, A, A, A, A, A, A, A, A, A, A, big, None]       # x w bias cw target stats grad dx dw db ws bytes stream
    for i in (0, 1, 4, 5, 10):
        a = list(bwd)
        a[i] = None
        assert lib.pp_xent_bwd(ctypes.byref(d), *a) == pp.PP_EINVAL, i
    for i in (6, 7, 8, 9):
        a = list(bwd)
        a[i] = A + 2
        assert lib.pp_xent_bwd(ctypes.byref(d), *a) == pp.PP_EINVAL, i
    a = list(bwd)
    a[11] = 0
    assert lib.pp_xent_bwd(ctypes.byref(d), *a) == pp.PP_ESIZE


def mats(*shapes, **kw):
    arr = (train.OrthoMat * len(shapes))()
    for e, (r, c) in zip(arr, shapes):
        e.rows, e.cols, e.u, e.u_rs, e.u_cs, e.o, e.o_rs, e.o_cs = r, c, A, c, 1, A, c, 1
        for k, v in kw.items():
            setattr(e, k, v)
    return arr


def ortho(lib, arr, n, dtype=pp.PP_F32, steps=5, coeffs=train.COEFFS, eps=1e-7, ws=A, nb=1 << 40):
    return lib.pp_ortho(arr, n, dtype, steps, (ctypes.c_float * 3)(*coeffs), eps, ws, nb, None)


def test_ortho_refusals(lib):
    nb = ctypes.c_size_t(0)
    one = mats((80, 90))
    assert lib.pp_ortho_workspace(one, 1, pp.PP_F32, ctypes.byref(nb)) == pp.PP_OK and nb.value > 0
    assert lib.pp_ortho_workspace(mats((0, 9), (4, 0)), 2, pp.PP_F32, ctypes.byref(nb)) == pp.PP_OK and nb.value == 0
    assert lib.pp_ortho_workspace(one, 1, 5, ctypes.byref(nb)) == pp.PP_EINVAL
    assert lib.pp_ortho_workspace(None, 1, pp.PP_F32, ctypes.byref(nb)) == pp.PP_EINVAL
    assert lib.pp_ortho_workspace(one, -1, pp.PP_F32, ctypes.byref(nb)) == pp.PP_EINVAL
    assert lib.pp_ortho_workspace(one, 1, pp.PP_F32, None) == pp.PP_EINVAL
    for shape in ((-1, 4), (4, -1)):
        assert ortho(lib, mats(shape), 1) == pp.PP_EINVAL
    for shape in ((1 << 22, 4), (4, 1 << 22), (40000, 40000), (1 << 20, 4096)):
        assert ortho(lib, mats(shape), 1) == pp.PP_EUNSUPPORTED, shape
    for kw in (dict(u=None), dict(o=None), dict(u=A + 2), dict(o=A + 1), dict(u_rs=-90), dict(o_cs=-1)):
        assert ortho(lib, mats((80, 90), **kw), 1) == pp.PP_EINVAL, kw
    for kw in (dict(dtype=9), dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=float("nan")), dict(ws=None), dict(ws=A + 8),
               dict(coeffs=(float("inf"), 0, 0))):
        assert ortho(lib, one, 1, **kw) == pp.PP_EINVAL, kw
    assert ortho(lib, one, 1, nb=1000) == pp.PP_ESIZE
    # polynomials that leave the range
    for coeffs in ((9.0, 0.0, 0.0), (3.0, -1.0, 1.0), (100.0, -300.0, 201.0)):
        assert ortho(lib, one, 1, coeffs=coeffs) == pp.PP_EUNSUPPORTED, coeffs
    # nothing to do is not an error, whatever the workspace
    assert ortho(lib, mats((0, 9)), 1, ws=None, nb=0) == pp.PP_OK and ortho(lib, None, 0, ws=None, nb=0) == pp.PP_OK


def test_muon_refusals(lib):
    def layer(**kw):
        arr = (train.MuonLayer * 1)()
        e = arr[0]
        e.rows, e.cols = 16, 90
        e.w = e.g = e.momentum = e.w_out = e.momentum_out = e.keep = A
        for k, v in kw.items():
            setattr(e, k, v)
        return arr

    def step(arr, dtype=pp.PP_F32, **kw):
        v = dict(lr=0.1, momentum=0.9, weight_decay=0.0, nesterov=1, steps=5, coeffs=(ctypes.c_float * 3)(*train.COEFFS), eps=1e-7)
        v.update(kw)
        return lib.pp_muon_step(arr, 1, dtype, ctypes.byref(train.MuonDesc(**v)), A, 0, None)

    assert step(layer(rows=200)) == pp.PP_ESIZE            # (well formed, but for the workspace)
    for kw in (dict(w=None), dict(g=None), dict(momentum=None), dict(w_out=None), dict(momentum_out=None), dict(w=A + 2),
               dict(momentum=A + 2), dict(keep=A + 1), dict(cols=91), dict(rows=-1)):
        assert step(layer(**kw)) == pp.PP_EINVAL, kw
    for kw in (dict(lr=float("nan")), dict(momentum=float("inf")), dict(weight_decay=float("nan")), dict(steps=0)):
        assert step(layer(), **kw) == pp.PP_EINVAL, kw
    assert step(layer(), dtype=3) == pp.PP_EINVAL
    assert lib.pp_muon_step(layer(), 1, pp.PP_F32, None, A, 1 << 30, None) == pp.PP_EINVAL


def test_binding_refuses_tensors():
    x, w, t = torch.zeros(4, 8), torch.zeros(5, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        pp.linear_xent_fwd(x, w, t)
    for args, kw in (((x, w, t), dict(reduction="max")), ((x[0], w, t), {}), ((x, w[0], t), {}), ((x, w[:, :7], t), {}),
                     ((x, w, t[:3]), {}), ((x, w, t.int()), {}), ((x, w, t), dict(bias=torch.zeros(4))),
                     ((x, w, t), dict(bias=torch.zeros(5, dtype=torch.float64))), ((x, w, t), dict(class_weight=torch.zeros(6))),
                     ((x, torch.zeros(5, 16)[:, ::2], t), {}), ((x, torch.zeros(5, 8, 3, 3), t), {}),
                     ((torch.zeros(2, 8, 4, 6).transpose(2, 3), w, torch.zeros(2, 6, 4, dtype=torch.int64)), {}),
                     ((torch.zeros(2, 8, 4, 6)[:, :, :, :5], w, torch.zeros(2, 4, 5, dtype=torch.int64)), {})):
        with pytest.raises(ValueError):
            pp.linear_xent_fwd(*args, **kw)
    with pytest.raises(TypeError):
        pp.linear_xent_fwd(x.double(), w.double(), t)
    with pytest.raises(TypeError):
        pp.linear_xent_fwd(x, w.bfloat16(), t)
    u = torch.zeros(4, 6)
    with pytest.raises(ValueError, match="GPU"):
        pp.orthogonalize(u)
    for args, kw in (([u, u.bfloat16()], {}), ([], {}), ([torch.zeros(4)], {}), ([torch.zeros(4, 3, 5).transpose(1, 2)[:, ::2]], {}),
                     ([u], dict(coeffs=(1.0, 2.0))), ([u], dict(out=[torch.zeros(4, 5)])), ([u], dict(out=[]))):
        with pytest.raises(ValueError):
            pp.orthogonalize(args, **kw)
    w, g, m = torch.zeros(4, 2, 3, 3), torch.zeros(4, 2, 3, 3), torch.zeros(4, 2, 3, 3)
    k = torch.zeros(4, 2, dtype=torch.int16)
    with pytest.raises(ValueError, match="GPU"):
        pp.muon_step(w, g, m, lr=0.1, keep=k)
    for a in ((w, g[:3], m, k), (w, g.bfloat16(), m, k), (w, g, m.double(), k), (w, g, m, k[:3]), (w, g, m, k.int()),
              (w, g.transpose(2, 3), m, k), (w[..., 0], g[..., 0], m[..., 0], k)):
        with pytest.raises(ValueError):
            pp.muon_step(*a[:3], lr=0.1, keep=a[3])
    with pytest.raises(ValueError):
        pp.muon_step([w], [g, g], [m], lr=0.1)


def test_keep_masks():
    lib = np.array([0x03A, 0x1B0, 0x1FF])
    pid = np.array([[0, 1], [2, 9]])
    got = pp.keep_masks(pid, np.array([[1, 1], [1, 0]]), lib)
    assert got.dtype == np.int16 and got.tolist() == [[0x03A, 0x1B0], [0x1FF, 0]]
    with pytest.raises(ValueError):
        pp.keep_masks(pid, np.ones((2, 2)), lib)
    with pytest.raises(ValueError):
        pp.keep_masks(pid[0], np.ones(2), lib)
