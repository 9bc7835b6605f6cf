"""Orthogonalised updates and the weight step (pp_ortho, pp_muon_step) on the GPU
against the formula in 64 bits.

Error bounds.  A step takes a singular value s to f(s) = a s + b s^3 + c s^5, so
an error made in X before a step comes out of it times at most max |f'| = a on
small singular values, where the other terms vanish (on the others |f'| is
smaller).  Each of the steps adds the roundings of its own products: with X, A
and B held to r of their norms and |A| <= 1.4, |B| <= 3, a step adds at most
(a + |b| + |c|) times about 4 r |X|, here 42 r.  After n steps the first one's
error has grown by a^(n - 1).  The bound on the error of the whole matrix
against the norm of the result is therefore
42 r (a^n - 1) / (a - 1) |X_0| / |result|, |X_0| = 1, and the result's norm is at
least that of one direction, 0.6.  It holds for any input; fp32 (three products
of fp16 pairs, fp32 sums): r = 2^-21.  For bf16, X's part that the products
drop is 2^-12 of each value; it enters through B X, |B| <= 3 on directions whose
s is near 1 and growing with s^2 below: dropped parts are independent roundings
that spread over all directions, so the matrix norms of the tests' inputs (no
direction dominates) give 2^-12 sqrt(steps) a on the result, and its own
rounding is 2^-8 of each value.
"""
import numpy as np
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
pytestmark = pytest.mark.gpu

MUON = (3.4445, -4.7750, 2.0315)
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def ref(u, steps=5, coeffs=MUON, eps=1e-7):
    x = u.double().reshape(u.shape[0], -1)
    x = x / (x.square().sum().sqrt() + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    a, b, c = coeffs
    for _ in range(steps):
        g = x @ x.t().contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    return (x.t() if tall else x).reshape(u.shape)


def limit(dtype, steps=5, a=MUON[0]):
    if dtype == "f32":
        return 42 * 2.0 ** -21 * (a ** steps - 1) / (a - 1) / 0.6
    return 2.0 ** -12 * steps ** 0.5 * a + 2.0 ** -8


def near(got, want, lim):
    got = got.double()
    assert got.shape == want.shape
    if want.numel() == 0:
        return
    off = float((got - want).norm() / want.norm())
    assert off <= lim, (off, lim)


def normal(seed, *shape, dtype="f32"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(DT[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (9, 1), (2, 3), (16, 144), (63, 65), (64, 64), (65, 64), (128, 130),
                                   (100, 1000), (777, 129), (257, 256)])
def test_one_matrix(dtype, shape):
    u = normal(1, *shape, dtype=dtype)
    o = pp.orthogonalize(u)
    assert o.dtype == u.dtype and o.is_contiguous()
    near(o, ref(u), limit(dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_tiles(dtype):
    # 128 x 128 tiles, then 256 x 256 ones, for every product
    for n in (2600, 5200):
        u = normal(2, n, n, dtype=dtype)
        near(pp.orthogonalize(u), ref(u), limit(dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_list_is_its_matrices(dtype):
    shapes = [(16, 144), (313, 256), (64, 64, 3, 3), (5, 1, 3, 3), (130, 40), (0, 5), (7, 0), (1, 300)] + [(9, 20)] * 70
    mats = [normal(10 + i, *s, dtype=dtype) for i, s in enumerate(shapes)]
    outs = pp.orthogonalize(mats)
    for u, o in zip(mats, outs):
        assert o.shape == u.shape
        near(o, ref(u) if u.numel() else u.double(), limit(dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("steps,coeffs", [(1, MUON), (2, MUON), (8, MUON), (5, (1.875, -1.25, 0.375)), (6, (1.5, -0.5, 0.0))])
def test_steps_and_coefficients(dtype, steps, coeffs):
    u = normal(3, 90, 200, dtype=dtype)
    near(pp.orthogonalize(u, steps=steps, coeffs=coeffs), ref(u, steps, coeffs), limit(dtype, steps, coeffs[0]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_low_rank_and_scales(dtype):
    # a few directions; entries tiny, huge and with one that dwarfs the rest
    u = (normal(4, 120, 4) @ normal(5, 4, 300)).to(DT[dtype])
    for scale in (1.0, 1e-20, 1e18):
        v = u * scale
        near(pp.orthogonalize(v, eps=0.0), ref(v, eps=0.0), limit(dtype))
    v = normal(6, 70, 90, dtype=dtype)
    v[3, 5] = 1e4
    near(pp.orthogonalize(v), ref(v), limit(dtype) if dtype == "f32" else 3 * limit(dtype))
    v = normal(7, 70, 90, dtype=dtype) * 1e-9      # eps counts here
    near(pp.orthogonalize(v), ref(v), limit(dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_zeros_and_what_is_not_finite(dtype):
    z = torch.zeros(40, 50, device="cuda", dtype=DT[dtype])
    assert bool((pp.orthogonalize(z) == 0).all())
    for bad in (float("nan"), float("inf")):
        u = normal(8, 40, 50, dtype=dtype)
        u[7, 9] = bad
        clean = normal(9, 40, 50, dtype=dtype)
        a, b = pp.orthogonalize([u, clean])
        assert bool(torch.isnan(a).all())
        assert torch.equal(b, pp.orthogonalize(clean))
    rows = normal(11, 40, 50, dtype=dtype)
    rows[5:20] = 0                                  # rows without anything
    o = pp.orthogonalize(rows)
    near(o, ref(rows), limit(dtype))
    assert bool((o[5:20] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_places(dtype):
    big = normal(12, 200, 300, dtype=dtype)
    views = [big[3:93, 7:210], big[::2, ::3], big.t()[5:250, 1:80], big[10:60, 20:120].t()]
    outs = pp.orthogonalize(views)
    # (the same list: which tiles a stage uses, and so the order of its sums, goes by all of them)
    for a, o in zip(pp.orthogonalize([v.contiguous() for v in views]), outs):
        assert torch.equal(o, a)
    dest = torch.zeros(200, 300, device="cuda", dtype=DT[dtype])
    alone = pp.orthogonalize(views[0])
    pp.orthogonalize([views[0]], out=[dest[3:93, 7:210]])
    assert torch.equal(dest[3:93, 7:210], alone) and int((dest != 0).sum()) <= 90 * 203
    mine = views[3].contiguous()
    alone = pp.orthogonalize(views[3])
    assert pp.orthogonalize(mine, out=mine) is mine and torch.equal(mine, alone)


def test_a_matrix_and_its_transpose():
    u = normal(13, 100, 260)
    assert torch.equal(pp.orthogonalize(u).t(), pp.orthogonalize(u.t()))


def layer(seed, c_out, c_in, dtype, pruned):
    shape = (c_out, c_in, 3, 3) if pruned else (c_out, c_in)
    w, g, m = normal(seed, *shape, dtype=dtype), normal(seed + 1, *shape, dtype=dtype), normal(seed + 2, *shape)
    kp = None
    if pruned:
        rng = np.random.default_rng(seed)
        lib = np.array([0x03A, 0x0B2, 0x0B8, 0x09A, 0x01B, 0x036, 0x0D8, 0x1B0])
        kp = pp.keep_masks(rng.integers(0, 8, (c_out, c_in)), rng.random((c_out, c_in)) < 0.5, lib)
        kp = torch.from_numpy(kp).cuda()
    return w, g, m, kp


def muon_ref(w, g, m, kp, lr=0.02, mu=0.95, nesterov=True, wd=0.01):
    on = torch.ones(w.shape, device="cuda", dtype=torch.bool)
    if kp is not None:
        on = torch.stack([(kp.long() >> t) & 1 for t in range(9)], -1).reshape(w.shape) != 0
    z = torch.zeros((), device="cuda", dtype=torch.float64)
    g, m, w = (torch.where(on, t.double(), z) for t in (g, m, w))
    m = mu * m + g
    o = ref(g + mu * m if nesterov else m)
    cols = w.numel() // w.shape[0]
    o = lr * max(1.0, w.shape[0] / cols) ** 0.5 * o
    return torch.where(on, (1 - lr * wd) * w - o, z), m, torch.where(on, o, z), on


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nesterov,wd", [(True, 0.01), (False, 0.0)])
def test_muon_step(dtype, nesterov, wd):
    layers = [layer(20 + 10 * i, *s) for i, s in enumerate(
        [(16, 16, dtype, True), (313, 256, dtype, False), (64, 64, dtype, True), (30, 7, dtype, True), (200, 90, dtype, False),
         (5, 1, dtype, True)])]
    ws, gs, ms, ks = (list(t) for t in zip(*layers))
    for w, g, m, k in layers:      # whatever lies on taps that are off has no say
        if k is not None:
            off = torch.stack([(k.long() >> t) & 1 for t in range(9)], -1).reshape(w.shape) == 0
            w[off], g[off], m[off] = float("nan"), float("inf"), float("nan")
    want = [muon_ref(w, g, m, k, nesterov=nesterov, wd=wd) for w, g, m, k in layers]
    out = ([torch.empty_like(w) for w in ws], [torch.empty_like(m) for m in ms])
    got = pp.muon_step(ws, gs, ms, lr=0.02, nesterov=nesterov, weight_decay=wd, keep=ks, out=out)
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    for w2, m2, (w, m, o, on) in zip(got[0], got[1], want):
        assert bool((w2[~on] == 0).all()) and bool((m2[~on] == 0).all())
        near(m2, m, 2.0 ** -22)
        off = float((w2.double() - w).norm())
        assert off <= limit(dtype) * float(o.norm()) + u * float(w.norm())
    same = [t.clone() for t in ws], [t.clone() for t in ms]
    back = pp.muon_step(*same[:1], gs, same[1], lr=0.02, nesterov=nesterov, weight_decay=wd, keep=ks)
    for a, b, c in zip(got[0] + got[1], back[0] + back[1], same[0] + same[1]):
        assert torch.equal(a, b) and b is c


def test_muon_single_and_streams():
    w, g, m, k = layer(50, 40, 20, "f32", True)
    want = pp.muon_step([w.clone()], [g], [m.clone()], lr=0.1, keep=[k])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = pp.muon_step(w.clone(), g, m.clone(), lr=0.1, keep=k)
    a = [w.clone(), m.clone()]
    torch.cuda.synchronize()
    pp.muon_step(a[0], g, a[1], lr=0.1, keep=k, stream=side)
    torch.cuda.synchronize()
    for x in (got, a):
        assert torch.equal(x[0], want[0][0]) and torch.equal(x[1], want[1][0])


def test_graph_replays():
    mats = [normal(60, 90, 200), normal(61, 300, 64)]
    pp.orthogonalize(mats)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = pp.orthogonalize(mats)
    for seed in (1, 2, 3):
        for i, t in enumerate(mats):
            t.copy_(normal(70 + 2 * seed + i, *t.shape))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, pp.orthogonalize(mats)):
            assert torch.equal(a, b)
        torch.cuda.synchronize()
