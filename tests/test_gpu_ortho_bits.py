"""fp32 updates keep fp32's precision: bounds that an iterate with 16-bit values in
its products does not meet.

The values between the products are pairs of fp16 values, 22 bits where fp32 has
24: every rounding of the plain fp32 iteration is at most four times as large,
and the product of the two rests, which is left out, is one more of that size
beside each.  So the error is at most 8 times that of the plain iteration in
fp32 on the same input, which carries the input's own condition (directions that
grow from nothing amplify either's roundings alike).  Where the plain one happens
to be exact: 4 roundings of 2^-22 a step.  One fp16 value in place of a pair errs
by 2^-12 a rounding, a thousand times as much: the oracle below, run both ways,
shows that the bound tells them apart.
"""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from test_gpu_ortho import MUON, layer, muon_ref, normal, ref   # noqa: E402


def plain(u, steps=5, coeffs=MUON, eps=1e-7):
    """The iteration in fp32."""
    x = u.float().reshape(u.shape[0], -1)
    x = x / (x.double().square().sum().sqrt() + eps).float()
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    a, b, c = coeffs
    for _ in range(steps):
        g = x @ x.t().contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    return (x.t() if tall else x).reshape(u.shape)


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def limit(u, want, steps=5, coeffs=MUON, eps=1e-7):
    return 8 * off(plain(u, steps, coeffs, eps), want) + 4 * steps * 2.0 ** -22


def emulated(u, planes, steps=5):
    """The iteration in 64 bits with X, A and B held as `planes` fp16 values in the products, all of their products but rest x rest."""
    def parts(v, scale):
        h = (v * scale).half().double()
        return h / scale, ((v * scale - h).half().double() / scale if planes == 2 else torch.zeros_like(h))

    def product(p, q):
        return p[0] @ q[0] + p[0] @ q[1] + p[1] @ q[0]

    x = u.double() / (u.double().norm() + 1e-7)
    a, b, c = MUON
    for _ in range(steps):
        X = parts(x, 8192.0)
        A = parts(product(X, (X[0].t(), X[1].t())), 4096.0)
        B = parts(a * torch.eye(len(x), dtype=x.dtype) + b * (A[0] + A[1]) + c * product(A, (A[0].t(), A[1].t())), 1024.0)
        x = product(B, X)
    return x


@pytest.mark.parametrize("kind", ["broad", "low rank", "one entry"])
def test_the_bound_tells_planes_apart(kind):
    g = torch.Generator().manual_seed(5)
    u = torch.randn(90, 200, generator=g)
    if kind == "low rank":
        u = u[:, :4] @ torch.randn(4, 200, generator=g)
    if kind == "one entry":
        u[3, 5] = 1e4
    want = ref(u)
    lim = limit(u, want)
    assert off(emulated(u, 2), want) <= lim < 0.1 * off(emulated(u, 1), want)


SHAPES = [(1, 1), (9, 1), (2, 3), (16, 144), (63, 65), (65, 64), (100, 1000), (313, 256), (777, 129), (512, 4608), (700, 900), (1500, 1601),
          (2600, 2600), (4010, 3970)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape):
    u = normal(51, *shape)
    want = ref(u)
    assert off(pp.orthogonalize(u), want) <= limit(u, want)


@pytest.mark.gpu
@pytest.mark.parametrize("steps,coeffs", [(1, MUON), (2, MUON), (8, MUON), (5, (1.875, -1.25, 0.375)), (6, (1.5, -0.5, 0.0))])
def test_steps_and_coefficients(steps, coeffs):
    for shape in ((40, 60), (90, 200)):
        u = normal(52, *shape)
        want = ref(u, steps, coeffs)
        assert off(pp.orthogonalize(u, steps=steps, coeffs=coeffs), want) <= limit(u, want, steps, coeffs)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(48, 60), (120, 300), (300, 120)])
def test_inputs_far_from_broad(shape):
    low = normal(53, shape[0], 4) @ normal(54, 4, shape[1])
    one = normal(55, *shape)
    one[3, 5] = 1e4
    rows = normal(56, *shape) * torch.logspace(-6, 0, shape[0], device="cuda")[:, None]
    for u, eps in ((low, 0.0), (low * 1e-20, 0.0), (low * 1e18, 0.0), (one, 1e-7), (rows, 1e-7), (normal(57, *shape) * 1e-9, 1e-7)):
        want = ref(u, eps=eps)
        assert off(pp.orthogonalize(u, eps=eps), want) <= limit(u, want, eps=eps)


@pytest.mark.gpu
def test_lists():
    mats = [normal(60 + i, *s) for i, s in enumerate([(313, 256), (1000, 513), (16, 144), (77, 1201), (64, 64, 3, 3)])]
    for u, o in zip(mats, pp.orthogonalize(mats)):
        want = ref(u)
        assert off(o, want) <= limit(u.reshape(u.shape[0], -1), want.reshape(u.shape[0], -1))


@pytest.mark.gpu
def test_weight_steps():
    layers = [layer(70 + 10 * i, *s) for i, s in enumerate([(16, 16, "f32", True), (128, 64, "f32", True), (313, 256, "f32", False)])]
    ws, gs, ms, ks = (list(t) for t in zip(*layers))
    got = pp.muon_step(ws, gs, ms, lr=0.02, weight_decay=0.01, keep=ks,
                       out=([torch.empty_like(w) for w in ws], [torch.empty_like(m) for m in ms]))
    for w2, (w, g, m, k) in zip(got[0], layers):
        want, mom, _, on = muon_ref(w, g, m, k)
        update = torch.where(on, g, torch.zeros_like(g)) + 0.95 * mom.float()
        # (the update is formed in fp32; W and its decay are rounded by 2^-23; a pruned layer's errors are part of the whole iterate's)
        o = ref(update.double())
        size = 0.02 * max(1.0, w.shape[0] / (w.numel() // w.shape[0])) ** 0.5 * float(o.norm())
        assert float((w2.double() - want).norm()) <= (limit(update, o) + 2.0 ** -22) * size + 2.0 ** -23 * float(w.norm())
