"""Softmax cross entropy of a linear head (pp_xent_*) on the GPU against the
formula in 64 bits.

Error bounds (u = 2^-24): a logit is a sum of d exact products and a bias in
fp32, in some order: (d + 64) u S with S = sum |x||w| + |b| (the 64 covers the
three-way split of fp32 features, each product of which is within 4 u, and the
bias).  With L the largest such bound of a token, its log-sum-exp moves by at
most L, plus the error of the exponentials and their fp32 sum (relative 2e-6,
the sum of positive terms keeps it) and one rounding; its loss by twice that.
The gradient of a logit is s (p - [v = y]): p moves by a relative 2 (L + 4e-6),
and G is rounded by r (bf16: 2^-8; fp32, three bf16 values: 2^-23).  A product
with G sums k terms: k u of the sum of magnitudes, and the output is rounded
once (bf16: 2^-8).
"""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND_G = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8}
ROUND_OUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def make(seed, n, d, hw, v, dtype, *, bias=True, weighted=False, ignored=0.0, layout="first", scale=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*s):
        return torch.randn(s, generator=g, device="cuda")

    x = normal(n, d, hw).to(DT[dtype])
    if layout == "tokens":
        assert hw == 1
        x = x.reshape(n, d)
    elif layout == "last":          # channels last: pixels d apart
        x = x.transpose(1, 2).contiguous().transpose(1, 2)
    elif layout == "rows":          # token rows inside wider rows
        wide = torch.full((n, d + 8), float("nan"), device="cuda", dtype=x.dtype)
        wide[:, 3:3 + d] = x.reshape(n, d)
        x = wide[:, 3:3 + d]
    elif layout == "slice":         # images inside larger ones
        wide = torch.full((n, d + 2, hw), float("nan"), device="cuda", dtype=x.dtype)
        wide[:, 1:1 + d] = x
        x = wide[:, 1:1 + d]
    w = (normal(v, d) * (scale / d ** 0.5)).to(DT[dtype])
    shape = (n,) if x.dim() == 2 else (n, hw)
    t = torch.randint(0, v, shape, generator=g, device="cuda")
    drop = torch.rand(shape, generator=g, device="cuda") < ignored
    t = torch.where(drop, torch.full_like(t, -100), t)
    b = normal(v) if bias else None
    cw = torch.rand(v, generator=g, device="cuda") + 0.5 if weighted else None
    gr = torch.rand(shape, generator=g, device="cuda") + 0.1
    return x, w, t, b, cw, gr


class Ref:
    """The formula in 64 bits, with the error bounds above."""

    def __init__(self, x, w, t, b=None, cw=None, grad=None, reduction="mean", ignore=-100):
        dtype = "bf16" if x.dtype == torch.bfloat16 else "f32"
        self.shape = x.shape
        n, d = x.shape[:2]
        xs = x.double().reshape(n, d, -1).permute(0, 2, 1).reshape(-1, d)
        w = w.double().reshape(w.shape[0], d)
        v = w.shape[0]
        y = t.reshape(-1)
        keep = y != ignore
        xs = torch.where(keep[:, None], xs, torch.zeros_like(xs))
        at = torch.where(keep, y, torch.zeros_like(y))
        l = xs @ w.t() + (0 if b is None else b.double())
        mag = xs.abs() @ w.abs().t() + (0 if b is None else torch.nan_to_num(b.double().abs(), posinf=0.0))
        lim = (d + 64) * U * mag.amax(1)
        self.lse = torch.logsumexp(l, 1)
        c = keep.double() if cw is None else keep.double() * cw.double()[at]
        each = torch.where(keep, c * (self.lse - l.gather(1, at[:, None])[:, 0]), torch.zeros_like(self.lse))
        self.lse = torch.where(keep, self.lse, torch.zeros_like(self.lse))
        self.lse_lim = lim + 2e-6 + 2 * U * self.lse.abs()
        each_lim = c * (2 * lim + 2e-6) + 4 * U * (each.abs() + c * self.lse.abs())
        self.div = c.sum() if reduction == "mean" and c.sum() > 0 else torch.ones((), device=x.device, dtype=torch.float64)
        if reduction == "none":
            self.loss, self.loss_lim = each, each_lim
        else:
            self.loss = each.sum() / self.div
            self.loss_lim = each_lim.sum() / self.div + 4 * U * self.loss.abs()
        s = c / self.div
        if grad is not None:
            s = s * (grad.double().reshape(-1) if reduction == "none" else grad.double().reshape(()))
        p = torch.exp(l - torch.logsumexp(l, 1, keepdim=True))
        hit = torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
        G = torch.where(keep[:, None], (p - hit) * s[:, None], torch.zeros_like(p))
        tokens = len(y)
        Glim = s[:, None].abs() * p * (2 * (lim[:, None] + 4e-6)) + G.abs() * (ROUND_G[dtype] + 4 * U) + 2 * U * s[:, None].abs() * hit
        self.dx = G @ w
        dxl = (Glim + (v + 64) * U * G.abs()) @ w.abs() + ROUND_OUT[dtype] * self.dx.abs()
        self.dw = G.t().contiguous() @ xs
        self.dw_lim = (Glim + (tokens + 64) * U * G.abs()).t().contiguous() @ xs.abs() + ROUND_OUT[dtype] * self.dw.abs()
        self.db = G.sum(0)
        # (summed before it is rounded to the operands' type)
        self.db_lim = (Glim + (tokens + 64) * U * G.abs()).sum(0)
        back = lambda z: z.reshape(n, -1, d).permute(0, 2, 1).reshape(self.shape)   # noqa: E731
        self.dx, self.dx_lim = back(self.dx), back(dxl)


def near(got, want, lim, what):
    got = got.double().reshape(want.shape)
    err = (got - want).abs()
    bad = ~(err <= lim + 1e-37)     # (a NaN is out)
    assert not bool(bad.any()), (what, int(bad.sum()), float((err / (lim + 1e-37)).nan_to_num(nan=1e30).max()))


def check(seed, n, d, hw, v, dtype, *, reduction="mean", with_grad=True, **kw):
    x, w, t, b, cw, gr = make(seed, n, d, hw, v, dtype, **kw)
    grad = None if not with_grad else gr if reduction == "none" else gr.reshape(-1)[:1].reshape(()).clone()
    ref = Ref(x, w, t, b, cw, grad, reduction)
    more = dict(bias=b, class_weight=cw, reduction=reduction)
    loss, stats = pp.linear_xent_fwd(x, w, t, **more)
    near(loss, ref.loss, ref.loss_lim, "loss")
    near(stats[:-1], ref.lse, ref.lse_lim, "lse")
    near(stats[-1], ref.div, 1e-5 * ref.div, "divisor")
    dx, dw, db = pp.linear_xent_bwd(x, w, t, stats, grad, **more)
    near(dx, ref.dx, ref.dx_lim, "dx")
    near(dw, ref.dw, ref.dw_lim, "dw")
    assert dx.dtype == x.dtype and dw.dtype == w.dtype and (db is None) == (b is None)
    if b is not None:
        near(db, ref.db, ref.db_lim, "db")
    loss2, dx2, dw2, db2 = pp.linear_xent_step(x, w, t, grad, **more)
    for a, c in ((loss, loss2), (dx, dx2), (dw, dw2), (db, db2)):
        assert a is None and c is None or torch.equal(a, c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,hw,v", [(1, 1, 1, 1), (1, 1, 1, 2), (1, 64, 1, 1000), (3, 5, 1, 7), (2, 63, 1, 65),
                                      (65, 128, 1, 64), (77, 203, 1, 501), (130, 257, 1, 1030)])
def test_tokens(dtype, n, d, hw, v):
    check(1, n, d, hw, v, dtype, layout="tokens")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["first", "last", "slice"])
@pytest.mark.parametrize("n,d,hw,v", [(1, 64, 49, 100), (3, 64, 64, 313), (2, 96, 77, 130), (5, 17, 4, 11)])
def test_pixels(dtype, layout, n, d, hw, v):
    check(2, n, d, hw, v, dtype, layout=layout, weighted=True, ignored=0.2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("bias,weighted,with_grad", [(False, False, False), (True, False, True), (False, True, True)])
def test_reductions(dtype, reduction, bias, weighted, with_grad):
    check(3, 100, 64, 1, 200, dtype, layout="rows", reduction=reduction, bias=bias, weighted=weighted, ignored=0.1,
          with_grad=with_grad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_tiles(dtype):
    check(4, 2050, 72, 1, 6600, dtype, layout="tokens", ignored=0.1)


@pytest.mark.parametrize("n,d,hw,v,layout", [(8200, 72, 1, 9000, "tokens"), (3, 40, 2800, 9100, "first")])
def test_several_pieces(n, d, hw, v, layout):
    check(5, n, d, hw, v, "bf16", layout=layout, ignored=0.1)


def test_statistics_in_several_pieces():
    # more classes and tokens than the forward pass keeps statistics of at once
    x, w, t, b, cw, _ = make(18, 16400, 64, 1, 70000, "bf16", layout="tokens", ignored=0.01)
    # (only the loss: the gradients' bounds would take tens of GB)
    l = x.double() @ w.double().t() + b.double()
    lim = (64 + 64) * U * (x.double().abs() @ w.double().abs().t() + b.double().abs()).amax(1)
    lse = torch.logsumexp(l, 1)
    keep = t != -100
    each = torch.where(keep, lse - l.gather(1, t.clamp(min=0)[:, None])[:, 0], torch.zeros_like(lse))
    loss, stats = pp.linear_xent_fwd(x, w, t, bias=b, reduction="none")
    near(loss, each, 2 * lim + 2e-6 + 4 * U * (each.abs() + lse.abs()), "loss")
    near(stats[:-1], torch.where(keep, lse, torch.zeros_like(lse)), lim + 2e-6 + 2 * U * lse.abs(), "lse")


def test_long_sums_are_split():
    # many tokens, few classes and features; few tokens, many classes
    check(6, 4, 32, 5000, 40, "bf16", weighted=True)
    check(6, 2, 64, 1, 30000, "f32", layout="tokens")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sharp_and_far_logits(dtype):
    # logits of hundreds: one class takes all, the others underflow
    check(7, 50, 64, 1, 300, dtype, layout="tokens", scale=200.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ignored_tokens_contribute_nothing(dtype):
    x, w, t, b, cw, _ = make(8, 2, 64, 40, 70, dtype, weighted=True)
    t[0, 3] = t[1, 0] = t[1, 39] = -100
    want = pp.linear_xent_step(x, w, t, bias=b, class_weight=cw)
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(DT[dtype]).min):
        y = x.clone()
        y[0, :, 3] = y[1, :, 0] = y[1, 5:, 39] = bad
        got = pp.linear_xent_step(y, w, t, bias=b, class_weight=cw)
        for a, c in zip(got, want):
            assert torch.equal(a, c)
        assert bool((got[1][0, :, 3] == 0).all()) and bool((got[1][1, :, 0] == 0).all())


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_all_ignored_and_no_tokens(reduction):
    x, w, t, b, _, _ = make(9, 2, 64, 9, 30, "bf16")
    t[:] = -100
    loss, dx, dw, db = pp.linear_xent_step(x, w, t, bias=b, reduction=reduction)
    assert all(bool((g == 0).all()) for g in (loss, dx, dw, db))
    for shape in ((0, 64), (0, 64, 3, 3), (2, 64, 0)):
        x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
        t = torch.empty((shape[0],) + shape[2:], device="cuda", dtype=torch.int64)
        loss, dx, dw, db = pp.linear_xent_step(x, w, t, bias=b, reduction=reduction)
        assert loss.shape == (t.shape if reduction == "none" else ())
        assert bool((loss == 0).all()) and dx.shape == x.shape and bool((dw == 0).all()) and bool((db == 0).all())
        loss, stats = pp.linear_xent_fwd(x, w, t, bias=b, reduction=reduction)
        assert stats.tolist() == [1.0]


def test_classes_that_are_off():
    # a bias of -inf takes a class out; a target there has an infinite loss
    x, w, t, b, _, _ = make(10, 40, 64, 1, 300, "f32", layout="tokens")
    off = torch.arange(300, device="cuda") % 3 == 0
    b = torch.where(off, torch.full_like(b, -float("inf")), b)
    t = torch.where(off[t], t + 1, t)
    ref = Ref(x, w, t, b, reduction="none")
    loss, dx, dw, db = pp.linear_xent_step(x, w, t, bias=b, reduction="none")
    near(loss, ref.loss, ref.loss_lim, "loss")
    near(dx, ref.dx, ref.dx_lim, "dx")
    near(dw, ref.dw, ref.dw_lim, "dw")
    assert bool((db[off] == 0).all()) and bool((dw[off] == 0).all())
    t[7] = 3
    loss, _ = pp.linear_xent_fwd(x, w, t, bias=b, reduction="none")
    assert loss[7] == float("inf") and bool(torch.isfinite(loss[:7]).all()) and bool(torch.isfinite(loss[8:]).all())
    loss, _ = pp.linear_xent_fwd(x, w, t, bias=torch.full_like(b, -float("inf")), reduction="none")
    assert bool(torch.isnan(loss).all())
    # the type's lowest value is a number like any other
    low = torch.where(off, torch.full_like(b, torch.finfo(torch.float32).min), torch.zeros_like(b))
    t = torch.where(off[t], t + 1, t)
    ref = Ref(x, w, t, torch.where(off, torch.full_like(b, -float("inf")), torch.zeros_like(b)), reduction="none")
    loss, dx, dw, db = pp.linear_xent_step(x, w, t, bias=low, reduction="none")
    near(loss, ref.loss, ref.loss_lim, "loss")
    near(dx, ref.dx, ref.dx_lim, "dx")


def test_target_outside_the_classes():
    x, w, t, b, _, _ = make(11, 30, 64, 1, 50, "f32", layout="tokens")
    good, _ = pp.linear_xent_fwd(x, w, t, bias=b, reduction="none")
    for bad in (50, -1, 1 << 40, -(1 << 40)):
        t2 = t.clone()
        t2[4] = bad
        loss, dx, dw, db = pp.linear_xent_step(x, w, t2, bias=b, reduction="none")
        assert torch.isnan(loss[4]) and torch.equal(loss[:4], good[:4]) and torch.equal(loss[5:], good[5:])
        assert bool(torch.isnan(dx[4]).all()) and bool(torch.isfinite(dx[:4]).all()) and bool(torch.isnan(dw).all())
        assert torch.isnan(pp.linear_xent_fwd(x, w, t2, bias=b)[0])
        assert torch.equal(pp.linear_xent_fwd(x, w, t2, bias=b, reduction="sum", ignore_index=bad)[0],
                           pp.linear_xent_fwd(x, w, torch.where(t2 == bad, torch.full_like(t2, -100), t2), bias=b, reduction="sum")[0])


def test_nan_features_reach_their_token_only():
    x, w, t, b, _, _ = make(12, 30, 64, 1, 50, "f32", layout="tokens")
    good, _ = pp.linear_xent_fwd(x, w, t, bias=b, reduction="none")
    x[9, 5] = float("nan")
    loss, dx, dw, db = pp.linear_xent_step(x, w, t, bias=b, reduction="none")
    assert torch.isnan(loss[9]) and torch.equal(loss[:9], good[:9]) and torch.equal(loss[10:], good[10:])
    assert bool(torch.isnan(dx[9]).all()) and bool(torch.isfinite(dx[10:]).all()) and bool(torch.isnan(db).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_against_differences(dtype):
    # central differences of the 64-bit loss along random directions
    x, w, t, b, cw, gr = make(13, 3, 32, 10, 40, dtype, weighted=True, ignored=0.1)
    dx, dw, db = pp.linear_xent_step(x, w, t, gr, bias=b, class_weight=cw, reduction="none")[1:]
    ref = Ref(x, w, t, b, cw, gr, "none")
    loss = lambda x, w, b: float((Ref(x, w, t, b, cw, None, "none").loss * gr.double().reshape(-1)).sum())   # noqa: E731
    h, g = 1e-5, torch.Generator(device="cuda").manual_seed(1)
    x, w, b = x.double(), w.double(), b.double()
    for k, (grad, lim) in enumerate(((dx, ref.dx_lim), (dw, ref.dw_lim), (db, ref.db_lim))):
        for _ in range(3):
            u = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)
            at = [[x, w, b], [x, w, b]]
            at[0][k], at[1][k] = at[0][k] + h * u, at[1][k] - h * u
            diff = (loss(*at[0]) - loss(*at[1])) / (2 * h)
            # (third derivatives of order one: h^2 |u|^3; rounding of the loss over h)
            assert abs(float((grad.double() * u).sum()) - diff) <= float((lim * u.abs()).sum()) + 1e-6


def test_some_gradients_only():
    x, w, t, b, _, _ = make(14, 2, 64, 30, 90, "bf16")
    full = pp.linear_xent_step(x, w, t, bias=b)[1:]
    _, stats = pp.linear_xent_fwd(x, w, t, bias=b)
    for need in ((True, False, False), (False, True, False), (False, False, True), (False, False, False)):
        got = pp.linear_xent_bwd(x, w, t, stats, bias=b, need=need)
        for a, c, k in zip(got, full, need):
            assert torch.equal(a, c) if k else a is None


def test_weights_as_a_convolution_and_with_a_pitch():
    x, w, t, b, _, _ = make(15, 2, 64, 30, 90, "bf16")
    want = pp.linear_xent_step(x, w, t, bias=b)
    got = pp.linear_xent_step(x.reshape(2, 64, 5, 6), w.reshape(90, 64, 1, 1), t.reshape(2, 5, 6), bias=b)
    assert got[1].shape == (2, 64, 5, 6) and got[2].shape == (90, 64, 1, 1)
    wide = torch.zeros(90, 71, device="cuda", dtype=w.dtype)
    wide[:, :64] = w
    pitched = pp.linear_xent_step(x, wide[:, :64], t, bias=b)
    for a, c, e in zip(want, got, pitched):
        assert torch.equal(a.reshape(-1), c.reshape(-1)) and torch.equal(a, e)


def test_streams_and_repeats():
    x, w, t, b, cw, _ = make(16, 8, 64, 100, 313, "bf16", weighted=True)
    want = pp.linear_xent_step(x, w, t, bias=b, class_weight=cw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [pp.linear_xent_step(x, w, t, bias=b, class_weight=cw, stream=s) for s in (side, None, side, None)]
    torch.cuda.synchronize()
    for g in got:
        for a, c in zip(want, g):
            assert torch.equal(a, c)


def test_graph_replays():
    x, w, t, b, _, _ = make(17, 8, 64, 100, 313, "bf16")
    pp.linear_xent_step(x, w, t, bias=b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pp.linear_xent_step(x, w, t, bias=b)
    for seed in (1, 2, 3):
        y = make(100 + seed, 8, 64, 100, 313, "bf16")
        x.copy_(y[0]), t.copy_(y[2])
        graph.replay()
        torch.cuda.synchronize()
        want = pp.linear_xent_step(x, w, t, bias=b)
        torch.cuda.synchronize()
        for a, c in zip(out, want):
            assert torch.equal(a, c)
