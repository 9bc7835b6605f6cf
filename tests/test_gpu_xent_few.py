"""The head of few tokens (up to 64, in fp32 128, with at least 192 classes a
token), whose kernels read w where it lies: token counts around the kernels'
sixteens, odd channels and classes, rows of w inside wider and misaligned ones.
Error bounds as for any number of tokens."""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from test_gpu_xent import DT, Ref, check, make, near   # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 32, 33, 48, 49, 64, 65, 96, 97, 128, 129])
def test_token_counts(dtype, n):
    check(n, n, 72, 1, 200 * n + 3, dtype, layout="tokens", weighted=n % 2 == 0, reduction="none" if n % 3 == 0 else "mean")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [7, 8, 9, 10, 11, 12, 63, 66, 129, 255, 256, 257, 1030])
@pytest.mark.parametrize("n,v", [(3, 577), (20, 4001), (64, 12400), (90, 17301), (128, 24577)])
def test_channels_and_classes(dtype, d, n, v):
    check(d, n, d, 1, v, dtype, layout="tokens")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("images", [3, 8])
@pytest.mark.parametrize("layout", ["first", "last", "rows", "slice"])
def test_layouts(dtype, images, layout):
    n, hw = (10 * images, 1) if layout == "rows" else (images, 13)
    check(5, n, 100, hw, 2600 * images, dtype, layout=layout, ignored=0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,left,pitch", [(64, 0, 64), (64, 1, 67), (64, 2, 68), (37, 3, 41), (38, 2, 46), (40, 8, 56)])
def test_rows_of_w(dtype, d, left, pitch):
    n, v = {"f32": (101, 19501), "bf16": (21, 4150)}[dtype]
    x, w, t, b, cw, gr = make(6, n, d, 1, v, dtype, layout="tokens")
    wide = torch.full((v, pitch), float("nan"), device="cuda", dtype=DT[dtype])
    wide[:, left:left + d] = w
    w = wide[:, left:left + d]
    grad = gr[0].reshape(()).clone()
    ref = Ref(x, w, t, b, cw, grad)
    loss, dx, dw, db = pp.linear_xent_step(x, w, t, grad, bias=b)
    near(loss, ref.loss, ref.loss_lim, "loss")
    near(dx, ref.dx, ref.dx_lim, "dx")
    near(dw, ref.dw, ref.dw_lim, "dw")
    near(db, ref.db, ref.db_lim, "db")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_only_some_gradients(dtype):
    x, w, t, b, _, _ = make(7, 19, 90, 1, 3700, dtype, layout="tokens")
    loss, dx, dw, db = pp.linear_xent_step(x, w, t, bias=b)
    _, stats = pp.linear_xent_fwd(x, w, t, bias=b)
    only = pp.linear_xent_bwd(x, w, t, stats, bias=b, need=(True, False, False))
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    only = pp.linear_xent_bwd(x, w, t, stats, bias=b, need=(False, True, True))
    assert only[0] is None and torch.equal(only[1], dw) and torch.equal(only[2], db)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_but_ignored(dtype):
    x, w, t, b, _, _ = make(8, 9, 40, 1, 1800, dtype, layout="tokens")
    x[:] = float("nan")
    loss, dx, dw, db = pp.linear_xent_step(x, w, torch.full_like(t, -100), bias=b)
    assert float(loss) == 0.0
    for g in (dx, dw, db):
        assert not bool(g.ne(0).any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_target_outside(dtype):
    x, w, t, b, _, _ = make(9, 5, 40, 1, 1000, dtype, layout="tokens")
    t[2] = 1000
    loss, dx, dw, db = pp.linear_xent_step(x, w, t, bias=b)
    assert bool(loss.isnan()) and bool(dx[2].isnan().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_past_32_bits(dtype):
    # (w and dw have more than 2^32 bytes, in bf16 more than 2^32 elements)
    d, v = 65536, {"f32": 17000, "bf16": 66000}[dtype]
    x, _, t, _, _, _ = make(10, 2, d, 1, v, dtype, layout="tokens", bias=False)
    t[0], t[1] = v - 1, 5
    w = torch.empty(v, d, device="cuda", dtype=DT[dtype])
    for i in range(0, v, 2000):
        w[i:i + 2000] = make(11 + i, 1, d, 1, min(2000, v - i), dtype, layout="tokens", bias=False)[1]
    loss, dx, dw, _ = pp.linear_xent_step(x, w, t)
    lse = torch.logsumexp(torch.cat([x.double() @ w[i:i + 2000].double().t().contiguous() for i in range(0, v, 2000)], 1), 1)
    for rows in (slice(0, 40), slice(v - 40, v)):
        lim = Ref(x, w[rows], torch.zeros_like(t))     # (its bound on a logit)
        l = x.double() @ w[rows].double().t().contiguous()
        G = torch.exp(l - lse[:, None]) / 2
        for i in range(2):
            at = int(t[i]) - (rows.start or 0)
            if 0 <= at < 40:
                G[i, at] -= 0.5
        want = G.t().contiguous() @ x.double()
        u = {"f32": 2.0 ** -21, "bf16": 2.0 ** -7}[dtype]
        bound = (2 * lim.lse_lim.max() + 1e-5) * (G.abs().t().contiguous() @ x.double().abs()) + u * (G.abs().t().contiguous() @ x.double().abs())
        near(dw[rows], want, bound, "dw")
    each = lse - torch.stack([(x[i].double() * w[int(t[i])].double()).sum() for i in range(2)])
    near(loss, each.mean(), 2 * lim.lse_lim.max() + 1e-5, "loss")
