"""Updates of zeros and of norms at the ends of fp32, which the scaling of X by
1 / (|U| + eps) meets with eps = 0: by matrices that a workgroup does whole and
by larger ones.  Error bounds as for any update."""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from test_gpu_ortho import DT, layer, limit, near, normal, ref   # noqa: E402

pytestmark = pytest.mark.gpu

SHAPES = [(16, 144), (40, 50), (100, 130), (300, 90)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [0.0, 1e-7])
def test_zeros(dtype, eps):
    zeros = [torch.zeros(s, device="cuda", dtype=DT[dtype]) for s in SHAPES]
    for o in pp.orthogonalize(zeros, eps=eps) + [pp.orthogonalize(z, eps=eps) for z in zeros]:
        assert bool((o == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c_out,c_in,pruned", [(16, 16, True), (128, 64, True), (30, 40, False), (130, 140, False)])
def test_layers_without_an_update(dtype, c_out, c_in, pruned):
    # no gradient and no momentum: the weights decay and nothing else happens to them
    w, g, m, keep = layer(40, c_out, c_in, dtype, pruned)
    on = torch.ones(w.shape, device="cuda", dtype=torch.bool)
    if pruned:
        on = torch.stack([(keep.long() >> t) & 1 for t in range(9)], -1).reshape(w.shape) != 0
    for decay, factor in ((0.0, 1.0), (0.5, 0.75)):
        got, momentum = pp.muon_step(w, torch.zeros_like(g), torch.zeros_like(m), lr=0.5, weight_decay=decay, keep=keep, eps=0.0,
                                     out=(torch.empty_like(w), torch.empty_like(m)))
        assert torch.equal(got, torch.where(on, w * factor, torch.zeros_like(w))) and bool((momentum == 0).all())


@pytest.mark.parametrize("dtype,scale", [("f32", 1e-42), ("f32", 1e-38), ("f32", 1e-30), ("f32", 1e30), ("f32", 5e37), ("bf16", 1e-38),
                                         ("bf16", 1e-30), ("bf16", 5e37)])
@pytest.mark.parametrize("shape", SHAPES)
def test_norms_at_the_ends_of_fp32(dtype, scale, shape):
    u = (normal(41, *shape).double() * scale).float().to(DT[dtype])
    assert bool(torch.isfinite(u).all())
    near(pp.orthogonalize(u, eps=0.0), ref(u, eps=0.0), limit(dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite(dtype, shape, bad):
    u = normal(42, *shape, dtype=dtype)
    u[3, 7] = bad
    assert bool(torch.isnan(pp.orthogonalize(u, eps=0.0)).all())
