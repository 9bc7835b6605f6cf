"""What autograd sees of the training operators: results without a graph, and
tensors written in place as changed."""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from test_gpu_ortho import layer, normal   # noqa: E402
from test_gpu_xent import make   # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("single", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_weight_step_counts_as_a_change(single, in_place):
    w, g, m, _ = layer(60, 90, 40, "f32", False)
    w.requires_grad_()
    x = normal(63, 5, 40).requires_grad_()
    y = (x @ w.t()).sum()
    before = w._version, m._version
    out = None if in_place else (torch.empty_like(w), torch.empty_like(m))
    if single:
        pp.muon_step(w, g, m, lr=0.1, out=out)
    else:
        pp.muon_step([w], [g], [m], lr=0.1, out=None if in_place else ([out[0]], [out[1]]))
    if in_place:
        assert w._version > before[0] and m._version > before[1]
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    else:
        assert (w._version, m._version) == before and out[0]._version > 0 and out[1]._version > 0
        y.backward()


def test_updates_in_place_count_as_a_change():
    u, v = normal(64, 30, 40), normal(65, 300, 90)
    before = u._version, v._version
    pp.orthogonalize([u, v])
    assert (u._version, v._version) == before
    pp.orthogonalize([u, v], out=[u, v])
    assert u._version > before[0] and v._version > before[1]
    before = u._version
    pp.orthogonalize(u, out=u)
    assert u._version > before


def test_features_with_a_graph():
    # the returned gradient of the features goes on through their own graph
    x, w, t, b, _, _ = make(22, 20, 64, 1, 90, "f32", layout="tokens")
    want = pp.linear_xent_step(x, w, t, bias=b)
    base = (x / 2).requires_grad_()
    features, w = base * 2, w.clone().requires_grad_()
    got = pp.linear_xent_step(features, w, t, bias=b)
    for a, c in zip(got, want):
        assert torch.equal(a, c) and not a.requires_grad
    features.backward(got[1])
    assert torch.equal(base.grad, 2 * want[1]) and w.grad is None
