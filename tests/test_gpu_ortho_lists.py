"""Long lists and long thin matrices: more matrices than one look-up of a
workgroup's tile takes (64) or one set-up launch brings (12), and matrices of a few
rows that are too long for a workgroup.  Error bounds as for any update."""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from test_gpu_ortho import layer, limit, muon_ref, near, normal, ref   # noqa: E402
from test_gpu_ortho_bits import limit as close   # noqa: E402

pytestmark = pytest.mark.gpu


def within(u, o, dtype):
    want = ref(u)
    near(o, want, min(close(u, want), limit(dtype)) if dtype == "f32" else limit(dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count", [12, 13, 64, 65, 130])
def test_long_lists(dtype, count):
    mats = [normal(100 + i, 66 + i % 9, 70 + 13 * (i % 17), dtype=dtype) for i in range(count)] + [normal(99, 16, 40, dtype=dtype)]
    for u, o in zip(mats, pp.orthogonalize(mats)):
        within(u, o, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 5000), (3, 9001), (5000, 2), (70001, 5), (17, 4099), (64, 40000)])
def test_long_and_thin(dtype, shape):
    u = normal(98, *shape, dtype=dtype)
    within(u, pp.orthogonalize(u), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_long_list_of_layers(dtype):
    layers = [layer(200 + 10 * i, 70 + i, 8 + i % 5, dtype, i % 3 != 0) for i in range(70)]
    ws, gs, ms, ks = (list(t) for t in zip(*layers))
    want = [muon_ref(w, g, m, k) for w, g, m, k in layers]
    got = pp.muon_step(ws, gs, ms, lr=0.02, weight_decay=0.01, keep=ks)
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    for w2, m2, (w, m, o, on) in zip(got[0], got[1], want):
        assert bool((w2[~on] == 0).all()) and bool((m2[~on] == 0).all())
        near(m2, m, 2.0 ** -22)
        assert float((w2.double() - w).norm()) <= limit(dtype) * float(o.norm()) + u * float(w.norm())
