"""What pp.h says of bf16 updates: five steps err by at most 2e-3 of the result's
norm beside its rounding to bf16, whatever the update's directions look like
(1.7e-3 and less as measured), and matrices that a workgroup does whole by 1e-4."""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from test_gpu_ortho import normal, ref   # noqa: E402

pytestmark = pytest.mark.gpu


def updates(m, n):
    one = normal(4, m, 1) @ normal(5, 1, n)
    entry = normal(7, m, n)
    entry[3, 5] = 1e2
    row = normal(7, m, n)
    row[3] *= 1e3
    return {"broad": normal(1, m, n), "four directions": normal(2, m, 4) @ normal(3, 4, n), "one direction": one + 1e-2 * normal(6, m, n),
            "one entry": entry, "one row": row, "rows of all sizes": normal(8, m, n) * torch.logspace(-3, 0, m, device="cuda")[:, None],
            "shifted": normal(9, m, n) + 1, "strong and broad": normal(10, m, n) / n ** 0.5 + normal(11, m, 16) @ normal(12, 16, n) / (16 * n) ** 0.5}


@pytest.mark.parametrize("shape", [(48, 60), (70, 90), (256, 2304), (1024, 1024)])
def test_error_beside_the_rounding(shape):
    for kind, u in updates(*shape).items():
        u = u.bfloat16()
        want = ref(u)
        size = float(want.norm())
        err = float((pp.orthogonalize(u).double() - want).norm()) / size
        rounding = float((want.bfloat16().double() - want).norm()) / size
        lim = 1e-4 if shape == (48, 60) else 2e-3
        assert err <= (rounding ** 2 + lim ** 2) ** 0.5, (kind, err, rounding)
