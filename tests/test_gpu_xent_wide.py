"""The head over a w whose rows lie far apart: d columns of a very wide matrix.
Up to 2^22 elements apart few tokens read them where they lie, beyond that they
are copied.  Error bounds as for any w."""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from test_gpu_xent import DT, Ref, make, near   # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,n,v,pitch", [("f32", 3, 600, 1 << 22), ("f32", 17, 3400, 1 << 20), ("bf16", 3, 600, 1 << 22),
                                             ("bf16", 3, 600, (1 << 22) - 1), ("f32", 3, 600, (1 << 22) + 1), ("f32", 1, 200, (1 << 25) + 8),
                                             ("bf16", 1, 200, (1 << 25) + 1), ("f32", 1, 200, 1 << 26), ("bf16", 1, 200, (1 << 26) + 8)])
def test_rows_of_w_far_apart(dtype, n, v, pitch):
    d = 64
    x, w, t, b, _, gr = make(21, n, d, 1, v, dtype, layout="tokens")
    wide = torch.full((v * pitch,), float("nan"), device="cuda", dtype=DT[dtype])
    far = wide.as_strided((v, d), (pitch, 1))
    far.copy_(w)
    grad = gr[0].reshape(()).clone()
    ref = Ref(x, w, t, b, None, grad)
    loss, dx, dw, db = pp.linear_xent_step(x, far, t, grad, bias=b)
    near(loss, ref.loss, ref.loss_lim, "loss")
    near(dx, ref.dx, ref.dx_lim, "dx")
    near(dw, ref.dw, ref.dw_lim, "dw")
    near(db, ref.db, ref.db_lim, "db")
    loss2, stats = pp.linear_xent_fwd(x, far, t, bias=b)
    assert torch.equal(loss, loss2)
    del wide, far
    torch.cuda.empty_cache()
