"""The loss's step through the C ABI: dx by strides of its own (channels last,
rows inside wider ones, images inside larger ones, from odd addresses), with
exactly the workspace that the query asks for and nothing written beside dx.
Error bounds as for any layout."""
import ctypes

import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from paper_2004_11250_amd import train   # noqa: E402
from test_gpu_xent import DT, Ref, make, near   # noqa: E402

pytestmark = pytest.mark.gpu


def step(x, w, t, b, dx):
    """pp_xent_step with x and dx [n, d, hw] by their strides, and the parts of its result."""
    lib, (n, d, hw), v = pp.load_library(), x.shape, w.shape[0]
    desc = train.XentDesc(pp.PP_BF16 if x.dtype == torch.bfloat16 else pp.PP_F32, train.PP_MEAN, n, d, hw, v, *x.stride(), *dx.stride(),
                          w.stride(0), -100)
    nb = ctypes.c_size_t(0)
    assert lib.pp_xent_workspace(ctypes.byref(desc), 3, ctypes.byref(nb)) == pp.PP_OK
    ws = torch.full((nb.value + 256,), 255, dtype=torch.uint8, device="cuda")       # (NaNs, and a guard behind)
    loss, stats = torch.empty((), device="cuda"), torch.empty(n * hw + 1, device="cuda")
    dw, db = torch.empty(v, d, device="cuda", dtype=w.dtype), torch.empty(v, device="cuda")
    got = lib.pp_xent_step(ctypes.byref(desc), x.data_ptr(), w.data_ptr(), b.data_ptr(), None, t.data_ptr(), None, loss.data_ptr(),
                           stats.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), ws.data_ptr(), nb.value,
                           torch.cuda.current_stream().cuda_stream)
    assert got == pp.PP_OK and bool((ws[nb.value:] == 255).all())
    return loss, dw, db


LAYOUTS = {   # of dx in a buffer: (elements, offset, strides)
    "first": lambda n, d, hw: (n * d * hw, 0, (d * hw, hw, 1)),
    "last": lambda n, d, hw: (n * d * hw, 0, (d * hw, 1, d)),
    "last, odd": lambda n, d, hw: (n * (d + 3) * hw + 8, 1, ((d + 3) * hw, 1, d + 3)),
    "last, wide rows": lambda n, d, hw: (n * (d + 8) * hw + 8, 8, ((d + 8) * hw, 1, d + 8)),
    "slice": lambda n, d, hw: (n * (d + 5) * hw + 8, 2 * hw, ((d + 5) * hw, hw, 1)),
    "pixels apart": lambda n, d, hw: (n * d * hw * 2 + 8, 3, (d * hw * 2, hw * 2, 2)),
    "images innermost": lambda n, d, hw: (n * d * hw, 0, (1, n, n * d)),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", sorted(LAYOUTS))
@pytest.mark.parametrize("n,d,hw,v", [(3, 64, 20, 313), (2, 75, 13, 700), (9, 96, 101, 313), (40, 200, 1, 90), (2, 64, 8, 4000), (7, 37, 1, 1500),
                                      (5, 136, 400, 3000)])
def test_dx_by_strides(dtype, layout, n, d, hw, v):
    x, w, t, b, _, _ = make(31, n, d, hw, v, dtype, ignored=0.1)
    size, first, strides = LAYOUTS[layout](n, d, hw)
    room = torch.full((size,), 7.0, device="cuda", dtype=DT[dtype])
    dx = room.as_strided((n, d, hw), strides, first)
    loss, dw, db = step(x, w, t, b, dx)
    ref = Ref(x, w, t, b)
    near(loss, ref.loss, ref.loss_lim, "loss")
    near(dx, ref.dx, ref.dx_lim, "dx")
    near(dw, ref.dw, ref.dw_lim, "dw")
    near(db, ref.db, ref.db_lim, "db")
    dx.fill_(7.0)
    assert bool((room == 7.0).all())     # (nothing beside it)
