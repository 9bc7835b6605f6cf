"""The gradient in several pieces of the classes: dx's sums carried from piece to
piece, dw and db at each piece's offset, targets in every piece, and a last,
smaller piece with tiles of its own and fewer k steps than dx's sum has parts.
That there are several pieces is seen in the workspace, which is smaller than
what G would take in one.  Error bounds as for any number of classes."""
import ctypes

import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from paper_2004_11250_amd import train   # noqa: E402
from test_gpu_xent import check   # noqa: E402

# (the last piece: 163, 429, 53 and 16 classes)
SIZES = [("bf16", 7982, 66, 1, 57507, "tokens"), ("bf16", 2, 116, 1981, 123309, "first"), ("f32", 8941, 53, 1, 16437, "tokens"),
         ("f32", 4, 90, 1989, 32784, "first")]


@pytest.mark.parametrize("dtype,n,d,hw,v,layout", SIZES)
@pytest.mark.parametrize("parts", [2, 3])
def test_sizes_have_several_pieces(dtype, n, d, hw, v, layout, parts):
    desc = train.XentDesc(pp.PP_F32 if dtype == "f32" else pp.PP_BF16, train.PP_MEAN, n, d, hw, v, d * hw, hw, 1, d * hw, hw, 1, d, -100)
    nb = ctypes.c_size_t(0)
    assert pp.load_library().pp_xent_workspace(ctypes.byref(desc), parts, ctypes.byref(nb)) == pp.PP_OK
    assert nb.value < n * hw * v * (6 if dtype == "f32" else 2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,d,hw,v,layout", SIZES)
def test_pieces(dtype, n, d, hw, v, layout):
    check(23, n, d, hw, v, dtype, layout=layout, ignored=0.1, weighted=dtype == "bf16", reduction="none" if hw > 1 else "mean")
    torch.cuda.empty_cache()
