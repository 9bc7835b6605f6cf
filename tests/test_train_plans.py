"""What the training operators decide on the host: which kernels a call gets, as
far as the workspace that it asks for tells."""
import ctypes

import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from paper_2004_11250_amd import train   # noqa: E402
from test_train_abi import A, desc, mats, ortho   # noqa: E402


@pytest.fixture(scope="module")
def lib():
    return pp.load_library()


def xent_bytes(lib, parts=3, **kw):
    nb = ctypes.c_size_t(0)
    assert lib.pp_xent_workspace(ctypes.byref(desc(**kw)), parts, ctypes.byref(nb)) == pp.PP_OK
    return nb.value


@pytest.mark.parametrize("dtype,n", [(pp.PP_F32, 1), (pp.PP_F32, 17), (pp.PP_F32, 128), (pp.PP_BF16, 1), (pp.PP_BF16, 64)])
@pytest.mark.parametrize("parts", [1, 2, 3])
def test_few_tokens_with_rows_of_w_far_apart(lib, dtype, n, parts):
    # The few-token kernels address w by 32-bit offsets from a descriptor of 16 or
    # 32 rows: rows further apart than 2^22 elements (2^29 bytes a descriptor) are
    # copied, for which the workspace then has room.
    v = 200 * n
    at = lambda pitch: xent_bytes(lib, parts, dtype=dtype, n=n, d=64, v=v, x_sn=64, x_sp=64, dx_sn=64, dx_sp=64, w_ld=pitch)   # noqa: E731
    copy = v * 64 * (6 if dtype == pp.PP_F32 else 2)
    assert at(1 << 22) == at(64)
    for pitch in ((1 << 22) + 1, 1 << 24, (1 << 24) + 8, 1 << 25, 1 << 26, (1 << 26) + 1, 1 << 31, 1 << 40):
        assert at(pitch) == at((1 << 22) + 8) >= copy, pitch
    assert at(64) != at(1 << 25)


def muon_layers(*shapes):
    arr = (train.MuonLayer * len(shapes))()
    for e, (r, c) in zip(arr, shapes):
        e.rows, e.cols, e.keep = r, c, None
        e.w = e.g = e.momentum = e.w_out = e.momentum_out = A
    return arr


def muon(lib, arr, n, ws, nb):
    d = train.MuonDesc(0.1, 0.9, 0.0, 1, 5, (ctypes.c_float * 3)(*train.COEFFS), 1e-7)
    return lib.pp_muon_step(arr, n, pp.PP_F32, ctypes.byref(d), ws, nb, None)


SMALL, STAGED, MIXED = [(16, 144), (9, 20)], [(80, 900), (313, 256)], [(16, 144), (313, 256), (0, 5)]


@pytest.mark.parametrize("shapes", [STAGED, MIXED])
def test_update_workspaces_are_what_the_calls_want(lib, shapes):
    for arr, query, call in ((mats(*shapes), lib.pp_ortho_workspace, lambda a, nb: ortho(lib, a, len(shapes), nb=nb)),
                             (muon_layers(*shapes), lib.pp_muon_workspace, lambda a, nb: muon(lib, a, len(shapes), A, nb))):
        nb = ctypes.c_size_t(0)
        assert query(arr, len(shapes), pp.PP_F32, ctypes.byref(nb)) == pp.PP_OK and nb.value > 0
        assert call(arr, nb.value - 1) == pp.PP_ESIZE


@pytest.mark.skipif(torch.cuda.is_available(), reason="the call gets as far as its launch, with addresses that are none")
def test_small_matrices_need_no_workspace(lib):
    nb = ctypes.c_size_t(1)
    assert lib.pp_ortho_workspace(mats(*SMALL), 2, pp.PP_F32, ctypes.byref(nb)) == pp.PP_OK and nb.value == 0
    assert ortho(lib, mats(*SMALL), 2, ws=None, nb=0) == pp.PP_EHIP
    nb = ctypes.c_size_t(1)
    assert lib.pp_muon_workspace(muon_layers(*SMALL), 2, pp.PP_F32, ctypes.byref(nb)) == pp.PP_OK and nb.value == 0
    assert muon(lib, muon_layers(*SMALL), 2, None, 0) == pp.PP_EHIP
