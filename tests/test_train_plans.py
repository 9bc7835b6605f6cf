"""What the training operators decide on the host: which kernels a call gets, as
far as the workspace that it asks for tells."""
import ctypes

import pytest

pp = pytest.importorskip("paper_2004_11250_amd")
from test_train_abi import desc   # noqa: E402


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
