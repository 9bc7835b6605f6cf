"""The head of few classes, all of which a workgroup has (up to 512, in bf16 up to
512 channels), around the sizes at which its tiles change.  Error bounds as
for any number of classes."""
import pytest

pp = pytest.importorskip("paper_2004_11250_amd")
from test_gpu_xent import check   # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [2, 63, 64, 65, 128, 255, 256, 257, 313, 448, 511, 512, 513])
def test_classes(dtype, v):
    check(v, 6, 96, 101, v, dtype, weighted=v % 2 == 0, ignored=0.2, reduction=["mean", "sum", "none"][v % 3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [66, 129, 511, 512, 513, 1000])
@pytest.mark.parametrize("d,v", [(64, 300), (511, 200), (512, 313), (513, 130), (31, 500)])
def test_tokens_and_channels(dtype, n, d, v):
    check(n, n, d, 1, v, dtype, layout="tokens", bias=v != 200)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["first", "last", "slice"])
def test_layouts(dtype, layout):
    check(4, 9, 100, 64, 313, dtype, layout=layout, ignored=0.5, weighted=True)
