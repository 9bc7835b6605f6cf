"""The loss of tokens that are nearly sure of their class: log(1 + e^-gap), however
large the logits are.

Two classes a token have a finite bias, and features are one channel of one each,
so logits are exact, the sum of exponentials has two terms that are not 0 (1 and
e^-gap, the latter within 2e-6 of itself), one addition of them (2^-24), and its
logarithm is within two units in its last place: 2^-24 + 3e-6 of the loss where
the target is the larger one; where it is the other, the gap is added, one
rounding more (2^-24 of the loss).
"""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
from test_gpu_xent import DT, near   # noqa: E402

pytestmark = pytest.mark.gpu

GAPS = [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 15, 20, 40]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0, 40, -96, 240])
@pytest.mark.parametrize("n,v", [(1, 300), (17, 3300), (64, 12300), (130, 70), (600, 313), (700, 3000)])
def test_loss(dtype, top, n, v):
    d, one, two = len(GAPS), v // 3, v - 2
    gap = torch.tensor(GAPS, dtype=torch.float64, device="cuda")
    w = torch.zeros(v, d, device="cuda")
    w[one], w[two] = top, top - gap.float()
    x = torch.eye(d, device="cuda").repeat(n // d + 1, 1)[:n].contiguous()
    b = torch.full((v,), -float("inf"), device="cuda")
    b[one] = b[two] = 0.0
    t = torch.where(torch.arange(n, device="cuda") % 5 == 4, two, one)
    gap = gap.repeat(n // d + 1)[:n]
    want = torch.log1p(torch.exp(-gap)) + torch.where(t == two, gap, torch.zeros_like(gap))
    lim = 2.0 ** -24 + (3e-6 + 2.0 ** -24) * want
    x, w = x.to(DT[dtype]), w.to(DT[dtype])
    assert torch.equal(w[two].float(), top - torch.tensor(GAPS, device="cuda"))
    loss, stats = pp.linear_xent_fwd(x, w, t, bias=b, reduction="none")
    near(loss, want, lim, "loss")
    # (the statistics hold the log-sum-exp in fp32)
    near(stats[:-1], top + torch.log1p(torch.exp(-gap)), lim + 2.0 ** -24 * (abs(top) + 1), "lse")
    near(pp.linear_xent_step(x, w, t, bias=b, reduction="none")[0], want, lim, "loss of a step")
    mean, _ = pp.linear_xent_fwd(x, w, t, bias=b)
    near(mean, want.mean(), lim.mean() + 2.0 ** -23 * want.mean(), "mean")
