"""Lists of matrices whose outputs are not each their own are refused: a list's
matrices are read and written in no order."""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")


def refused(match):
    return pytest.raises(ValueError, match=match)


def test_updates():
    a, b, c = (torch.zeros(8, 8) for _ in range(3))
    with refused("another matrix's input"):
        pp.orthogonalize([a, b], out=[b, a])
    with refused("another matrix's input"):
        pp.orthogonalize([a, b], out=[c, a])
    with refused("the same tensor"):
        pp.orthogonalize([a, b], out=[c, c])
    with refused("GPU"):     # each its own, one input twice, empty ones: well formed, but not on a GPU
        pp.orthogonalize([a, b], out=[a, b])
    with refused("GPU"):
        pp.orthogonalize([a, a], out=[b, c])
    with refused("GPU"):
        e = torch.zeros(0, 8)
        pp.orthogonalize([e, e], out=[e, e])
    with refused("GPU"):     # halves of one matrix
        pp.orthogonalize([a[:, :4], a[:, 4:]], out=[a[:, :4], a[:, 4:]])


def test_weight_steps():
    w, g, m, w2, m2, x = (torch.zeros(8, 8) for _ in range(6))
    with refused("the same tensor"):
        pp.muon_step([w, w], [g, g], [m, m2], lr=0.1)
    with refused("the same tensor"):
        pp.muon_step([w, w2], [g, g], [m, m], lr=0.1)
    with refused("another matrix's input"):
        pp.muon_step([w, w2], [g, g], [m, m2], lr=0.1, out=([w2, w], [m, m2]))
    with refused("another matrix's input"):
        pp.muon_step(w, g, m, lr=0.1, out=(m, x))
    with refused("another tensor"):
        pp.muon_step(w, g, m, lr=0.1, out=(g, m))
    for out in (None, ([w, w2], [m, m2]), ([x, w2], [m, m2])):
        with refused("GPU"):
            pp.muon_step([w, w2], [g, g], [m, m2], lr=0.1, out=out)


def test_outputs_that_share_their_elements():
    u = torch.zeros(8, 8)
    for out in (torch.zeros(8, 1).expand(8, 8), torch.zeros(1, 8).expand(8, 8), torch.zeros(1, 1).expand(8, 8)):
        with refused("share their memory"):
            pp.orthogonalize(u, out=out)
        with refused("GPU"):      # (an input may)
            pp.orthogonalize(out)
    with refused("GPU"):
        pp.orthogonalize(torch.zeros(1, 8), out=torch.zeros(8).expand(1, 8))
