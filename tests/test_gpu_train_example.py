"""The training operators run together: the example's loss falls and its pruned
layer stays on its patterns."""
import os
import sys

import pytest

pp = pytest.importorskip("paper_2004_11250_amd")
pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_loss_falls_and_the_layer_stays_pruned():
    import train_pruned_head as ex
    losses, w, on = ex.train(steps=8)
    assert max(losses) == losses[0], losses
    assert losses[-1] < 0.7 * losses[0], losses
    assert bool((w[~on] == 0).all()) and float((w[on] != 0).float().mean()) > 0.99
