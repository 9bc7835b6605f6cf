"""A training step around the pruning projections: the end of the colourization
network (a pruned 3x3 layer, ReLU, and the 1x1 head over 313 colour bins) is
fine-tuned with the layer kept on its patterns.

    python examples/train_pruned_head.py [steps]

Each step runs the pruned layer (pp.conv2d_fwd), the head's softmax cross entropy
with its gradients (pp.linear_xent_step), the layer's weight gradient (nine
products in torch), and one orthogonalised weight step of both layers
(pp.muon_step, the pruned one with its tap masks), then packs the layer's new
weights for the next step.  The targets come from a network of the same shape
with other weights.  Prints the loss of each step.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2004_11250_amd as pp   # noqa: E402
import workloads   # noqa: E402

CHANNELS, BINS, SIZE, BATCH = 256, 313, 32, 4


def weights(seed):
    """A pruned 3x3 layer (keep ratio and patterns of the colourization network) and a head."""
    g = np.random.default_rng(seed)
    w = g.normal(0.0, np.sqrt(2.0 / (CHANNELS * 9 * 0.3 * 4 / 9)), (CHANNELS, CHANNELS, 3, 3)).astype(np.float32)
    pid, energy = pp.project_patterns(w, workloads.CANON8)
    conn = pp.project_connectivity(energy, int(0.3 * CHANNELS * CHANNELS))
    head = g.normal(0.0, 4.0 / np.sqrt(CHANNELS), (BINS, CHANNELS)).astype(np.float32)
    return w, pid, conn, torch.from_numpy(head).cuda()


def layer_of(w, pid, conn):
    return pp.PackedLayer.from_weights(w, None, pid, conn, workloads.CANON8, device="cuda")


def weight_gradient(x, dy):
    """Gradient of a 3x3 convolution's weights (stride 1, padding 1): one product a tap."""
    n, c, h, w = x.shape
    rows = dy.permute(1, 0, 2, 3).reshape(dy.shape[1], -1)
    xp = torch.nn.functional.pad(x, (1, 1, 1, 1))
    taps = [rows @ xp[:, :, i:i + h, j:j + w].permute(0, 2, 3, 1).reshape(-1, c) for i in range(3) for j in range(3)]
    return torch.stack(taps, -1).reshape(dy.shape[1], c, 3, 3)


def train(steps=12, lr=0.02, seed=1):
    """The losses, and the fine-tuned weights with the layer's tap masks."""
    w, pid, conn, head = weights(seed)
    keep = torch.from_numpy(pp.keep_masks(pid, conn, workloads.CANON8)).cuda()
    on = torch.stack([(keep.long() >> t) & 1 for t in range(9)], -1).reshape(w.shape).bool()
    w = torch.from_numpy(w).cuda() * on
    x = torch.rand(BATCH, CHANNELS, SIZE, SIZE, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")
    tw, tpid, tconn, thead = weights(seed + 100)
    features = pp.conv2d_fwd(layer_of(tw, tpid, tconn), x, relu=True)
    target = torch.einsum("vc,nchw->nvhw", thead, features).argmax(1)

    momenta = [torch.zeros_like(w), torch.zeros_like(head)]
    bias, losses = torch.zeros(BINS, device="cuda"), []
    for _ in range(steps):
        features = pp.conv2d_fwd(layer_of(w.cpu().numpy(), pid, conn), x, relu=True)
        loss, dfeatures, dhead, dbias = pp.linear_xent_step(features, head, target, bias=bias)
        dw = weight_gradient(x, torch.where(features > 0, dfeatures, torch.zeros_like(dfeatures)))
        pp.muon_step([w, head], [dw, dhead], momenta, lr=lr, keep=[keep, None])
        bias -= 10.0 * lr * dbias
        losses.append(float(loss))
    return losses, w, on


if __name__ == "__main__":
    for i, v in enumerate(train(int(sys.argv[1]) if len(sys.argv) > 1 else 12)[0]):
        print(f"step {i:3d}  loss {v:.4f}", flush=True)
