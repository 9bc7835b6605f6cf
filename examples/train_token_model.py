"""A small token model trained on the GPU: a table of embeddings that is the head's
weights too, one layer between, and the next token as the target.

    python examples/train_token_model.py [steps]

Each step looks the tokens up (pp.embed_fwd), runs the layer, takes the loss with
the head's gradients (pp.linear_xent_step), adds the lookup's gradient to the
head's (pp.embed_bwd), and makes one clipped AdamW step (pp.grad_norm,
pp.adamw_step): the table's moments in 8 bits, the others' in 32.  After the first
step, whose launches are eager, the whole step is one recorded HIP graph: the step
count and the clipping factor stay on the GPU.  Prints the loss of each step.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2004_11250_amd as pp   # noqa: E402

VOCAB, WIDTH, TOKENS, PAD = 1000, 128, 512, 0


class Model:
    def __init__(self, seed=1):
        g = torch.Generator("cuda").manual_seed(seed)

        def normal(*shape):
            return torch.randn(shape, generator=g, device="cuda")

        self.table = normal(VOCAB, WIDTH) * 0.05
        self.w = normal(WIDTH, WIDTH) / WIDTH ** 0.5
        self.bias = torch.zeros(VOCAB, device="cuda")
        self.step = torch.zeros((), dtype=torch.int64, device="cuda")
        self.table_state = pp.AdamWState(self.table, bits=8)
        self.state = pp.AdamWState([self.w, self.bias])

    def gradients(self, ids, target):
        """The loss, and the gradients of table, w and bias."""
        scale = WIDTH ** 0.5
        x = pp.embed_fwd(ids, self.table, scale=scale, ignore_index=PAD)
        z = x @ self.w.t()
        loss, dh, dhead, dbias = pp.linear_xent_step(torch.relu(z), self.table, target, bias=self.bias, ignore_index=PAD)
        dz = torch.where(z > 0, dh, 0.0)
        dtable = pp.embed_bwd(ids, dz @ self.w, VOCAB, scale=scale, ignore_index=PAD, add=dhead, out=dhead)
        return loss, [dtable, dz.t() @ x, dbias]

    def update(self, grads, lr):
        _, factor = pp.grad_norm(grads, max_norm=1.0)
        self.step += torch.isfinite(factor)         # (where it is not, no step is taken, and none counts)
        more = dict(lr=lr, step=self.step, grad_scale=factor)
        pp.adamw_step([self.table], grads[:1], self.table_state, weight_decay=0.01, **more)
        pp.adamw_step([self.w, self.bias], grads[1:], self.state, weight_decay=[0.01, 0.0], **more)

    def train_step(self, ids, target, lr):
        loss, grads = self.gradients(ids, target)
        self.update(grads, lr)
        return loss


def batch(seed):
    """Tokens of a chain in which each token has two likely followers; some are padding."""
    g = torch.Generator("cuda").manual_seed(seed)
    coin, ids = torch.rand(TOKENS, generator=g, device="cuda"), torch.randint(1, VOCAB, (TOKENS,), generator=g, device="cuda")
    ids = torch.where(coin < 0.1, PAD, ids)
    target = 1 + (ids * 7 + torch.where(coin < 0.7, 3, 11)) % (VOCAB - 1)
    return ids, torch.where(ids == PAD, PAD, target)


def train(steps=20, lr=3e-3, seed=1, graph=True):
    """The losses, and the model."""
    model = Model(seed)
    ids, target = batch(0)
    losses, recorded, loss = [], None, None
    for k in range(steps):
        new = batch(k)
        ids.copy_(new[0])
        target.copy_(new[1])
        if recorded is not None:
            recorded.replay()
        else:
            loss = model.train_step(ids, target, lr)
        losses.append(float(loss))
        if graph and recorded is None:
            recorded = torch.cuda.CUDAGraph()
            with torch.cuda.graph(recorded):
                loss = model.train_step(ids, target, lr)
    return losses, model


if __name__ == "__main__":
    for i, v in enumerate(train(int(sys.argv[1]) if len(sys.argv) > 1 else 20)[0]):
        print(f"step {i:3d}  loss {v:.4f}", flush=True)
