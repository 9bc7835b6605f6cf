"""Timing cases of the training operators, over their range of use.

Four kinds of case:

  score  ``linear_xent_fwd``: softmax cross entropy of a linear (1x1) head over
         ``v`` classes, forward only, as an evaluation pass calls it: the loss, and
         each token's log-sum-exp (0 where ignored) with the loss's divisor behind.
  step   ``linear_xent_step``: the same with its gradients, as a training step
         calls it.  Features are channels first, ``n`` x ``d`` x ``hw``: pixels of
         a feature map, or single tokens where ``hw`` is 1.
  ortho  ``orthogonalize``: a list of updates orthogonalised by Newton-Schulz
         products.
  muon   ``muon_step``: momentum, orthogonalised update and weight step of a list
         of layers; pruned 3x3 layers stay on their kept taps.

``shapes`` lists matrices as "rows x columns x count", joined by commas; for muon,
columns are input channels times taps, and a trailing "p" marks a pruned 3x3 layer.

``own`` false: the operators written out in elementary torch operations in 32 bits.
``own`` true: the library's entry points.  ``exact``: the same in 64 bits, the loss
by automatic differentiation and the orthogonalisation as a polynomial of the Gram
matrix of the input.
"""
from __future__ import annotations

import math

import torch

own = False

IGNORE = -100
COEFFS = (3.4445, -4.7750, 2.0315)
STEPS = 5
EPS = 1e-7
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _xent(name, kind, n, d, hw, v, dtype, *, bias=True, weighted=False, ignored=0.0, reduction="mean"):
    return dict(name=name, kind=kind, n=n, d=d, hw=hw, v=v, dtype=dtype, bias=bias, weighted=weighted,
                ignored=ignored, reduction=reduction)


def _mats(name, kind, shapes, dtype):
    return dict(name=name, kind=kind, shapes=shapes, dtype=dtype)


# the pruned layers of VGG-16 and of the colourization network (c_out x 9 c_in x how many)
VGG = "64x576x1p,128x576x1p,128x1152x1p,256x1152x1p,256x2304x2p,512x2304x1p,512x4608x5p"
COLOR = "64x576x1p,128x576x1p,128x1152x1p,256x1152x1p,256x2304x4p,512x2304x1p,512x4608x5p"


def listed():
    return [
        # one feature vector scored against a thousand classes: launches and host time count
        _xent("score_1_bf16", "score", 1, 512, 1, 1000, "bf16"),
        # an evaluation pass over a large vocabulary: four thousand tokens
        _xent("score_vocab_bf16", "score", 4096, 1024, 1, 32768, "bf16", bias=False, ignored=0.02),
        # the colourization head's training step: 8 images of 64 x 64 pixels, 313 colour bins, rebalanced classes
        _xent("color_b8_bf16", "step", 8, 256, 4096, 313, "bf16", weighted=True, ignored=0.05),
        # the same head for a batch of 2 in fp32
        _xent("color_b2_f32", "step", 2, 256, 4096, 313, "f32", weighted=True, ignored=0.05),
        # a training step over a large vocabulary, the largest call
        _xent("vocab_bf16", "step", 8192, 1024, 1, 50000, "bf16", bias=False, ignored=0.02),
        # sizes that divide by nothing, a loss and an incoming gradient for each token
        _xent("ragged_f32", "step", 777, 203, 1, 5003, "f32", ignored=0.1, reduction="none"),
        # one update of the smallest pruned layer (16 -> 16): latency
        _mats("ortho_16x144_f32", "ortho", "16x144x1", "f32"),
        # one large square projection's update in bf16
        _mats("ortho_4096_bf16", "ortho", "4096x4096x1", "bf16"),
        # a few updates of odd sizes, taller than wide among them
        _mats("ortho_ragged_f32", "ortho", "1000x513x2,313x256x1,77x1201x1", "f32"),
        # the step of the colourization head alone
        _mats("muon_head_f32", "muon", "313x256x1", "f32"),
        # the step of all pruned VGG-16 layers at once, fp32 and kept on their patterns
        _mats("muon_vgg_f32", "muon", VGG, "f32"),
        # the step of all pruned colourization layers in bf16
        _mats("muon_color_bf16", "muon", COLOR, "bf16"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("score", "step", "step", "ortho", "muon"))
    dtype = rng.choice(("bf16", "f32"))
    if kind in ("score", "step"):
        d = _logint(rng, 48, 2048)
        if rng.random() < 0.5:
            d = max(64, d // 64 * 64)
        if rng.random() < 0.5:      # pixels
            n, hw, v = rng.randint(1, 8), _logint(rng, 49, 4096), _logint(rng, 100, 2000)
        else:                       # tokens
            n, hw, v = _logint(rng, 1, 8192), 1, _logint(rng, 500, 50000)
        most = 3e11 if dtype == "bf16" else 6e10   # n hw v d; the largest listed has 4.2e11
        v = max(100, min(v, int(most / (n * hw * d))))
        return _xent("", kind, n, d, hw, v, dtype, bias=rng.random() < 0.5, weighted=rng.random() < 0.5,
                     ignored=rng.choice((0.0, 0.1)), reduction=rng.choice(("mean", "mean", "sum", "none")))
    shapes = []
    for _ in range(rng.randint(1, 6)):
        if kind == "muon" and rng.random() < 0.5:
            shapes.append("%dx%dx%dp" % (_logint(rng, 16, 512), 9 * _logint(rng, 16, 512), rng.randint(1, 3)))
        else:
            top = 4096 if dtype == "bf16" and not shapes else 1024
            shapes.append("%dx%dx1" % (_logint(rng, 16, top), _logint(rng, 16, top)))
    return _mats("", kind, ",".join(shapes), dtype)


def _shapes(case):
    """[(rows, columns, pruned)] of a case, in order."""
    got = []
    for s in case["shapes"].split(","):
        r, c, k = s.rstrip("p").split("x")
        got += [(int(r), int(c), s.endswith("p"))] * int(k)
    return got


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    if case["kind"] in ("score", "step"):
        n, d, hw, v = case["n"], case["d"], case["hw"], case["v"]
        target = torch.randint(0, v, (n, hw), generator=g, device="cuda")
        # logits of standard deviation 2 about a part that knows the target: what a head under training sees
        w = normal(v, d) * (2.0 / math.sqrt(d))
        x = normal(n, d, hw) + 0.5 * w[target].transpose(1, 2)
        drop = uniform(n, hw) < case["ignored"]
        s = dict(case=case, x=x.to(dt), w=w.to(dt), target=torch.where(drop, torch.full_like(target, IGNORE), target))
        s["bias"] = 0.1 * normal(v) if case["bias"] else None
        s["class_weight"] = 0.5 + uniform(v) if case["weighted"] else None
        s["grad"] = uniform(n, hw) if case["kind"] == "step" and case["reduction"] == "none" else None
        if hw == 1:
            s["x"] = s["x"].reshape(n, d)
            s["target"] = s["target"].reshape(n)
            s["grad"] = None if s["grad"] is None else s["grad"].reshape(n)
        return s

    grads, weights, momenta, keep = [], [], [], []
    # four taps of nine, all with the centre; half of the kernels kept
    masks = torch.tensor([0x03A, 0x0B2, 0x0B8, 0x09A, 0x01B, 0x036, 0x0D8, 0x1B0], device="cuda")
    for r, c, pruned in _shapes(case):
        # gradients have a few strong directions and a broad rest
        k = min(r, c, 16)
        u = normal(r, c) / math.sqrt(c) + normal(r, k) @ normal(k, c) / math.sqrt(k * c)
        if case["kind"] == "ortho":
            grads.append(u.to(dt))
            continue
        shape = (r, c // 9, 3, 3) if pruned else (r, c)
        kept = None
        w = normal(r, c) * math.sqrt(2.0 / c)
        m = u + 0.3 * normal(r, c) / math.sqrt(c)
        if pruned:
            kept = masks[torch.randint(0, 8, (r, c // 9), generator=g, device="cuda")]
            kept = torch.where(uniform(r, c // 9) < 0.5, kept, torch.zeros_like(kept))
            on = _on(kept).reshape(r, c)
            w, m = w * on, m * on
            kept = kept.to(torch.int16)
        grads.append(u.to(dt).reshape(shape))
        weights.append(w.to(dt).reshape(shape))
        momenta.append((8.0 * m).reshape(shape))
        keep.append(kept)
    s = dict(case=case, grads=grads)
    if case["kind"] == "muon":
        s.update(weights=weights, momenta=momenta, keep=keep,
                 out=([torch.empty_like(w) for w in weights], [torch.empty_like(m) for m in momenta]))
    return s


def _on(kept):
    """Tap masks [o][c] -> 0/1 fp32 [o][c][9]."""
    taps = torch.arange(9, device=kept.device)
    return ((kept.to(torch.int64)[..., None] >> taps) & 1).float()


# ---------------------------------------------------------------------------
# the operators in their plain form
# ---------------------------------------------------------------------------

def _tokens(x):
    """Features [n][d][...] -> [tokens][d] in 32 bits."""
    return x.float() if x.dim() == 2 else x.float().transpose(1, 2).reshape(-1, x.shape[1])


def _plain_xent(s):
    case = s["case"]
    x, w, y = _tokens(s["x"]), s["w"].float(), s["target"].reshape(-1)
    keep = y != IGNORE
    at = torch.where(keep, y, torch.zeros_like(y))
    x = torch.where(keep[:, None], x, torch.zeros_like(x))
    logits = x @ w.t()
    if s["bias"] is not None:
        logits += s["bias"]
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    z = e.sum(1, keepdim=True)
    lse = (top + torch.log(z))[:, 0]
    cw = keep.float()
    if s["class_weight"] is not None:
        cw = cw * s["class_weight"][at]
    loss = cw * (lse - logits.gather(1, at[:, None])[:, 0])
    den = cw.sum() if case["reduction"] == "mean" else torch.ones((), device=x.device)
    den = torch.where(den > 0, den, torch.ones_like(den))
    out = loss.reshape(s["target"].shape) if case["reduction"] == "none" else loss.sum() / den
    if case["kind"] == "score":
        return out, torch.cat([torch.where(keep, lse, torch.zeros_like(lse)), den.reshape(1)])
    scale = cw / den
    if s["grad"] is not None:
        scale = scale * s["grad"].reshape(-1)
    p = e / z
    p.scatter_add_(1, at[:, None], torch.full_like(p[:, :1], -1.0))
    p *= scale[:, None]
    dx = p @ w
    if s["x"].dim() == 3:
        dx = dx.reshape(case["n"], case["hw"], case["d"]).transpose(1, 2).contiguous()
    dw = p.t() @ x
    db = p.sum(0) if s["bias"] is not None else None
    return out, dx.to(s["x"].dtype), dw.to(s["w"].dtype), db


def _plain_ortho(u):
    x = u.float()
    x = x / (torch.sqrt((x * x).sum()) + EPS)
    if u.shape[0] > u.shape[1]:
        x = x.t()
    a, b, c = COEFFS
    for _ in range(STEPS):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def _plain_muon(w, g, m, kept):
    r = w.shape[0]
    on = 1.0 if kept is None else _on(kept).reshape(r, -1)
    g = g.float().reshape(r, -1) * on
    m = MOMENTUM * m.reshape(r, -1) + g
    o = _plain_ortho(g + MOMENTUM * m)
    up = LR * math.sqrt(max(1.0, r / o.shape[1]))
    new = ((1.0 - LR * DECAY) * w.float().reshape(r, -1) - up * o) * on
    return new.reshape(w.shape).to(w.dtype), (m * on).reshape(w.shape)


def run(s):
    case = s["case"]
    if own:
        import paper_2004_11250_amd as pp
        if case["kind"] in ("score", "step"):
            more = dict(bias=s["bias"], class_weight=s["class_weight"], ignore_index=IGNORE,
                        reduction=case["reduction"])
            if case["kind"] == "score":
                return pp.linear_xent_fwd(s["x"], s["w"], s["target"], **more)
            return pp.linear_xent_step(s["x"], s["w"], s["target"], grad=s["grad"], **more)
        if case["kind"] == "ortho":
            return pp.orthogonalize(s["grads"], steps=STEPS, coeffs=COEFFS, eps=EPS)
        return pp.muon_step(s["weights"], s["grads"], s["momenta"], lr=LR, momentum=MOMENTUM, nesterov=True,
                            weight_decay=DECAY, keep=s["keep"], steps=STEPS, coeffs=COEFFS, eps=EPS, out=s["out"])
    if case["kind"] in ("score", "step"):
        return _plain_xent(s)
    if case["kind"] == "ortho":
        return [_plain_ortho(u).to(u.dtype).contiguous() for u in s["grads"]]
    got = [_plain_muon(*v) for v in zip(s["weights"], s["grads"], s["momenta"], s["keep"])]
    return [v[0] for v in got], [v[1] for v in got]


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def _exact_xent(s):
    case = s["case"]
    y = s["target"].reshape(-1)
    rows = torch.nonzero(y != IGNORE)[:, 0]
    feats = s["x"] if s["x"].dim() == 2 else s["x"].permute(0, 2, 1).reshape(-1, case["d"])
    x = feats[rows].double().requires_grad_()
    w = s["w"].double().requires_grad_()
    b = None if s["bias"] is None else s["bias"].double().requires_grad_()
    z = torch.nn.functional.linear(x, w, b)
    each = -torch.log_softmax(z, 1)[torch.arange(len(rows), device=x.device), y[rows]]
    cw = torch.ones_like(each) if s["class_weight"] is None else s["class_weight"].double()[y[rows]]
    each = each * cw
    if case["reduction"] == "none":
        loss = torch.zeros(y.shape, dtype=torch.float64, device=x.device)
        loss[rows] = each.detach()
        loss = loss.reshape(s["target"].shape)
        g = torch.ones_like(each) if s["grad"] is None else s["grad"].double().reshape(-1)[rows]
        total = (each * g).sum()
    else:
        total = each.sum() / (cw.sum() if case["reduction"] == "mean" and len(rows) else 1.0)
        loss = total.detach()
    if case["kind"] == "score":
        stats = torch.zeros(len(y) + 1, dtype=torch.float64, device=x.device)
        stats[rows] = torch.logsumexp(z.detach(), 1)
        stats[-1] = cw.sum() if case["reduction"] == "mean" and len(rows) else 1.0
        return loss, stats
    got = torch.autograd.grad(total, [x, w] + ([] if b is None else [b]))
    dx = torch.zeros(feats.shape, dtype=torch.float64, device=x.device)
    dx[rows] = got[0]
    if s["x"].dim() == 3:
        dx = dx.reshape(case["n"], case["hw"], case["d"]).permute(0, 2, 1).contiguous()
    return loss, dx, got[1], (got[2] if b is not None else None)


def _exact_ortho(u):
    """p(U U^T) U: every Newton-Schulz step multiplies by a polynomial of the first Gram matrix."""
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / (torch.linalg.vector_norm(x) + EPS)
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    a, b, c = COEFFS
    gram, product = x @ x.T.contiguous(), eye
    for _ in range(STEPS):
        q = a * eye + b * gram + c * gram.matmul(gram)
        product, gram = q @ product, q @ gram @ q
    x = product @ x
    return x.T if tall else x


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("score", "step"):
        return _exact_xent(s)
    if case["kind"] == "ortho":
        return [_exact_ortho(u).contiguous() for u in s["grads"]]
    weights, momenta = [], []
    for w, g, m, kept in zip(s["weights"], s["grads"], s["momenta"], s["keep"]):
        flat = (w.shape[0], w.numel() // w.shape[0])
        on = torch.ones(flat, dtype=torch.bool, device=w.device)
        if kept is not None:
            on = torch.stack([(kept >> t) & 1 for t in range(9)], -1).reshape(flat) != 0
        g = g.double().reshape(flat).masked_fill(~on, 0.0)
        m = g + MOMENTUM * m.double().reshape(flat)
        step = _exact_ortho(g + MOMENTUM * m) * (LR * math.sqrt(max(1.0, flat[0] / flat[1])))
        w = w.double().reshape(flat)
        weights.append((w - LR * DECAY * w - step).masked_fill(~on, 0.0).reshape(g.shape[0], *kept.shape[1:], 3, 3)
                       if kept is not None else w - LR * DECAY * w - step)
        momenta.append(m.masked_fill(~on, 0.0).reshape(weights[-1].shape))
    return weights, momenta


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("score", "step"):
        t, d, v = case["n"] * case["hw"], case["d"], case["v"]
        moved = size * (t * d + v * d) + 8 * t + 4 * v * (case["bias"] + case["weighted"])
        moved += 4 * t if case["reduction"] == "none" else 4
        if case["kind"] == "score":
            return {"bytes": moved, "flops": 2 * t * d * v}
        # the logits once, and the two products of the gradient
        moved += size * (t * d + v * d) + 4 * v * case["bias"] + (4 * t if case["reduction"] == "none" else 0)
        return {"bytes": moved, "flops": 6 * t * d * v}
    moved = flops = 0
    for r, c, pruned in _shapes(case):
        m, n = min(r, c), max(r, c)
        # the Gram matrix and its square are symmetric: one triangle each; then the product with the matrix
        flops += STEPS * (m * m * n + m ** 3 + 2 * m * m * n)
        moved += 2 * size * r * c
        if case["kind"] == "muon":
            moved += (size + 8) * r * c + (2 * r * c // 9 if pruned else 0)
    return {"bytes": moved, "flops": flops}
