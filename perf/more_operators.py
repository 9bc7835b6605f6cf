"""Timing cases of the operators around a table of embeddings and of the weight
step of every other parameter, over their range of use.

Four kinds of case:

  look   ``embed_fwd``: rows of a ``v`` x ``d`` table by ids, times a scale.
  grad   ``embed_bwd``: the table's gradient from its features' gradient, added
         to another gradient of the table where ``add`` is set (a table that is
         the head's weights too).
  adamw  ``adamw_step``: one AdamW step of a list of tensors, their moments held
         in 32 bits or in 8.
  norm   ``grad_norm``: the norm of a list of gradients, and the factor that
         brings it to ``MAX_NORM`` at most.

``ids`` says how ids are spread: "text" log-uniform (token ids sorted by how often
they occur), "pixels" (colour bins: three in ten are one bin, the others normal
about it), "uniform".  ``shapes`` lists tensors as "rows x columns x count" (or
"size x count"), joined by commas; a trailing "p" marks a pruned 3x3 layer, whose
columns are input channels times taps.  Pruned layers come first.

All tensors of a list are views of one buffer, each from a multiple of 128
elements on, with zeros between; outputs are such buffers too.  Moments of 8 bits
are returned as the bfloat16 values that they stand for:

  first   blocks of 128 elements: code (e4m3) times the block's scale, which is
          its largest magnitude / 448
  second  blocks of 128 elements: the square of (value of the code times the
          block's scale), the scale being the block's largest square root; code c
          above 0 is 2^(q / 16 - 127) (1 + (q mod 16) / 16) with q = c + 1777
          (integer division: 4 bits of the exponent, 4 of the mantissa), code 0
          is 0.  A value above 0 has a code above 0.

``own`` false: the operators written out in elementary torch operations.  ``own``
true: the library's entry points.  ``exact``: the same in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

IGNORE = -100
BETAS, EPS, LR, DECAY = (0.9, 0.999), 1e-8, 1e-3, 0.01
MAX_NORM = 1.0
BLOCK = 128
TINY = 2.0 ** -100        # the least scale
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _embed(name, kind, t, v, d, w, y, *, ids="uniform", scale=1.0, ignored=0.0, add=False):
    return dict(name=name, kind=kind, t=t, v=v, d=d, w=w, y=y, ids=ids, scale=scale, ignored=ignored, add=add)


def _adamw(name, shapes, w, g, bits, *, step=1000, copies=False, device=False):
    return dict(name=name, kind="adamw", shapes=shapes, w=w, g=g, bits=bits, step=step, copies=copies, device=device)


def _norm(name, shapes, g):
    return dict(name=name, kind="norm", shapes=shapes, g=g)


# VGG-16: the pruned layers (c_out x 9 c_in x how many), the first layer, the biases
VGG = ("64x576x1p,128x576x1p,128x1152x1p,256x1152x1p,256x2304x2p,512x2304x1p,512x4608x5p,"
       "64x27x1,64x2,128x2,256x3,512x6")
# 24 blocks of a projection up, one square, and a vector
BLOCKS = "512x2048x24,512x512x24,512x24"


def listed():
    return [
        # one token of a generating loop: launch and host time count
        _embed("look_1_bf16", "look", 1, 50000, 1024, "bf16", "bf16", ids="text", scale=32.0),
        # the tokens of a training batch
        _embed("look_vocab_bf16", "look", 8192, 50000, 1024, "bf16", "bf16", ids="text", scale=32.0),
        # the same batch's gradient of the whole table
        _embed("grad_vocab_bf16", "grad", 8192, 50000, 1024, "bf16", "bf16", ids="text", scale=32.0),
        # colour bins of 8 images of 64 x 64 pixels: few rows, one of which has a third of all pixels
        _embed("grad_color_bf16", "grad", 32768, 313, 256, "bf16", "bf16", ids="pixels", scale=16.0, ignored=0.05),
        # a table that is the head's weights as well: the gradient is added to the head's, a long batch
        _embed("grad_tied_bf16", "grad", 32768, 50000, 1024, "bf16", "bf16", ids="text", add=True),
        # sizes that divide by nothing, fp32
        _embed("grad_ragged_f32", "grad", 777, 5003, 203, "f32", "f32", ids="text", ignored=0.1),
        # the colourization head alone: latency
        _adamw("adamw_head_f32", "313x256x1,313x1", "f32", "f32", 32),
        # all of VGG-16's convolutions and biases, the pruned ones kept on their patterns
        _adamw("adamw_vgg_f32", VGG, "f32", "f32", 32),
        # a table and a head over a large vocabulary in bf16, moments in 8 bits: the largest call
        _adamw("adamw_vocab_bf16_8", "50000x1024x2", "bf16", "bf16", 8),
        # 72 tensors held in fp32 with bf16 copies for the next forward pass, moments in 8 bits, step and scale on the device
        _adamw("adamw_blocks_f32_8", BLOCKS, "f32", "bf16", 8, copies=True, device=True),
        # the norms of the same lists
        _norm("norm_vgg_f32", VGG, "f32"),
        _norm("norm_blocks_bf16", BLOCKS, "bf16"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("look", "grad", "grad", "adamw", "adamw", "norm"))
    if kind in ("look", "grad"):
        t, v, d = _logint(rng, 1, 65536), _logint(rng, 50, 200000), _logint(rng, 32, 4096)
        if rng.random() < 0.5:
            d = max(32, d // 64 * 64)
        v = max(50, min(v, int(6e7 / d)))
        t = max(1, min(t, int(6e7 / d)))
        w, y = rng.choice((("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")))
        return _embed("", kind, t, v, d, w, y, ids=rng.choice(("text", "text", "pixels", "uniform")),
                      scale=rng.choice((1.0, 16.0, 0.1)), ignored=rng.choice((0.0, 0.1)),
                      add=kind == "grad" and rng.random() < 0.3)
    shapes, left = [], 4e7
    for _ in range(rng.randint(1, 8)):
        if kind == "adamw" and rng.random() < 0.3:
            r, c, k = 16 * rng.randint(1, 32), 72 * rng.randint(1, 64), rng.randint(1, 3)
            s = "%dx%dx%dp" % (r, c, k)
        elif rng.random() < 0.3:
            r, c, k = 1, _logint(rng, 1, 5000), rng.randint(1, 30)
            s = "%dx%d" % (c, k)
        else:
            r, c, k = _logint(rng, 3, 20000), _logint(rng, 5, 3000), rng.randint(1, 4)
            s = "%dx%dx%d" % (r, c, k)
        if r * c * k <= left:
            left -= r * c * k
            shapes.append(s)
    shapes = ",".join(sorted(shapes or ["313x1"], key=lambda s: not s.endswith("p")))
    if kind == "norm":
        return _norm("", shapes, rng.choice(("f32", "bf16")))
    w, g = rng.choice((("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")))
    return _adamw("", shapes, w, g, rng.choice((32, 8)), step=_logint(rng, 1, 100000),
                  copies=w == "f32" and rng.random() < 0.5, device=rng.random() < 0.5)


def _shapes(case):
    """[(shape, pruned)] of a case, in order."""
    got = []
    for s in case["shapes"].split(","):
        *size, k = (int(n) for n in s.rstrip("p").split("x"))
        pruned = s.endswith("p")
        got += [((size[0], size[1] // 9, 3, 3) if pruned else tuple(size), pruned)] * k
    return got


def _places(shapes):
    """Where each tensor of a list begins in its buffer, and the buffer's size."""
    at, total = [], 0
    for shape in shapes:
        at.append(total)
        total += -(-math.prod(shape) // BLOCK) * BLOCK
    return at, total


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 31)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    if case["kind"] in ("look", "grad"):
        t, v, d = case["t"], case["v"], case["d"]
        if case["ids"] == "text":
            ids = torch.exp(uniform(t).double() * math.log(v + 1.0)).long() - 1
        elif case["ids"] == "pixels":
            ids = torch.where(uniform(t) < 0.3, torch.zeros((), device="cuda"), normal(t) * v / 6).long() + v // 2
        else:
            ids = torch.randint(0, v, (t,), generator=g, device="cuda")
        ids = ids.clamp(0, v - 1)
        ids = torch.where(uniform(t) < case["ignored"], torch.full_like(ids, IGNORE), ids)
        s = dict(case=case, ids=ids)
        if case["kind"] == "look":
            s["w"] = (normal(v, d) / math.sqrt(d)).to(DTYPES[case["w"]])
        else:
            s["dy"] = (normal(t, d) / math.sqrt(t)).to(DTYPES[case["y"]])
            s["add"] = (normal(v, d) / math.sqrt(v)).to(DTYPES[case["w"]]) if case["add"] else None
        return s

    shapes = _shapes(case)
    at, total = _places([shape for shape, _ in shapes])

    def views(flat):
        return [flat[a:a + math.prod(shape)].view(shape) for a, (shape, _) in zip(at, shapes)]

    def inside():
        """1 at the tensors' elements, 0 between them."""
        on = torch.zeros(total, device="cuda")
        for one in views(on):
            one.fill_(1.0)
        return on

    grads = normal(total) * inside() * 1e-3
    for one in views(grads):
        if one.dim() > 1:     # rows (channels, tokens) differ in size, and some get no gradient
            r = one.shape[0]
            size = torch.exp(normal(r)) * (uniform(r) < 0.8)
            one *= size.reshape(r, *[1] * (one.dim() - 1))
    flat_g = grads.to(DTYPES[case["g"]])
    s = dict(case=case, flat_g=flat_g, g=views(flat_g))
    if case["kind"] == "norm":
        return s

    flat_w = (normal(total) * inside() * 0.02).to(DTYPES[case["w"]])
    # moments as some hundred steps of such gradients leave them
    m = (0.3 * grads + 0.2e-3 * normal(total)) * inside()
    v = (0.5 * grads.square() + 0.1e-6 * uniform(total)) * inside()
    pruned = [shape for shape, p in shapes if p]
    if pruned:
        # four taps of nine, all with the centre; half of the kernels kept
        masks = torch.tensor([0x03A, 0x0B2, 0x0B8, 0x09A, 0x01B, 0x036, 0x0D8, 0x1B0], device="cuda")
        cells = sum(math.prod(shape) for shape in pruned) // 9
        kept = masks[torch.randint(0, 8, (cells,), generator=g, device="cuda")]
        kept = torch.where(uniform(cells) < 0.5, kept, torch.zeros_like(kept)).to(torch.int16)
        n = 9 * cells
        on = _on(kept).reshape(-1)
        flat_w[:n] *= on.to(flat_w.dtype)
        m[:n] *= on
        v[:n] *= on
        s["flat_keep"], s["keep"], first = kept, [], 0
        for shape, p in shapes:
            n = math.prod(shape) // 9
            s["keep"].append(kept[first:first + n].view(shape[:2]) if p else None)
            first += n if p else 0
    else:
        s["flat_keep"], s["keep"] = None, None
    s.update(flat_w=flat_w, w=views(flat_w), w_out=torch.zeros_like(flat_w))
    s["copies"] = torch.zeros_like(flat_w, dtype=torch.bfloat16) if case["copies"] else None
    s["views"] = (views(s["w_out"]), views(s["copies"]) if case["copies"] else None)
    if case["device"]:
        s["step"] = torch.tensor(case["step"], dtype=torch.int64, device="cuda")
        s["scale"] = uniform(1)[0] * 0.5 + 0.5
    else:
        s["step"], s["scale"] = case["step"], None
    if case["bits"] == 8:
        s["moments"] = _encode(m, v)
    else:
        s["moments"] = (m, v)
    if own:
        import paper_2004_11250_amd as pp
        s["state"] = pp.AdamWState(s["w"], bits=case["bits"])
        s["state_out"] = pp.AdamWState(s["w"], bits=case["bits"])
        for name, t in zip(("m", "v", "m_scale", "v_scale"), s["moments"]):
            getattr(s["state"], name).copy_(t)
    return s


def _on(kept):
    """Tap masks [kernel] -> 0/1 fp32 [kernel][9]."""
    taps = torch.arange(9, device=kept.device)
    return ((kept.to(torch.int64)[..., None] >> taps) & 1).float()


# ---------------------------------------------------------------------------
# the operators in their plain form
# ---------------------------------------------------------------------------

def _encode(m, v):
    """Moments of 32 bits -> codes and scales."""
    m, r = m.view(-1, BLOCK), torch.sqrt(v).view(-1, BLOCK)
    ms = (m.abs().amax(1) / 448.0).clamp(min=TINY)
    vs = r.amax(1).clamp(min=TINY)
    mc = (m / ms[:, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    r = r / vs[:, None]
    bits = r.view(torch.int32)
    code = ((bits + 0x3FFFF + ((bits >> 19) & 1)) >> 19) - 1777
    vc = torch.where(r > 0, code.clamp(1, 255), torch.zeros_like(code)).to(torch.uint8)
    return mc.view(-1), vc.view(-1), ms, vs


def _decode(mc, vc, ms, vs):
    m = mc.float().view(-1, BLOCK) * ms[:, None]
    q = vc.to(torch.int32)
    r = torch.where(q > 0, (q + 1777) << 19, q).view(torch.float32).view(-1, BLOCK) * vs[:, None]
    return m.view(-1), (r * r).view(-1)


def _plain_adamw(s):
    case = s["case"]
    w, g = s["flat_w"].float(), s["flat_g"].float()
    m, v = _decode(*s["moments"]) if case["bits"] == 8 else s["moments"]
    if s["scale"] is not None:
        g = g * s["scale"]
    on = None
    if s["flat_keep"] is not None:
        on = torch.ones_like(w)
        on[:9 * s["flat_keep"].numel()] = _on(s["flat_keep"]).view(-1)
        g = g * on
    m = BETAS[0] * m + (1.0 - BETAS[0]) * g
    v = BETAS[1] * v + (1.0 - BETAS[1]) * (g * g)
    if on is not None:
        m, v = m * on, v * on
    if case["device"]:
        c1, c2 = (1.0 - torch.pow(torch.full((), b, dtype=torch.float64, device=w.device), s["step"]) for b in BETAS)
        c1, c2 = c1.float(), c2.float()
    else:
        c1, c2 = (1.0 - b ** s["step"] for b in BETAS)
    w = (1.0 - LR * DECAY) * w - LR * (m / c1) / (torch.sqrt(v / c2) + EPS)
    if on is not None:
        w = w * on
    if case["bits"] == 8:
        m, v = (x.to(torch.bfloat16) for x in _decode(*_encode(m, v)))
    copies = w.to(torch.bfloat16) if case["copies"] else None
    return w.to(s["flat_w"].dtype), copies, m, v


def _plain_look(s):
    case = s["case"]
    drop = s["ids"] == IGNORE
    rows = s["w"][torch.where(drop, torch.zeros_like(s["ids"]), s["ids"])].float() * case["scale"]
    return torch.where(drop[:, None], torch.zeros_like(rows), rows).to(DTYPES[case["y"]])


def _plain_grad(s):
    # (a row's sum can be long: in 64 bits where the result has 32)
    case = s["case"]
    wide = torch.float64 if case["w"] == "f32" else torch.float32
    v = case["v"]
    dw = torch.zeros(v + 1, case["d"], dtype=wide, device="cuda")
    dw.index_add_(0, torch.where(s["ids"] == IGNORE, torch.full_like(s["ids"], v), s["ids"]), s["dy"].to(wide))
    dw = dw[:v] * case["scale"]
    if s["add"] is not None:
        dw = dw + s["add"]
    return dw.to(DTYPES[case["w"]])


def _plain_norm(s):
    norm = torch.sqrt(s["flat_g"].float().square().sum())
    return norm, torch.clamp(MAX_NORM / norm, max=1.0)


def run(s):
    case = s["case"]
    if own:
        import paper_2004_11250_amd as pp
        if case["kind"] == "look":
            return pp.embed_fwd(s["ids"], s["w"], scale=case["scale"], ignore_index=IGNORE, dtype=DTYPES[case["y"]])
        if case["kind"] == "grad":
            return pp.embed_bwd(s["ids"], s["dy"], case["v"], scale=case["scale"], ignore_index=IGNORE,
                                dtype=DTYPES[case["w"]], add=s["add"])
        if case["kind"] == "norm":
            return pp.grad_norm(s["g"], max_norm=MAX_NORM)
        w_out, copies = s["views"]
        pp.adamw_step(s["w"], s["g"], s["state"], lr=LR, step=s["step"], betas=BETAS, eps=EPS, weight_decay=DECAY,
                      keep=s["keep"], copies=copies, grad_scale=s["scale"], out=(w_out, s["state_out"]))
        m, v = s["state_out"].values(torch.bfloat16) if case["bits"] == 8 else (s["state_out"].m, s["state_out"].v)
        return s["w_out"], s["copies"], m, v
    return {"look": _plain_look, "grad": _plain_grad, "norm": _plain_norm, "adamw": _plain_adamw}[case["kind"]](s)


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def _exact_blocks(m, v):
    """Moments in 64 bits -> what their codes of 8 bits stand for."""
    m, r = m.reshape(-1, BLOCK), v.reshape(-1, BLOCK) ** 0.5
    ms = torch.clamp(m.abs().max(1, keepdim=True).values / 448.0, min=TINY)
    vs = torch.clamp(r.max(1, keepdim=True).values, min=TINY)
    # e4m3: 3 bits after the leading one, of 2^-6 at least; then 4 bits, of 2^-16 and a step at least
    x, e = m / ms, None
    e = (torch.frexp(x)[1] - 1).clamp(min=-6)
    x = torch.ldexp(torch.round(torch.ldexp(x, 3 - e)), e - 3).clamp(-448.0, 448.0)
    y = r / vs
    e = torch.frexp(y)[1] - 1
    y = torch.where(y > 0, torch.ldexp(torch.round(torch.ldexp(y, 4 - e)), e - 4).clamp(2.0 ** -16 * 1.125, 1.0), y)
    return (x * ms).reshape(-1), ((y * vs) ** 2).reshape(-1)


def _exact_adamw(s):
    case = s["case"]
    shapes = _shapes(case)
    at, total = _places([shape for shape, _ in shapes])
    if case["bits"] == 8:
        mc, vc, ms, vs = s["moments"]
        m0 = mc.double().reshape(-1, BLOCK) * ms.double()[:, None]
        q = vc.double()
        e = torch.floor((q + 1777) / 16)
        r = torch.where(q > 0, 2.0 ** (e - 127) * (1.0 + (q + 1777 - 16 * e) / 16), q)
        m0, v0 = m0.reshape(-1), ((r.reshape(-1, BLOCK) * vs.double()[:, None]) ** 2).reshape(-1)
    else:
        m0, v0 = s["moments"]
    t = int(s["step"])
    scale = 1.0 if s["scale"] is None else float(s["scale"])
    outs = [torch.zeros(total, dtype=torch.float64, device="cuda") for _ in range(3)]
    keeps = s["keep"] or [None] * len(shapes)
    for a, (shape, _), kept in zip(at, shapes, keeps):
        b = a + math.prod(shape)
        g = s["flat_g"][a:b].double() * scale
        off = None
        if kept is not None:
            off = torch.stack([(kept >> k) & 1 for k in range(9)], -1).reshape(-1) == 0
            g = g.masked_fill(off, 0.0)
        m = m0[a:b].double().lerp(g, 1.0 - BETAS[0])
        v = v0[a:b].double().lerp(g ** 2, 1.0 - BETAS[1])
        w = s["flat_w"][a:b].double()
        w = w - LR * DECAY * w - LR / (1.0 - BETAS[0] ** t) * m / ((v / (1.0 - BETAS[1] ** t)) ** 0.5 + EPS)
        for o, x in zip(outs, (w, m, v)):
            o[a:b] = x if off is None else x.masked_fill(off, 0.0)
    w, m, v = outs
    if case["bits"] == 8:
        m, v = _exact_blocks(m, v)
    return w, (w if case["copies"] else None), m, v


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(s)
    if case["kind"] == "norm":
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.double()) for g in s["g"]]))
        return norm, torch.minimum(MAX_NORM / norm, torch.ones_like(norm))
    ids = s["ids"]
    live = torch.nonzero(ids != IGNORE)[:, 0]
    if case["kind"] == "look":
        y = torch.zeros(case["t"], case["d"], dtype=torch.float64, device="cuda")
        y[live] = torch.nn.functional.embedding(ids[live], s["w"].double()) * case["scale"]
        return y
    # tokens in the order of their ids: a row's sum is a difference of running sums, a part of the features at a time
    order = live[torch.argsort(ids[live], stable=True)]
    ends = torch.searchsorted(ids[order], torch.arange(case["v"] + 1, device="cuda"))
    dw = torch.zeros(case["v"], case["d"], dtype=torch.float64, device="cuda")
    for c in range(0, case["d"], 256):
        run_ = torch.cumsum(s["dy"][order, c:c + 256].double(), 0)
        run_ = torch.cat([torch.zeros_like(s["dy"][:1, c:c + 256], dtype=torch.float64), run_])
        dw[:, c:c + 256] = run_[ends[1:]] - run_[ends[:-1]]
    dw *= case["scale"]
    return dw if s["add"] is None else dw + s["add"].double()


def work(case):
    def size(name):
        return 4 if case[name] == "f32" else 2

    if case["kind"] in ("look", "grad"):
        t, v, d = case["t"], case["v"], case["d"]
        if case["kind"] == "look":
            return {"bytes": 8 * t + min(t, v) * d * size("w") + t * d * size("y"), "flops": t * d}
        return {"bytes": 8 * t + t * d * size("y") + v * d * size("w") * (2 if case["add"] else 1), "flops": t * d + v * d}
    n = sum(math.prod(shape) for shape, _ in _shapes(case))
    if case["kind"] == "norm":
        return {"bytes": n * size("g") + 8, "flops": 2 * n}
    moved = n * (size("g") + 2 * size("w") + (2 if case["copies"] else 0))
    moved += sum(2 * math.prod(shape) // 9 for shape, p in _shapes(case) if p)
    # moments read and written; those of 8 bits with two scales a block, and their values once more
    moved += n * 16 if case["bits"] == 32 else n * 4 + 16 * n // BLOCK + n * 4
    return {"bytes": moved, "flops": 15 * n}
