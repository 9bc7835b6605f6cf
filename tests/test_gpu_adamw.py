"""AdamW steps (pp_adamw_step, pp_adamw_values) and gradient norms (pp_grad_norm) on
the GPU against the formulas in 64 bits.

Error bounds, with u = 2^-24 (half a step of fp32 beside 1).
  m'  b1, 1 - b1, scale G, and the two products with their sum are rounded: at most
      4 u (b1 |m| + (1 - b1) |g|).
  v'  likewise with g g: 6 u v'.
  W'  decay and its product: 2 u |W|.  The update U = rate m' / (r c2 + eps): the
      rate, c2, eps, two products and a sum, each u; r = sqrt(v'), whose instruction
      is off by up to a unit in the last place (2 u), from v' (3 u); the reciprocal's
      instruction (2 u): 14 u of the update, and m''s error through it, 4 u of
      Umax, the update with b1 |m| + (1 - b1) |g| in the place of m'; the last sum:
      u |W'|.  In all 4 u |W| + 20 u Umax, and half a step of the weights' type.
8-bit moments.  A first moment is rounded to 4 bits, 2^-4 of itself, or by half of
the least step, 2^-10 of the scale; a second one's root to 5 bits, 2^-5 of itself
(what lies below the least code, 1.125 2^-16 of the scale, is held as that).  The
scales are rounded too: a few u, covered by a part in 1000 of these."""
import math

import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
B = 128
SHAPES = [(1,), (7,), (128,), (129,), (0,), (3, 5), (16, 16, 3, 3), (100, 513), (30011,)]


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(seed, *shape):
    return torch.randn(shape, generator=rng(seed), device="cuda")


def spread(seed, *shape):
    """Values whose sizes differ by many orders."""
    return normal(seed, *shape) * torch.exp(3.0 * normal(seed + 1, *shape))


class Run:
    """A list with its state after some steps, and the exact step from there."""

    def __init__(self, seed, shapes, w, g, bits, keep=(), shift=0):
        def make(k, dt, size):
            got = []
            for i, s in enumerate(shapes):
                n = math.prod(s)
                flat = torch.zeros(n + shift, device="cuda", dtype=dt)   # (shift: not aligned)
                flat[shift:] = (normal(seed + 100 * k + i, n) * size).to(dt)
                got.append(flat[shift:].view(s))
            return got

        self.w, self.g = make(1, DT[w], 0.1), make(2, DT[g], 1e-2)
        self.state = pp.AdamWState(self.w, bits=bits)
        m, v = spread(seed + 7, self.state.elements) * 1e-3, spread(seed + 9, self.state.elements).square() * 1e-6
        for t in (m, v):
            inside = torch.zeros_like(t)
            for x in self.state.split(inside):
                x.fill_(1.0)
            t *= inside
        self.keep = None
        if keep:
            self.keep = [None] * len(shapes)
            for i in keep:
                self.keep[i] = torch.randint(0, 512, shapes[i][:2], generator=rng(seed + i), device="cuda").to(torch.int16)
        if bits == 32:
            self.state.m.copy_(m), self.state.v.copy_(v)
        else:
            for name, t in zip(("m", "v", "m_scale", "v_scale"), encode(m, v)):
                getattr(self.state, name).copy_(t)
        self.copies = [torch.full(s, 9.0, device="cuda", dtype=torch.bfloat16) for s in shapes] if w == "f32" else None

    def clone(self):
        new = object.__new__(Run)
        new.w, new.g, new.keep = [t.clone() for t in self.w], self.g, self.keep
        new.copies = None if self.copies is None else [t.clone() for t in self.copies]
        new.state = pp.AdamWState(self.w, bits=self.state.bits)
        for a, b in zip(new.state.buffers(), self.state.buffers()):
            if a is not None:
                a.copy_(b)
        return new

    def bits(self):
        return [t.clone().view(torch.uint8) for t in self.w + [t for t in self.state.buffers() if t is not None] + (self.copies or [])]

    def moments(self):
        """What the state holds, in 64 bits."""
        if self.state.bits == 32:
            return self.state.m.double(), self.state.v.double()
        return decode(*self.state.buffers())

    def exact(self, lr, step, betas, eps, decay, scale):
        """Per tensor (W', m', v' and their bounds)."""
        m, v = (self.state.split(t) for t in self.moments())
        got = []
        for i, (w, g) in enumerate(zip(self.w, self.g)):
            w, g = w.double(), g.double() * scale
            on = torch.ones_like(w)
            if self.keep and self.keep[i] is not None:
                on = torch.stack([(self.keep[i].long() >> t) & 1 for t in range(9)], -1).view(w.shape).double()
                g = g * on
            m1 = (betas[0] * m[i] + (1 - betas[0]) * g) * on
            v1 = (betas[1] * v[i] + (1 - betas[1]) * g * g) * on
            msize = (betas[0] * m[i].abs() + (1 - betas[0]) * g.abs()) * on
            den = (v1 / (1 - betas[1] ** step)).sqrt() + eps
            rate = lr / (1 - betas[0] ** step)
            new = ((1 - lr * decay[i]) * w - rate * m1 / den) * on
            wlim = 4 * U * w.abs() + 20 * U * rate * msize / den
            if self.w[i].dtype == torch.bfloat16:
                wlim = wlim + 2.0 ** -8 * (new.abs() + wlim)
            got.append((new, wlim * on, m1, 4 * U * msize, v1, 6 * U * v1))
        return got


def encode(m, v):
    """Moments as codes and scales, in 64 bits."""
    m, r = m.double().view(-1, B), v.double().sqrt().view(-1, B)
    ms = (m.abs().amax(1) / 448).clamp(min=2.0 ** -100).float()
    vs = r.amax(1).clamp(min=2.0 ** -100).float()
    mc = (m / ms.double()[:, None]).clamp(-448, 448).float().to(torch.float8_e4m3fn)
    r = r / vs.double()[:, None]
    e = torch.frexp(r)[1] - 1
    q = torch.round(torch.ldexp(r, 4 - e)) + 16 * (e + 126)      # (16 .. 32 for the bits, from the exponent's 2^-127 on)
    vc = torch.where(r > 0, (q - 1777).clamp(1, 255), torch.zeros_like(q)).to(torch.uint8)
    return mc.view(-1), vc.view(-1), ms, vs


def decode(mc, vc, ms, vs):
    q = vc.long()
    r = torch.where(q > 0, 2.0 ** ((q + 1777) // 16 - 127).double() * (1 + ((q + 1777) % 16).double() / 16), 0.0)
    m = mc.double().view(-1, B) * ms.double()[:, None]
    return m.view(-1), (r.view(-1, B) * vs.double()[:, None]).square().view(-1)


def within(got, want, lim, what):
    bad = ~((got.double() - want).abs() <= lim)
    assert not bad.any(), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist())


def check(run, lr=1e-2, step=7, betas=(0.9, 0.999), eps=1e-8, decay=0.1, scale=None, out=None, device=False):
    n = len(run.w)
    decays = list(decay) if isinstance(decay, (list, tuple)) else [decay] * n
    real = 1.0 if scale is None else float(scale)
    want = run.exact(lr, step, betas, eps, decays, real)
    before = [t.clone() for t in run.w]
    sources = [run.moments()[0].clone(), run.moments()[1].clone()]
    kw = dict(lr=lr, step=step)
    if device:
        kw = dict(lr=torch.tensor([lr], device="cuda"), step=torch.tensor(step, device="cuda"))
    w, state = pp.adamw_step(run.w, run.g, run.state, betas=betas, eps=eps, weight_decay=decay, keep=run.keep, copies=run.copies,
                             grad_scale=None if scale is None else torch.tensor(scale, device="cuda"), out=out, **kw)
    if out is not None:
        assert all(torch.equal(a, b) for a, b in zip(before, run.w)) and torch.equal(run.moments()[0], sources[0])
    held = state.split(state.m), state.split(state.v)
    if state.bits == 8:
        dm, dv = decode(*state.buffers())
        for got, exact in zip(state.values(), (dm, dv)):     # (a product or two of fp32 values)
            assert bool(((got.double() - exact).abs() <= 3 * U * exact.abs() + 2.0 ** -140).all())
        for got, exact in zip(state.values(torch.bfloat16), (dm, dv)):
            assert bool(((got.double() - exact).abs() <= 1.01 * 2.0 ** -8 * exact.abs() + 2.0 ** -133).all())
        held = state.split(dm), state.split(dv)
        ms, vs = (x.double().repeat_interleave(B) for x in (state.m_scale, state.v_scale))
        ms, vs = state.split(ms), state.split(vs)
    for i, (nw, wlim, m, mlim, v, vlim) in enumerate(want):
        within(w[i], nw, wlim, ("w", i))
        if run.copies is not None:
            assert torch.equal(run.copies[i], w[i].to(torch.bfloat16)), i
        if state.bits == 32:
            within(held[0][i], m, mlim, ("m", i))
            within(held[1][i], v, vlim, ("v", i))
        else:
            within(held[0][i], m, 1.001 * torch.maximum(2.0 ** -4 * m.abs(), 2.0 ** -10 * ms[i]) + mlim, ("m", i))
            r = v.sqrt()
            least = 1.125 * 2.0 ** -16 * vs[i] * (r > 0)
            within(held[1][i].sqrt(), torch.maximum(r, least), 1.001 * 2.0 ** -5 * torch.maximum(r, least), ("v", i))
    # what lies between the tensors is 0
    for t in state.buffers()[:2]:
        rest = t.view(torch.uint8).clone()
        for x in state.split(rest.view(t.dtype)):
            x.view(-1).view(torch.uint8).zero_()
        assert not bool(rest.any())
    return w, state


TYPES = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")]


@pytest.mark.parametrize("w,g", TYPES)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_step(w, g, bits, shift):
    check(Run(1, SHAPES, w, g, bits, keep=(6,), shift=shift), decay=[0.1 * i for i in range(len(SHAPES))], scale=0.25)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("step", [1, 2, 1000, 10 ** 9])
@pytest.mark.parametrize("betas,eps", [((0.9, 0.999), 1e-8), ((0.0, 0.0), 1e-3), ((0.95, 0.9999), 0.0), ((0.5, 0.5), 10.0)])
@pytest.mark.parametrize("device", [False, True])
def test_parameters(bits, step, betas, eps, device):
    # (a learning rate that fp32 holds, so that both ways of giving it are the same)
    check(Run(2, [(50, 33), (9,)], "f32", "f32", bits), lr=0.0078125, step=step, betas=betas, eps=eps, device=device)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("cells", [(1, 1), (5, 3), (128, 1), (64, 64), (300, 7), (257, 129)])
def test_pruned_layers(bits, cells):
    run = Run(3, [(*cells, 3, 3), (40,), (*cells, 3, 3)], "f32", "bf16", bits, keep=(0, 2))
    on = torch.stack([(run.keep[0].long() >> t) & 1 for t in range(9)], -1).view(run.w[0].shape).bool()
    want = run.exact(1e-2, 7, (0.9, 0.999), 1e-8, [0.1] * 3, 1.0)
    # what taps that are off hold is never looked at
    run.g[0][~on] = float("nan")
    run.w[2][0, 0] = float("inf")
    run.keep[2][0, 0] = 0
    w, state = pp.adamw_step(run.w, run.g, run.state, lr=1e-2, step=7, weight_decay=0.1, keep=run.keep)
    within(w[0], want[0][0], want[0][1], "w")
    assert bool((w[0][~on] == 0).all()) and bool((w[2][0, 0] == 0).all())
    for t in state.values():
        assert bool((state.split(t)[0][~on] == 0).all()) and bool((state.split(t)[2][0, 0] == 0).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(bits):
    shapes = [(1 + 37 * i % 211,) for i in range(150)] + [(70, 90)] * 3
    check(Run(4, shapes, "f32", "bf16", bits))


@pytest.mark.parametrize("w,g", TYPES)
@pytest.mark.parametrize("bits", [32, 8])
def test_out_and_in_place(w, g, bits):
    run = Run(5, SHAPES, w, g, bits, keep=(6,))
    other = run.clone()
    out = [torch.full_like(t, 3.0) for t in run.w], pp.AdamWState(run.w, bits=bits)
    for t in out[1].buffers():
        if t is not None:
            t.view(torch.uint8).fill_(5)
    new, state = check(run, out=out)
    check(other)
    assert all(torch.equal(a, b) for a, b in zip(new, other.w))
    for a, b in zip(state.buffers(), other.state.buffers()):
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf")])
def test_no_step(bits, scale):
    run = Run(6, SHAPES, "f32", "bf16", bits, keep=(6,))
    run.copies = None
    before = run.bits()
    s = torch.tensor(scale, device="cuda")
    pp.adamw_step(run.w, run.g, run.state, lr=1.0, step=1, grad_scale=s, keep=run.keep)
    assert all(torch.equal(a, b) for a, b in zip(before, run.bits()))
    out = [torch.full_like(t, 3.0) for t in run.w], pp.AdamWState(run.w, bits=bits)
    copies = [torch.zeros_like(t, dtype=torch.bfloat16) for t in run.w]
    pp.adamw_step(run.w, run.g, run.state, lr=1.0, step=1, grad_scale=s, out=out, copies=copies)
    assert all(torch.equal(a, b) for a, b in zip(run.w, out[0]))
    assert all(torch.equal(a.bfloat16(), b) for a, b in zip(run.w, copies))
    for a, b in zip(run.state.buffers(), out[1].buffers()):
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_codes_of_every_kind():
    # a block of all codes survives a step without gradient: the scales shrink, the codes stay
    state = pp.AdamWState([(512,)], bits=8)
    codes = torch.arange(512, device="cuda") % 256
    codes[(codes & 127) == 127] = 0x7E              # (no NaN)
    state.m.view(torch.uint8).copy_(codes)
    state.v.copy_(torch.arange(512, device="cuda") % 256)
    for blocks in (state.m.view(torch.uint8).view(-1, B), state.v.view(-1, B)):
        blocks[:, 0] = 0x7E if blocks is not state.v else 255
    state.v.view(-1, B)[:, 1] = 255
    state.m_scale.copy_(torch.tensor([1e-3, 1e-30, 7.0, 1e20], device="cuda"))
    state.v_scale.copy_(torch.tensor([1e-5, 1e-15, 3.0, 1e15], device="cuda"))
    m, v = state.m.view(torch.uint8).clone(), state.v.clone()
    ms, vs = state.m_scale.clone(), state.v_scale.clone()
    w, g = torch.zeros(512, device="cuda"), torch.zeros(512, device="cuda")
    for k in range(1, 4):
        pp.adamw_step([w], [g], state, lr=1e-3, step=k, betas=(0.9, 0.96))
        now = state.m.view(torch.uint8)
        # (1e-30 0.9^3 = 7.29e-31 is below the least scale, 2^-100 = 7.89e-31: there the scale is that, and the
        # codes are of values rounded anew, half a step or 2^-10 of the scale off)
        above = torch.tensor([True, k < 3, True, True], device="cuda")
        on = above.repeat_interleave(B)
        assert torch.equal(now[on] & 127, m[on] & 127) and torch.equal(state.v, v), k
        assert bool(((state.m_scale / ms - 0.9 ** k).abs() < 1e-5)[above].all())
        assert bool(((state.v_scale / vs - 0.96 ** (k / 2)).abs() < 1e-5).all())
    assert float(state.m_scale[1]) == 2.0 ** -100
    was = m.view(torch.float8_e4m3fn).double()[B:2 * B] * float(ms[1]) * 0.9 ** 3
    held = state.m.double()[B:2 * B] * 2.0 ** -100
    assert bool(((held - was).abs() <= 1.001 * torch.maximum(2.0 ** -4 * was.abs(), torch.full_like(was, 2.0 ** -110))).all())


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf"), 1e30])
def test_gradients_that_are_not_finite(what):
    shapes = [(300,)]
    clean, hit = Run(8, shapes, "f32", "f32", 8), None
    hit = clean.clone()
    hit.g = [clean.g[0].clone()]
    clean.g[0][5], hit.g[0][5] = 0.0, what
    clean.state.m.view(torch.uint8)[5] = 0
    clean.state.v[5] = 0
    check(clean)
    pp.adamw_step(hit.w, hit.g, hit.state, lr=1e-2, step=7, weight_decay=0.1)
    rest = torch.arange(300, device="cuda") != 5
    assert torch.equal(clean.w[0][rest], hit.w[0][rest])
    m, v = hit.state.values()
    if math.isfinite(what):        # a huge one takes its block's resolution, and no more
        assert bool(torch.isfinite(hit.w[0]).all()) and bool(torch.isfinite(m).all())
        assert float(m[5]) > 0.9e29 and 3e38 < float(v[5]) <= 3.4028235e38
        assert bool((v[:128][rest[:128]] > 0).all())
    else:
        assert bool(torch.isnan(m[5])) and not bool(torch.isfinite(hit.w[0][5]))
        assert torch.equal(m[:300][rest], clean.state.values()[0][:300][rest]) and torch.equal(v, clean.state.values()[1])
        pp.adamw_step(hit.w, [torch.zeros(300, device="cuda")], hit.state, lr=1e-2, step=8)
        assert bool(torch.isnan(hit.w[0][5])) and bool(torch.isfinite(hit.w[0][rest]).all())


def test_32_bits_keep_what_is_not_finite():
    run = Run(9, [(300,)], "f32", "f32", 32)
    run.g[0][5], run.g[0][6] = float("nan"), float("inf")
    pp.adamw_step(run.w, run.g, run.state, lr=1e-2, step=7)
    rest = (torch.arange(300, device="cuda") - 5.5).abs() > 1
    assert bool(torch.isnan(run.w[0][5:7]).all()) and bool(torch.isfinite(run.w[0][rest]).all())


def test_graph():
    run = Run(10, [(60, 70), (33,)], "f32", "bf16", 8)
    other = run.clone()
    step, lr = torch.tensor(1, device="cuda"), torch.tensor(1e-3, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm, scale = pp.grad_norm(run.g, max_norm=0.5)
        pp.adamw_step(run.w, run.g, run.state, lr=lr, step=step, grad_scale=scale, copies=run.copies)
    for k in range(4):
        for i, g in enumerate(run.g):
            g.copy_(normal(50 + 2 * k + i, *g.shape))
        step.fill_(k + 1)
        lr.fill_(1e-3 * (k + 1))
        graph.replay()
        a, s = pp.grad_norm(run.g, max_norm=0.5)
        pp.adamw_step(other.w, run.g, other.state, lr=lr, step=k + 1, grad_scale=s, copies=other.copies)
        assert float(a) == float(norm) and float(s) == float(scale)
        # (bias corrections of the host and of the device may differ in a last place)
        for x, y in zip(run.w, other.w):
            assert bool(((x - y).abs() <= 4 * U * x.abs() + 1e-8).all())
        other = run.clone()
        torch.cuda.synchronize()


def test_offsets_past_32_bits():
    n = (1 << 31) + 300
    w = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-5:] = 1.0
    g[7] = 1.0
    state = pp.AdamWState([(n,)], bits=8)
    pp.adamw_step(w, g, state, lr=0.5, step=1)
    assert w[-5:].tolist() == [-0.5] * 5 and float(w[7]) == -0.5 and int((w != 0).sum()) == 6
    norm, _ = pp.grad_norm([g])
    assert abs(float(norm) - 6 ** 0.5) < 1e-6
    m, v = state.values(torch.bfloat16)
    assert int((m != 0).sum()) == 6 and abs(float(m[n - 1]) - 0.1) < 1e-3 and abs(float(v[n - 1]) - 1e-3) < 1e-5


@pytest.mark.parametrize("g", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", [[(1,)], [(0,), (3,)], SHAPES, [(2000, 3001)], [(5,)] * 400])
def test_norm(g, shapes):
    # squares and sums in 64 bits, then one rounding
    for shift in (0, 1):
        grads = Run(11, shapes, "f32", g, 32, shift=shift).g
        want = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
        norm, scale = pp.grad_norm(grads)
        assert norm.shape == scale.shape == () and abs(float(norm) - want) <= 1.01 * U * want and float(scale) == 1.0
        for most in (want / 3, want * 2):
            norm, scale = pp.grad_norm(grads, max_norm=most)
            expect = min(1.0, float(torch.tensor(most)) / want) if want else 1.0
            assert abs(float(scale) - expect) <= 1.01 * U


def test_norms_of_every_size():
    one = torch.zeros(1000, device="cuda")
    assert [float(x) for x in pp.grad_norm([one], max_norm=1.0)] == [0.0, 1.0]
    for value in (1e-38, 1e-25, 1e25, 3e38):
        one.fill_(0.0)[17] = value
        norm, scale = pp.grad_norm([one], max_norm=1e-3)
        size = float(one[17])
        assert abs(float(norm) - size) <= 2 * U * size
        assert abs(float(scale) - min(1.0, float(torch.tensor(1e-3)) / size)) <= 2 * U
    one.fill_(3e38)                       # a norm that fp32 does not hold, of gradients that it does
    norm, scale = pp.grad_norm([one], max_norm=1.0)
    assert float(norm) == math.inf and abs(float(scale) * 3e38 * 1000 ** 0.5 - 1.0) < 1e-2
    for bad in (math.inf, -math.inf, math.nan):
        one.fill_(1.0)[999] = bad
        for most in (None, 1.0):
            norm, scale = pp.grad_norm([one, one], max_norm=most)
            assert not math.isfinite(float(norm)) and math.isnan(float(scale))


def test_what_autograd_sees():
    w = normal(1, 20, 30).requires_grad_()
    y = (w * w).sum()
    state = pp.AdamWState([w])
    before = w._version, state.m._version
    new, same = pp.adamw_step(w, normal(2, 20, 30), state, lr=0.1, step=1)
    assert new is w and same is state and w._version > before[0] and state.m._version > before[1]
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_lists_are_checked_on_the_gpu_too():
    w, g = [normal(1, 4, 6), normal(2, 9)], [normal(3, 4, 6), normal(4, 9)]
    state = pp.AdamWState(w)
    before = [t.clone() for t in w]
    go = lambda w=w, g=g, **kw: pp.adamw_step(w, g, state, lr=1e-3, step=1, **kw)   # noqa: E731
    for bad in ([w[0].t().contiguous(), w[1]], [w[0].view(24), w[1]], [w[1], w[0]]):
        with pytest.raises(ValueError, match="shapes"):
            go(w=bad)
        with pytest.raises(ValueError, match="shapes"):
            go(g=bad)
    for bad in ([normal(5, 6, 4).t(), g[1]], [g[0], g[1].bfloat16()], [g[0], g[1].cpu()], [normal(6, 1, 6).expand(4, 6), g[1]]):
        with pytest.raises(ValueError, match="contiguous"):
            go(g=bad)
    with pytest.raises(ValueError, match="same tensor"):
        pp.adamw_step([w[1], w[1]], [g[1], g[1]], pp.AdamWState([w[1], w[1]]), lr=1e-3, step=1)
    with pytest.raises(ValueError, match="another tensor of the call"):
        go(out=([g[0], w[1]], state))
    with pytest.raises(ValueError, match="another tensor's input"):
        pp.adamw_step([w[1], before[1]], [g[1], g[1]], pp.AdamWState([w[1], w[1]]), lr=1e-3, step=1,
                      out=([before[1], normal(9, 9)], pp.AdamWState([w[1], w[1]])))
    with pytest.raises(ValueError, match="contiguous"):
        pp.grad_norm([g[0], normal(5, 6, 4).t()])
    assert all(torch.equal(a, b) for a, b in zip(w, before))
    go()
    assert not torch.equal(w[0], before[0])


@pytest.mark.parametrize("bits", [32, 8])
def test_second_moments_below_the_normal_range(bits):
    # beta2 = 1/2 halves v; eps = 0: the update is m' / sqrt(v') to the bounds above
    n = 64
    w, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    state = pp.AdamWState([w], bits=bits)
    v = torch.ldexp(torch.ones(n, device="cuda"), -148 + torch.arange(n, device="cuda"))      # 2^-148 .. 2^-85
    m = v.sqrt() * 0.25
    if bits == 32:
        state.m[:n], state.v[:n] = m, v
        pp.adamw_step([w], [g], state, lr=1.0, step=10 ** 6, betas=(0.5, 0.5), eps=0.0, weight_decay=0.0)
        # (the least step there is 2^-149, so that half of an odd number of them is off by 2^-150; the update is of
        # what is held)
        assert bool(((state.v[:n].double() - v.double() / 2).abs() <= 2.0 ** -150).all())
        want = -(m.double() / 2) / state.v[:n].double().sqrt()
        assert bool(((w.double() - want).abs() <= 20 * U * want.abs()).all())
    else:
        pad = torch.zeros(B - n, device="cuda")
        for name, t in zip(("m", "v", "m_scale", "v_scale"), encode(torch.cat([m, pad]), torch.cat([v, pad]))):
            getattr(state, name).copy_(t)
        # (the scales are 2^-42.5 and 2^-44.5 / 448: codes reach down to 2^-58 of the root; below it they are the least)
        _, was = decode(*state.buffers())
        pp.adamw_step([w], [g], state, lr=1.0, step=10 ** 6, betas=(0.5, 0.5), eps=0.0, weight_decay=0.0)
        _, now = decode(*state.buffers())
        assert bool(torch.isfinite(w).all()) and bool((now[:n] > 0).all()) and bool((now[n:] == 0).all())
        root, held = (was / 2).sqrt()[:n], now.sqrt()[:n]
        least = 1.125 * 2.0 ** -16 * float(state.v_scale[0])
        want = root.clamp(min=least)
        assert bool(((held - want).abs() <= 1.001 * 2.0 ** -5 * want).all())


@pytest.mark.parametrize("w,g,bits", [("f32", "f32", 32), ("f32", "bf16", 32), ("bf16", "bf16", 32), ("bf16", "f32", 32), ("f32", "bf16", 8),
                                      ("f32", "f32", 8), ("bf16", "bf16", 8), ("bf16", "f32", 8)])
@pytest.mark.parametrize("shift", [0, 1])
def test_steps_past_the_caches(w, g, bits, shift):
    # more than 256 MB in all: the small tensors of the list go the same way
    check(Run(12, SHAPES + [(26000011,)], w, g, bits, keep=(6,), shift=shift))
