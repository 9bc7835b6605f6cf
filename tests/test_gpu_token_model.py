"""The lookup, the loss, their gradients, the clipping and the AdamW steps run
together, as the example of a token model has them.

Error bound of the gradients: each is a chain of three sums of at most 1000 fp32
products or terms, each off by at most 1000 2^-24 of its terms' size, 6e-5; the
chain by 2e-4 of the gradient's norm."""
import os
import sys

import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import train_token_model as ex   # noqa: E402


def loss64(table, w, bias, ids, target):
    live = ids != ex.PAD
    x = table[ids] * ex.WIDTH ** 0.5 * live[:, None]
    logits = torch.relu(x @ w.t()) @ table.t() + bias
    each = torch.logsumexp(logits, 1) - logits.gather(1, target[:, None])[:, 0]
    return each[target != ex.PAD].mean()


def test_gradients():
    m = ex.Model(3)
    m.bias.normal_(generator=torch.Generator("cuda").manual_seed(4))
    ids, target = ex.batch(5)
    loss, grads = m.gradients(ids, target)
    params = [p.double().requires_grad_() for p in (m.table, m.w, m.bias)]
    want = loss64(*params, ids, target)
    assert abs(float(loss) - float(want.detach())) <= 1e-5 * float(want.detach())
    exact = torch.autograd.grad(want, params)
    for got, g in zip(grads, exact):
        assert got.shape == g.shape and float((got - g).norm() / g.norm()) <= 2e-4
    # against differences of the loss in 64 bits (of second order: off by the square of the step)
    with torch.no_grad():
        for k in range(3):
            d = torch.randn(params[k].shape, generator=torch.Generator("cuda").manual_seed(k), device="cuda").double() + \
                3.0 * exact[k] / exact[k].square().mean().sqrt()
            h = 1e-6
            up, down = ([p + (s * h * d if i == k else 0.0) for i, p in enumerate(params)] for s in (1.0, -1.0))
            slope = (loss64(*up, ids, target) - loss64(*down, ids, target)) / (2 * h)
            assert abs(float((grads[k] * d).sum()) - float(slope)) <= 1e-3 * abs(float(slope)), k


def test_padding_reaches_nothing():
    m = ex.Model(3)
    none = torch.full((ex.TOKENS,), ex.PAD, device="cuda")
    loss, grads = m.gradients(none, none)
    assert float(loss) == 0.0 and all(not bool(g.any()) for g in grads)


def state_of(m):
    return [m.table, m.w, m.bias] + [t for s in (m.table_state, m.state) for t in s.buffers() if t is not None]


def test_recorded_steps_are_the_eager_ones():
    (a, m), (b, n) = ex.train(6, graph=True), ex.train(6, graph=False)
    assert a == b and int(m.step) == 6
    for x, y in zip(state_of(m), state_of(n)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_a_step_on_another_stream():
    m, n = ex.Model(7), ex.Model(7)
    ids, target = ex.batch(8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.train_step(ids, target, 1e-3)
    n.train_step(ids, target, 1e-3)
    torch.cuda.synchronize()
    for x, y in zip(state_of(m), state_of(n)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_two_graphs():
    # two recorded steps of two models, replayed in turn and at once
    models, graphs, data = [ex.Model(k) for k in range(2)], [], [ex.batch(k) for k in range(2)]
    for m, (ids, target) in zip(models, data):
        m.train_step(ids, target, 1e-3)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.train_step(ids, target, 1e-3)
        graphs.append(g)
    side = torch.cuda.Stream()
    for k in range(3):
        side.wait_stream(torch.cuda.current_stream())
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.current_stream().wait_stream(side)
    for k, m in enumerate(models):
        n = ex.Model(k)
        for _ in range(4):
            n.train_step(*data[k], 1e-3)
        for x, y in zip(state_of(m), state_of(n)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_a_step_that_is_left_out_does_not_count():
    # first, between others, and in a recorded step: what follows is as if it had not been
    for graph in (False, True):
        models = [ex.Model(11), ex.Model(11)]
        data = [ex.batch(k) for k in range(4)]
        bad = torch.zeros((), device="cuda")

        def step(m, ids, target):
            _, grads = m.gradients(ids, target)
            grads[2] += bad
            m.update(grads, 1e-3)

        ids, target = (t.clone() for t in data[0])
        if graph:
            recorded = torch.cuda.CUDAGraph()
            with torch.cuda.graph(recorded):
                step(models[0], ids, target)
        taken = 0
        for k, wrong in enumerate((float("nan"), 0.0, float("inf"), 0.0)):
            bad.fill_(wrong)
            ids.copy_(data[k][0])
            target.copy_(data[k][1])
            recorded.replay() if graph else step(models[0], ids, target)
            if not wrong:
                taken += 1
                step(models[1], *data[k])
            assert int(models[0].step) == int(models[1].step) == taken
            for x, y in zip(state_of(models[0]), state_of(models[1])):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), k


def test_a_step_that_is_not_finite_is_left_out():
    m = ex.Model(9)
    ids, target = ex.batch(10)
    m.train_step(ids, target, 1e-3)
    before = [t.clone().view(torch.uint8) for t in state_of(m)]
    _, grads = m.gradients(ids, target)
    grads[2][5] = float("inf")
    m.update(grads, 1e-3)
    assert all(torch.equal(a, b.view(torch.uint8)) for a, b in zip(before, state_of(m)))
