"""The deeper classifier of examples/: the operators of include/gns_layers.h run together with those next to the update step."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture()
def model():
    from deep_classifier import DeepClassifier
    m = DeepClassifier(nodes=3000, batch=200)
    yield m
    m.close()


def test_it_trains_and_answers(model):
    losses = model.train(20)
    assert len(losses) == 20 and all(l == l and abs(l) < 100 for l in losses)
    seeds = torch.arange(200, dtype=torch.int32, device=model.dev)
    for fp8 in (False, True):
        index, value = model.answer(seeds, 7, fp8=fp8)
        assert bool(((index >= 0) & (index < model.classes)).all()) and bool((value <= 0).all())
        assert bool((value[:, :-1] >= value[:, 1:]).all())


def test_gradients_of_a_step_are_those_of_the_loss(model):
    """Against torch's for the same inputs (from the checkpoints' values) in 64 bits."""
    from deep_classifier import BETA, GROUPS
    from paper_2106_06150_amd import learn
    seeds = torch.randperm(3000, generator=torch.Generator().manual_seed(3))[:200].to(torch.int32).to(model.dev)
    with torch.no_grad():
        model.gamma += 0.2 * torch.randn(model.hidden, generator=torch.Generator().manual_seed(4)).to(model.dev)
        model.beta += 0.2 * torch.randn(model.hidden, generator=torch.Generator().manual_seed(5)).to(model.dev)
    loss = model.gradients(seeds, 11)

    def kept(name):
        c = model.kept[name]
        out = torch.empty((200, c.width), device=model.dev)
        learn.gns_checkpoint_load(model.ctx, *c.packed, out, 200)
        return out.double().cpu()

    params = [model.w1, model.b1, model.gamma, model.beta, model.w2, model.b2]
    w1, b1, gamma, beta, w2, b2 = (p.detach().double().cpu().requires_grad_() for p in params)
    x, mean = kept("x"), kept("mean")
    z = torch.cat([x, mean], 1) @ w1 + b1
    z = z + (model.z.double().cpu() - z).detach()         # the layers' values are of the rows before they were kept in 8 bits
    g = z.view(200, GROUPS, -1)
    g = (g - g.mean(2, keepdim=True)) / torch.sqrt(g.var(2, unbiased=False, keepdim=True) + 1e-5)
    h = torch.nn.functional.silu(g.reshape(200, -1) * gamma + beta)
    h = h + (kept("h") - h).detach()
    logits = torch.cat([h, x], 1) @ w2 + b2
    logits = logits + (model.logits.double().cpu() - logits).detach()
    log_p = torch.log_softmax(logits[:, :model.classes], 1)
    labels = model.labels[seeds.long()].long().cpu()
    total = -(log_p[torch.arange(200), labels] - BETA * (log_p.exp() * log_p).sum(1)).mean()
    total.backward()
    # a few hundred products' roundings each, by way of two layers
    assert abs(float(loss) - float(total.detach())) < 1e-4
    for got, want in zip(params, (w1, b1, gamma, beta, w2, b2)):
        assert float((got.grad.double().cpu() - want.grad).norm() / want.grad.norm()) < 1e-5


def test_a_step_moves_the_weights_along_orthogonal_matrices(model):
    from deep_classifier import COEFFICIENTS, MU
    seeds = torch.arange(200, dtype=torch.int32, device=model.dev)
    model.train(2)
    before = [w.detach().double().cpu() for w in (model.w1, model.w2)]
    momenta = [m.double().cpu() for m in model.momenta]
    model.step(seeds, 5)
    for w, old, m, how, now in zip((model.w1, model.w2), before, momenta, model.how, model.momenta):
        grad = w.grad.double().cpu()
        m = MU * m + grad
        x = grad + MU * m
        x = x / (x.norm() + 1e-7)
        x = x.t() if x.shape[0] > x.shape[1] else x
        for a, b, c in COEFFICIENTS:
            gram = x @ x.t()
            x = a * x + (b * gram + c * gram @ gram) @ x
        x = x.t() if old.shape[0] > old.shape[1] else x
        want = how.struct.keep * old + how.struct.rate * x
        # mu is a float: 2^-24 of it; five steps let errors of 22 bits grow by 3.4445 each at most, times the rate
        assert float((now.double().cpu() - m).norm()) <= 4 * 2.0 ** -24 * float(m.norm())
        room = abs(how.struct.rate) * 5 * 3.4445 ** 5 * 16 * 2.0 ** -22 + 4 * 2.0 ** -24 * float(want.norm())
        assert float((w.detach().double().cpu() - want).norm()) <= room
