"""The node classifier of examples/: the operators next to the update step, run together as a program would."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_classifier_learns_and_answers_alike_in_8_bits():
    from node_classifier import NodeClassifier
    model = NodeClassifier(nodes=4000, batch=256)
    try:
        losses = model.train(120)
        # guessing among 47 classes costs log 47 = 3.85
        assert losses[0] > 3.0 and sum(losses[-10:]) / 10 < 0.6 * losses[0]
        seeds = torch.arange(256, dtype=torch.int32, device=model.dev)
        exact, exact_logp = model.answer(seeds, 7, int8=False)
        index, logp = model.answer(seeds, 7)
        labels = model.labels[seeds.long()]
        assert float((exact[:, 0] == labels).float().mean()) > 0.4
        # rows and weights in 8 bits are each off by 1/254 of their largest value at most: few best classes are that close
        assert float((index[:, 0] == exact[:, 0]).float().mean()) > 0.9
        assert float((logp[:, 0] - exact_logp[:, 0]).abs().median()) < 0.1
    finally:
        model.close()


def test_gradients_of_a_step_are_those_of_the_loss():
    """The step's gradients against torch's for the same inputs (from the checkpoints' values) in 64 bits."""
    from node_classifier import BETA, NodeClassifier
    from paper_2106_06150_amd import learn
    model = NodeClassifier(nodes=3000, batch=200)
    try:
        seeds = torch.randperm(3000, generator=torch.Generator().manual_seed(3))[:200].to(torch.int32).to(model.dev)
        before = [p.detach().clone() for p in (model.w1, model.b1, model.w2, model.b2)]
        loss = model.step(seeds, 11)

        def kept(name):
            c = model.kept[name]
            out = torch.empty((200, c.width), device=model.dev)
            learn.gns_checkpoint_load(model.ctx, *c.packed, out, 200)
            return out.double().cpu()

        w1, b1, w2, b2 = (p.double().cpu().requires_grad_() for p in before)
        x, mean = kept("x"), kept("mean")
        z = torch.cat([x, mean], 1) @ w1 + b1
        # the mask of the exact activations, and h as it was kept: straight through the rounding to 8 bits
        mask = ((model.kept["h"].positive.cpu()[:, :, None] >> torch.arange(32)) & 1).reshape(200, -1)[:, :model.hidden].double()
        h = z * mask
        h = h + (kept("h") - h).detach()
        # the loss's gradient was taken where the exact activations led
        logits = torch.cat([h, x], 1) @ w2 + b2
        logits = logits + (model.logits.double().cpu() - logits).detach()
        log_p = torch.log_softmax(logits[:, :model.classes], 1)
        labels = model.labels[seeds.long()].long().cpu()
        total = -(log_p[torch.arange(200), labels] - BETA * (log_p.exp() * log_p).sum(1)).mean()
        total.backward()
        assert abs(float(loss) - float(total.detach())) < 1e-4
        for got, want in ((model.w1.grad, w1.grad), (model.b1.grad, b1.grad), (model.w2.grad, w2.grad), (model.b2.grad, b2.grad)):
            got = got.double().cpu()
            assert float((got - want).norm() / want.norm()) < 1e-5
    finally:
        model.close()
