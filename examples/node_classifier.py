"""A node classifier trained and used with the operators next to the update step, on a synthetic graph:

  sample, gather, aggregate                       one layer of Global Neighbor Sampling
  h = relu([x | neighbors' mean] W1 + b1)         gns_sage_dense; x, the mean and h kept in 8 bits (gns_checkpoint_save)
  logits = [h | x] W2 + b2                        gns_sage_dense
  loss = -mean log p(label) - beta * entropy      gns_log_probs, gns_log_probs_backward
  gradients of W2, b2, h, then W1, b1             gns_sage_dense_backward, from the checkpoints
  answers: both layers in 8-bit integers          gns_sage_dense_int8; the best classes by gns_log_probs

    python examples/node_classifier.py --steps 200
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2106_06150_amd import binding as B  # noqa: E402
from paper_2106_06150_amd import learn, synth  # noqa: E402

BETA = 0.01                       # weight of the entropy in the loss


class Checkpoint:
    """8-bit rows of one activation, of at most `rows` rows, and where they are positive."""

    def __init__(self, rows, width, dev):
        groups = learn.checkpoint_groups(width)
        self.width = width
        self.packed = (torch.empty((rows, 32 * groups), dtype=torch.int8, device=dev),
                       torch.empty((rows, groups), dtype=torch.uint8, device=dev))
        self.positive = torch.empty((rows, groups), dtype=torch.int32, device=dev)

    def save(self, ctx, x, rows):
        learn.gns_checkpoint_save(ctx, x, *self.packed, self.positive, rows)


class Int8Layer:
    """Weights [k, n] as n rows of 8 bits with a scale each."""

    def __init__(self, ctx, w, bias):
        k, n = w.shape
        self.q = torch.empty((n, learn.int8_stride(k)), dtype=torch.int8, device=w.device)
        self.scale, self.bias = torch.empty(n, device=w.device), bias
        learn.gns_quantize_rows(ctx, w.t().contiguous(), None, self.q, self.scale, n)


class NodeClassifier:
    def __init__(self, nodes=20000, feat=100, hidden=128, classes=47, batch=512, fanout=10, seed=1):
        dev = self.dev = torch.device("cuda:0")
        gen = torch.Generator(device=dev).manual_seed(seed)
        graph = synth.chung_lu_graph(nodes, 8 * nodes, 2.1, seed, device=dev)
        x = synth.node_features(nodes, feat, seed + 1, device=dev)
        self.x, self.feat, self.hidden, self.classes, self.batch = x, feat, hidden, classes, batch
        # a node's class depends on its features and on its neighbors'
        degree = torch.diff(graph.indptr.long())
        row = torch.repeat_interleave(torch.arange(nodes, device=dev), degree)
        mean = torch.zeros_like(x).index_add_(0, row, x[graph.indices.long()]) / degree.clamp(min=1)[:, None]
        pick = torch.randn((2, feat, classes), device=dev, generator=gen)
        self.labels = (x @ pick[0] + 3.0 * mean @ pick[1]).argmax(1).to(torch.int32)
        self.graph = B.make_graph(graph.indptr, graph.indices, feat_dev=x)
        self.config = B.make_config([fanout], [B.GNS_CACHE_FIRST], nodes // 100, batch, flag_mode=B.GNS_FLAGS_PER_CACHE)
        self.workspace = B.alloc_workspace(self.graph, self.config, dev)
        self.ctx = B.gns_create(self.graph, self.config, self.workspace)
        self.blocks = B.BlockBuffers(self.graph, self.config, dev)
        B.gns_sample_cache(self.ctx, seed, 0)

        def weights(k, n):
            return (torch.randn((k, n), device=dev, generator=gen) * (1.5 / k) ** 0.5).requires_grad_()

        # widths of the update step are multiples of four; what is behind the last class is never looked at
        self.width = (classes + 3) // 4 * 4
        self.w1, self.b1 = weights(2 * feat, hidden), torch.zeros(hidden, device=dev, requires_grad=True)
        self.w2, self.b2 = weights(hidden + feat, self.width), torch.zeros(self.width, device=dev, requires_grad=True)
        self.adam = torch.optim.Adam([self.w1, self.b1, self.w2, self.b2], lr=0.003)
        cap = self.blocks.array[0].cap_src
        self.x_in = torch.empty((cap, feat), device=dev)
        self.mean = torch.empty((batch, feat), device=dev)
        self.h = torch.empty((batch, hidden), device=dev)
        self.logits = torch.empty((batch, self.width), device=dev)
        self.d_logits = torch.zeros((batch, self.width), device=dev)
        self.d_in = torch.empty((batch, hidden + feat), device=dev)
        self.logp, self.entropy, self.stats = (torch.empty(s, device=dev) for s in ((batch,), (batch,), (batch, 2)))
        self.kept = {"x": Checkpoint(batch, feat, dev), "mean": Checkpoint(batch, feat, dev), "h": Checkpoint(batch, hidden, dev)}
        space = learn.gns_sage_dense_backward_workspace_bytes
        self.space = learn.alloc_workspace(max(
            space(self.ctx, hidden, feat, self.width, batch), space(self.ctx, feat, feat, hidden, batch),
            learn.gns_sage_dense_int8_workspace_bytes(self.ctx, 2 * feat, batch),
            learn.gns_sage_dense_int8_workspace_bytes(self.ctx, hidden + feat, batch),
            learn.gns_log_probs_workspace_bytes(self.ctx, classes, 5, batch)), dev)

    def inputs(self, seeds, batch_seed):
        """Features of the seeds (a view) and their sampled neighbors' mean."""
        block = self.blocks.array[0]
        B.gns_sample_blocks(self.ctx, batch_seed, seeds, self.blocks.array)
        B.gns_gather_features(self.ctx, self.blocks.tensors[0]["src_nodes"], block.num_src, self.x_in)
        B.gns_aggregate(self.ctx, block, self.x_in, self.feat, self.mean)
        return self.x_in[:self.batch], self.mean

    def step(self, seeds, batch_seed):
        """One training step; the mean loss, on the device."""
        ctx, n, classes = self.ctx, seeds.numel(), self.classes
        labels = self.labels[seeds.long()]
        x, mean = self.inputs(seeds, batch_seed)
        B.gns_sage_dense(ctx, x, mean, self.w1.detach(), self.b1.detach(), True, self.h, n)
        B.gns_sage_dense(ctx, self.h, x, self.w2.detach(), self.b2.detach(), False, self.logits, n)
        for name, rows in (("x", x), ("mean", mean), ("h", self.h)):
            self.kept[name].save(ctx, rows, n)
        learn.gns_log_probs(ctx, self.logits[:, :classes], labels, self.logp, self.entropy, self.stats, None, None, n, self.space)
        loss = -(self.logp[:n].mean() + BETA * self.entropy[:n].mean())
        g_logp, g_entropy = torch.full((n,), -1.0 / n, device=self.dev), torch.full((n,), -BETA / n, device=self.dev)
        learn.gns_log_probs_backward(ctx, self.logits[:, :classes], labels, self.stats, self.entropy, g_logp, g_entropy, self.d_logits[:, :classes], n)
        k = self.kept
        for p in (self.w1, self.b1, self.w2, self.b2):
            p.grad = torch.empty_like(p)
        learn.gns_sage_dense_backward(ctx, self.d_logits, None, k["h"].packed, self.hidden, k["x"].packed, self.feat, self.w2.detach(),
                                      self.w2.grad, self.b2.grad, self.d_in, n, self.space)
        learn.gns_sage_dense_backward(ctx, self.d_in[:, :self.hidden], k["h"].positive, k["x"].packed, self.feat, k["mean"].packed, self.feat,
                                      self.w1.detach(), self.w1.grad, self.b1.grad, None, n, self.space)
        self.adam.step()
        return loss

    def train(self, steps, seed=100):
        gen = torch.Generator(device=self.dev).manual_seed(seed)
        losses = []
        for i in range(steps):
            seeds = torch.randperm(self.x.shape[0], device=self.dev, generator=gen)[:self.batch].to(torch.int32)
            losses.append(self.step(seeds, seed + i))
        return torch.stack(losses).tolist()

    def answer(self, seeds, batch_seed, int8=True, top=5):
        """The `top` best classes of the seeds and their log probabilities."""
        ctx, n = self.ctx, seeds.numel()
        x, mean = self.inputs(seeds, batch_seed)
        if int8:
            one, two = Int8Layer(ctx, self.w1.detach(), self.b1.detach()), Int8Layer(ctx, self.w2.detach(), self.b2.detach())
            learn.gns_sage_dense_int8(ctx, x, mean, one.q, one.scale, one.bias, True, self.h, n, self.space)
            learn.gns_sage_dense_int8(ctx, self.h, x, two.q, two.scale, two.bias, False, self.logits, n, self.space)
        else:
            B.gns_sage_dense(ctx, x, mean, self.w1.detach(), self.b1.detach(), True, self.h, n)
            B.gns_sage_dense(ctx, self.h, x, self.w2.detach(), self.b2.detach(), False, self.logits, n)
        index = torch.empty((n, top), dtype=torch.int32, device=self.dev)
        value = torch.empty((n, top), device=self.dev)
        learn.gns_log_probs(ctx, self.logits[:, :self.classes], None, None, None, None, index, value, n, self.space)
        return index, value

    def close(self):
        torch.cuda.synchronize()
        B.gns_destroy(self.ctx)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=200)
    args = ap.parse_args()
    model = NodeClassifier()
    losses = model.train(args.steps)
    seeds = torch.arange(model.batch, dtype=torch.int32, device=model.dev)
    labels = model.labels[seeds.long()]
    exact, _ = model.answer(seeds, 7, int8=False)
    index, _ = model.answer(seeds, 7)
    print("loss %.3f -> %.3f; right answers: fp32 %.1f %%, 8 bits %.1f %%, among the five best %.1f %%; same answer %.1f %%" % (
        losses[0], losses[-1], 100 * (exact[:, 0] == labels).float().mean(), 100 * (index[:, 0] == labels).float().mean(),
        100 * (index == labels[:, None]).any(1).float().mean(), 100 * (index[:, 0] == exact[:, 0]).float().mean()))
    model.close()


if __name__ == "__main__":
    main()
