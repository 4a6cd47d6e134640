"""Trains a two-layer GraphSAGE on minibatches that `Massive` samples, with
features held in 8 (or 4) bits all the way: in the pinned store of the remote
nodes, over the host link, in the prefetch buffer and in the batch.

  python examples/train_sage.py [--steps 60] [--bits 8] [--width 128]

A step: the sampler's blocks and packed rows; the mean over each row's sampled
neighbours, read from the packed rows; a layer on a node's own row and that
mean; the same once more on the hidden rows; cross-entropy; the gradients back
through both layers and the hidden mean; an AdamW step with states in 8 bits.
Nodes' labels are what a fixed random map of their features says, so that there
is something to learn.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import synth  # noqa: E402
from paper_2410_22697_amd import AdamW, Massive, RowFormat, block_mean, linear, pack_rows, unpack_rows  # noqa: E402


class Setup:
    """One partition of the small workload: its features packed, the sampler over them, a model and its optimizer."""

    def __init__(self, bits=8, width=128, classes=16, seed=0):
        self.w = w = synth.get("cl10k")
        self.g = g = synth.partition_graph(w)
        own, remote = (torch.from_numpy(synth.features(ids, w.d, w.dtype, w.seed).reshape(-1).view(np.float32)).view(-1, w.d)
                       for ids in (g.local_gid, g.halo_gid))
        self.fmt = RowFormat(w.d, bits)
        rows = [pack_rows(x.cuda(), self.fmt).cpu() for x in (own, remote)]
        self.store = rows[1].pin_memory()
        self.sampler = Massive(g.L, g.H, g.indptr, g.indices, g.halo_gid, g.halo_degree, rows[0], self.store, self.fmt.row_bytes,
                               w.fanout, w.buffer_pct, w.gamma, w.delta, w.philox_seed)
        self.batch = self.sampler.alloc_batch(w.batch)
        self.schedule = synth.Schedule(g.L, w.train_pct, w.batch, w.seed)
        gen = torch.Generator().manual_seed(seed)
        self.labels = (own @ torch.randn(w.d, classes, generator=gen)).argmax(1).cuda()

        def weights(n, k):
            return (torch.randn(n, k, generator=gen) / k ** 0.5).cuda().requires_grad_()

        self.params = [weights(width, 2 * w.d), torch.zeros(width, device="cuda", requires_grad=True),
                       weights(classes, 2 * width), torch.zeros(classes, device="cuda", requires_grad=True)]
        self.optimizer = AdamW(self.params, lr=5e-3, weight_decay=0.0, state_bits=8)

    def sample(self, t):
        """Minibatch t: (seeds, packed rows of its frontier, [(indptr, indices) of each hop])."""
        seeds = torch.from_numpy(np.ascontiguousarray(self.schedule.seeds(t), np.int32)).cuda()
        b, r = self.batch, self.sampler.sample(seeds, self.batch)
        self.sampler.evict_step()
        blocks = [(b.indptr[k][:r.n[k] + 1], b.indices[k][:r.e[k]]) for k in range(len(r.e))]
        return seeds, b.feat[:r.n[-1]], blocks

    def logits(self, packed, blocks):
        """Layer by layer from the outer hop in: the rows of a hop's frontier come first among the next one's."""
        w1, b1, w2, b2 = self.params
        (inner, outer) = blocks
        n0, n1 = inner[0].numel() - 1, outer[0].numel() - 1
        own = unpack_rows(packed[:n1], self.fmt)
        hidden = linear(own, w1, b1, act="relu", x2=block_mean(packed, *outer, fmt=self.fmt))
        return linear(hidden[:n0], w2, b2, x2=block_mean(hidden, *inner))

    def step(self, t):
        seeds, packed, blocks = self.sample(t)
        loss = torch.nn.functional.cross_entropy(self.logits(packed, blocks), self.labels[seeds.long()])
        for p in self.params:
            p.grad = None
        loss.backward()
        self.optimizer.step()
        return loss.detach()


def train(steps=60, bits=8, width=128, report=print):
    s = Setup(bits, width)
    losses = []
    for t in range(steps):
        losses.append(s.step(t))
        if report and (t % 10 == 9 or t == steps - 1):
            report("step %3d  loss %.4f" % (t + 1, float(torch.stack(losses[-10:]).mean())))
    return torch.stack(losses).cpu()


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--steps", type=int, default=60)
    a.add_argument("--bits", type=int, default=8, choices=(8, 4))
    a.add_argument("--width", type=int, default=128)
    args = a.parse_args()
    train(args.steps, args.bits, args.width)
