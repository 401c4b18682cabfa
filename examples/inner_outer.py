"""Replicas that train between outer steps: the inner step's operators and the outer step over one arena.

    python examples/inner_outer.py [--workers 8] [--outer 6] [--inner 10]

Every worker's row of the arena holds a small next-token model: a tied embedding table and two matrices of a residual
block. An inner step looks the worker's tokens up in its own table (embed_lookup), runs the block and the tied output
head with torch, adds the lookup's gradient to the head's (embed_gradient, accumulate) and updates the matrices by their
orthogonalised momentum (muon_step), the table by plain gradient descent. After the inner steps of a round, random pairs
of workers exchange (plan_groups, outer_step), and the replicas' spread is logged.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_10911_amd as nl  # noqa: E402

VOCAB, WIDTH, HIDDEN, TOKENS = 211, 96, 192, 256


class Replicas:
    def __init__(self, workers, seed=0):
        self.W = workers
        sizes = [VOCAB * WIDTH, WIDTH * HIDDEN, HIDDEN * WIDTH]
        offsets = [0, sizes[0], sizes[0] + sizes[1]]
        self.segments = list(zip(offsets, sizes))
        stride = -(-sum(sizes) // 64) * 64
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        start = torch.zeros(stride, device="cuda")
        start[:sum(sizes)].normal_(0.0, 0.05, generator=gen)
        self.phi = start.repeat(workers, 1)                 # slow weights, the same everywhere
        self.theta = self.phi.clone()                       # fast weights
        self.delta = torch.zeros_like(self.phi)             # outer momentum
        self.grad = torch.zeros_like(self.phi)
        self.momentum = torch.zeros_like(self.phi)          # of the inner steps
        self.outer_plan = nl.LaunchPlan(self.phi, self.delta, self.theta, stride, workers, nl.F32, self.segments)
        matrices = [(offsets[1], WIDTH, HIDDEN), (offsets[2], HIDDEN, WIDTH)]
        self.muon_plan = nl.MuonPlan(matrices, stride, workers)
        self.embedding_plan = nl.EmbeddingPlan(0, VOCAB, WIDTH, stride, workers, TOKENS)
        self.shapes = [(VOCAB, WIDTH), (WIDTH, HIDDEN), (HIDDEN, WIDTH)]
        self.looked_up = torch.empty((workers, TOKENS, WIDTH), device="cuda")
        self.spread = torch.empty(len(self.segments) + 1, dtype=torch.float64, device="cuda")
        self.gen = gen
        # the language: every token has three likely successors
        self.successors = torch.randint(VOCAB, (VOCAB, 3), generator=gen, device="cuda")

    def views(self, array):
        return [array[:, o:o + n].unflatten(1, shape) for (o, n), shape in zip(self.segments, self.shapes)]

    def text(self):
        """[W, TOKENS + 1] tokens of fresh text for every worker."""
        tokens = torch.empty((self.W, TOKENS + 1), dtype=torch.int64, device="cuda")
        tokens[:, 0] = torch.randint(VOCAB, (self.W,), generator=self.gen, device="cuda")
        pick = torch.randint(3, (self.W, TOKENS), generator=self.gen, device="cuda")
        for t in range(TOKENS):
            tokens[:, t + 1] = self.successors[tokens[:, t], pick[:, t]]
        return tokens

    def inner_step(self, lr=0.05, table_lr=0.5):
        tokens = self.text()
        inputs, targets = tokens[:, :-1].contiguous(), tokens[:, 1:]
        scale = WIDTH ** 0.5
        nl.embed_lookup(self.embedding_plan, self.theta, nl.F32, inputs, nl.I64, TOKENS, scale, self.looked_up, nl.F32)
        x = self.looked_up.requires_grad_()
        table, up, down = (v.detach().requires_grad_() for v in self.views(self.theta))
        h = x + torch.relu(x @ up) @ down
        logits = h @ table.mT
        loss = (logits.logsumexp(-1) - logits.gather(-1, targets[..., None])[..., 0]).mean(1)
        dx, *gradients = torch.autograd.grad(loss.sum(), [x, table, up, down])
        self.looked_up = x.detach()
        for view, g in zip(self.views(self.grad), gradients):
            view.copy_(g)
        nl.embed_gradient(self.embedding_plan, dx.contiguous(), nl.F32, inputs, nl.I64, TOKENS, scale, self.grad, nl.F32, accumulate=True)
        nl.muon_step(self.muon_plan, self.theta, nl.F32, self.grad, nl.F32, self.momentum, (lr, 0.9, 0.0))
        self.views(self.theta)[0].add_(self.views(self.grad)[0], alpha=-table_lr)
        return loss.detach()

    def outer_step(self, step, hparams=(0.5, 0.7, 0.7)):
        members, offsets = nl.plan_groups(17, step, self.W, 2)
        nl.replica_spread(self.outer_plan, self.theta, nl.F32, self.spread)
        nl.outer_step(self.outer_plan, self.phi, self.delta, self.theta, hparams, members, offsets)
        return self.spread[-1]


def train(workers=8, outer=6, inner=10, seed=0, say=print):
    """Mean loss of every round's last inner step."""
    replicas, losses = Replicas(workers, seed), []
    for t in range(outer):
        for _ in range(inner):
            loss = replicas.inner_step()
        spread = replicas.outer_step(t)
        losses.append(loss.mean().item())
        say(f"round {t}: loss {losses[-1]:.3f} (workers {loss.min().item():.3f} to {loss.max().item():.3f}), "
            f"replicas {spread.item():.2e} apart before the exchange")
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--workers", type=int, default=8)
    parser.add_argument("--outer", type=int, default=6)
    parser.add_argument("--inner", type=int, default=10)
    a = parser.parse_args()
    train(a.workers, a.outer, a.inner)
