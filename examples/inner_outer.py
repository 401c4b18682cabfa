"""Replicas that train between outer steps: the inner step's operators and the outer step over one arena.

    python examples/inner_outer.py [--workers 8] [--outer 6] [--inner 10] [--norm]

Every worker's row of the arena holds a small next-token model: a tied embedding table, the two matrices of a residual
block and, if it is asked for, a norm in front of the output head. An inner step looks the worker's tokens up in its own table (embed_lookup), runs
block, norm, tied head and loss (linear, layer_norm, token_log_probs) and their gradients, adds the lookup's gradient to the
head's (embed_gradient, accumulate) and updates the matrices by their orthogonalised momentum (muon_step), the rest by plain
gradient descent. After the inner steps of a round, random pairs of workers exchange (plan_groups, outer_step), and the
replicas' spread is logged.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_10911_amd as nl  # noqa: E402

VOCAB, WIDTH, HIDDEN, TOKENS = 211, 96, 192, 256


class Replicas:
    def __init__(self, workers, seed=0, norm=False):
        self.W, self.norm = workers, norm
        self.shapes = [(VOCAB, WIDTH), (WIDTH, HIDDEN), (HIDDEN, WIDTH)] + ([(WIDTH,), (WIDTH,)] if norm else [])
        sizes = [math.prod(shape) for shape in self.shapes]
        offsets = [sum(sizes[:i]) for i in range(len(sizes))]
        self.segments = list(zip(offsets, sizes))
        stride = -(-sum(sizes) // 64) * 64
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        start = torch.zeros(stride, device="cuda")
        start[:sum(sizes[:3])].normal_(0.0, 0.05, generator=gen)
        if norm:
            start[offsets[3]:offsets[4]] = 1.0              # its weights
        self.phi = start.repeat(workers, 1)                 # slow weights, the same everywhere
        self.theta = self.phi.clone()                       # fast weights
        self.delta = torch.zeros_like(self.phi)             # outer momentum
        self.grad = torch.zeros_like(self.phi)
        self.momentum = torch.zeros_like(self.phi)          # of the inner steps
        self.outer_plan = nl.LaunchPlan(self.phi, self.delta, self.theta, stride, workers, nl.F32, self.segments)
        matrices = [(offsets[1], WIDTH, HIDDEN), (offsets[2], HIDDEN, WIDTH)]
        self.muon_plan = nl.MuonPlan(matrices, stride, workers)
        self.embedding_plan = nl.EmbeddingPlan(0, VOCAB, WIDTH, stride, workers, TOKENS)
        self.linear_plan = nl.LinearPlan([(offsets[1], WIDTH, HIDDEN), (offsets[2], HIDDEN, WIDTH), (0, WIDTH, VOCAB, None, True)],
                                         stride, workers, TOKENS)
        if norm:
            self.norm_plan = nl.LayerNormPlan([(offsets[3], offsets[4], WIDTH)], stride, workers, TOKENS)
        self.loss_plan = nl.LogProbPlan(VOCAB, workers, TOKENS)
        new = lambda *shape: torch.empty((workers, TOKENS, *shape), device="cuda")  # noqa: E731
        self.x, self.h, self.dh, self.dx = (new(WIDTH) for _ in range(4))
        self.last, self.dlast = (new(WIDTH), new(WIDTH)) if norm else (self.h, self.dh)     # what the head takes
        self.before, self.hidden, self.dhidden = (new(HIDDEN) for _ in range(3))
        self.logits, self.stats, self.log_probs, self.norms = new(VOCAB), new(2), new(), new()
        self.dlog_probs = torch.full((workers, TOKENS), -1.0 / TOKENS, device="cuda")      # of the mean loss
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

    def forward(self, inputs, targets):
        """Mean loss of every worker."""
        T, f32, theta = TOKENS, nl.F32, self.theta
        nl.embed_lookup(self.embedding_plan, theta, f32, inputs, nl.I64, T, WIDTH ** 0.5, self.x, f32)
        nl.linear(self.linear_plan, 0, self.x, f32, theta, f32, T, self.hidden, f32, activation=nl.ACT_RELU, before=self.before)
        nl.linear(self.linear_plan, 1, self.hidden, f32, theta, f32, T, self.h, f32, residual=self.x)
        if self.norm:
            nl.layer_norm(self.norm_plan, 0, self.h, f32, theta, f32, T, 1e-5, self.last, f32, stats=self.stats)
        nl.linear(self.linear_plan, 2, self.last, f32, theta, f32, T, self.logits, f32)
        nl.token_log_probs(self.loss_plan, self.logits, f32, targets, nl.I64, T, self.log_probs, norms=self.norms)
        return -self.log_probs.mean(1)

    def backward(self, inputs, targets):
        """Gradients of the mean losses of the last forward pass into grad."""
        T, f32, theta, grad = TOKENS, nl.F32, self.theta, self.grad
        nl.token_log_probs_gradient(self.loss_plan, self.logits, f32, targets, nl.I64, T, self.norms, self.dlog_probs, self.logits, f32)
        nl.linear_gradient(self.linear_plan, 2, self.logits, f32, self.last, f32, theta, f32, T, self.dlast, f32, grad, f32)
        if self.norm:
            nl.layer_norm_gradient(self.norm_plan, 0, self.dlast, f32, self.h, f32, theta, f32, self.stats, T, self.dh, f32, grad, f32)
        nl.linear_gradient(self.linear_plan, 1, self.dh, f32, self.hidden, f32, theta, f32, T, self.dhidden, f32, grad, f32)
        # the residual branch's gradient is what the block's is added to
        nl.linear_gradient(self.linear_plan, 0, self.dhidden, f32, self.x, f32, theta, f32, T, self.dx, f32, grad, f32,
                           activation=nl.ACT_RELU, before=self.before, add=self.dh)
        nl.embed_gradient(self.embedding_plan, self.dx, f32, inputs, nl.I64, T, WIDTH ** 0.5, grad, f32, accumulate=True)

    def inner_step(self, lr=0.05, table_lr=0.5):
        tokens = self.text()
        inputs, targets = tokens[:, :-1].contiguous(), tokens[:, 1:].contiguous()
        loss = self.forward(inputs, targets)
        self.backward(inputs, targets)
        nl.muon_step(self.muon_plan, self.theta, nl.F32, self.grad, nl.F32, self.momentum, (lr, 0.9, 0.0))
        weights, gradients = self.views(self.theta), self.views(self.grad)
        for weight, gradient in zip(weights[:1] + weights[3:], gradients[:1] + gradients[3:]):
            weight.add_(gradient, alpha=-table_lr)
        return loss

    def outer_step(self, step, hparams=(0.5, 0.7, 0.7)):
        members, offsets = nl.plan_groups(17, step, self.W, 2)
        nl.replica_spread(self.outer_plan, self.theta, nl.F32, self.spread)
        nl.outer_step(self.outer_plan, self.phi, self.delta, self.theta, hparams, members, offsets)
        return self.spread[-1]


def train(workers=8, outer=6, inner=10, seed=0, say=print, norm=False):
    """Mean loss of every round's last inner step."""
    replicas, losses = Replicas(workers, seed, norm), []
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
    parser.add_argument("--norm", action="store_true")
    a = parser.parse_args()
    train(a.workers, a.outer, a.inner, norm=a.norm)
