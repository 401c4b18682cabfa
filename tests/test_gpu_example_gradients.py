"""The example's inner step against torch's in 64 bits, and its training with a norm in front of the head."""
import importlib.util
import math
import os

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu


def example():
    spec = importlib.util.spec_from_file_location("inner_outer", os.path.join(ROOT, "examples", "inner_outer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("norm", [False, True])
def test_gradients_are_those_of_autograd(norm):
    """The example's gradients against torch's in 64 bits, of every tensor. Its sums are of up to 256 numbers in binary32, one after the other in
    a chain of ten operators: 2^-24 times the number of additions is 2^-13 of the gradients' norm."""
    module = example()
    replicas = module.Replicas(3, norm=norm)
    replicas.theta.add_(0.02 * torch.randn(replicas.theta.shape, generator=torch.Generator().manual_seed(1)).cuda())
    tokens = replicas.text()
    inputs, targets = tokens[:, :-1].contiguous(), tokens[:, 1:].contiguous()
    loss = replicas.forward(inputs, targets)
    replicas.backward(inputs, targets)
    leaf = replicas.theta.cpu().double().requires_grad_()
    table, up, down, *of_norm = replicas.views(leaf)
    x = torch.stack([t[i] for t, i in zip(table, inputs.cpu())]) * module.WIDTH ** 0.5
    h = x + torch.relu(x @ up) @ down
    if norm:
        d = h - h.mean(-1, keepdim=True)
        h = d * (d.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * of_norm[0][:, None] + of_norm[1][:, None]
    want = -(h @ table.mT).log_softmax(-1).gather(-1, targets.cpu()[..., None])[..., 0].mean(1)
    want.sum().backward()
    assert ((loss.cpu().double() - want).abs() <= 2.0 ** -13 * want.abs()).all()
    for got, exact in zip(replicas.views(replicas.grad.cpu().double()), replicas.views(leaf.grad)):
        assert (got - exact).norm() <= 2.0 ** -13 * exact.norm()


def test_training_with_a_norm_runs():
    losses = example().train(workers=2, outer=2, inner=2, say=lambda line: None, norm=True)
    assert len(losses) == 2 and all(math.isfinite(v) for v in losses)
