"""Activations and their slopes at infinity: the limits of their formulas."""
import math

import pytest
import torch

from test_gpu_linear import ACTS, Layer, backward, forward

pytestmark = pytest.mark.gpu
INFINITE = torch.tensor([math.inf, -math.inf, math.nan, 1.0], dtype=torch.bfloat16)


@pytest.mark.parametrize("act", list(ACTS))
def test_infinite_numbers(act):
    """z as x, through a matrix of one."""
    layer = Layer(1, 1, 1, bias=False)
    one = torch.ones((1, layer.stride), dtype=torch.bfloat16)
    plan = layer.plan(4)
    got, before = forward(layer, plan, INFINITE.view(1, 4, 1), one, act, None, torch.bfloat16)
    got, before = got.view(-1), before.view(-1)
    assert before[0] == math.inf and before[1] == -math.inf and before[2].isnan()
    assert got[0] == math.inf and got[1] == (-math.inf if act == "none" else 0.0) and got[2].isnan() and got[3].isfinite()
    if act == "none":
        return
    for dtype in (torch.bfloat16, torch.float32):
        dx, _ = backward(layer, plan, torch.full((1, 4, 1), 2.0, dtype=dtype), INFINITE.view(1, 4, 1), one, act, INFINITE.view(1, 4, 1).to(dtype), None,
                         torch.bfloat16, one, False)
        dx = dx.view(-1)
        assert dx[0] == 2.0 and dx[1] == 0.0 and dx[2].isnan() and dx[3].isfinite()
