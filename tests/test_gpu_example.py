"""The example that runs inner and outer steps together learns its language, and the same from the same seed."""
import importlib.util
import math
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


def example():
    spec = importlib.util.spec_from_file_location("inner_outer", os.path.join(ROOT, "examples", "inner_outer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_replicas_learn():
    module = example()
    losses = module.train(workers=4, outer=5, inner=8, say=lambda line: None)
    # untrained, the loss is that of a guess; three successors a token leave log 3
    assert losses[-1] < 0.8 * math.log(module.VOCAB) and losses[-1] < losses[0]
    assert all(math.isfinite(v) for v in losses)
