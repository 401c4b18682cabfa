"""Gradients of norms that no workgroup holds, over more tokens than there are workgroups: a workgroup takes several tokens, and the weights'
gradients are sums of several groups'."""
import pytest

from test_gpu_layer_norm import check_gradient

pytestmark = pytest.mark.gpu

SIZES = [  # W, T, width, gap, bias
    (2, 300, 9000, 0, True), (1, 130, 8193, 1, True), (3, 70, 16392, 4, False), (5, 61, 8200, 0, True), (1, 259, 20001, 0, True),
]


@pytest.mark.parametrize("types", [("f32", "f32", "f32", "f32", "f32"), ("bf16", "bf16", "f32", "bf16", "f32"), ("bf16", "bf16", "bf16", "bf16", "bf16")], ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradient(size, types):
    check_gradient(size, *types, accumulate=size[0] % 2 == 0, with_add=size[1] % 2 == 0)


@pytest.mark.parametrize("accumulate,with_add", [(False, False), (True, False), (False, True), (True, True)])
def test_gradient_added_and_written(accumulate, with_add):
    check_gradient((2, 150, 8300, 0, True), "bf16", "bf16", "f32", "bf16", "f32", accumulate, with_add)
