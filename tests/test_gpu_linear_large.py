"""Large products on the GPU at sizes that are known to take the kernels that they are for (tests/test_product_plans.py asks): every tile, layout,
format and end, in 64 bits number by number, and as a whole: a bound that grows with k for the worst case would hide digits that are lost."""
import math

import pytest
import torch

import model_plain as plain
import product_shapes as shapes
from test_gpu_linear import DTYPES, Layer, backward, check_gradient, forward, randn, same_bits, within

pytestmark = pytest.mark.gpu


def check_digits(got, a, b, out, floats):
    """got = a b. The norm of what it is off: roundings to bf16 are 2^-8 / sqrt(3) of the lower end of a number's binade, 0.00166 of the number in the
    mean square: once for a bf16 result, once more if one float operand is rounded beside a bf16 one. A float result: the matrix cores add
    sixteen products at a time, 3 k / 16 roundings of random sign of sums that grow as their root, 0.43 U each: below 7.5e-7 for k of 9001,
    and operands of 22 bits. Each row by itself may be off by twice that: rows are as long as some hundred numbers."""
    exact, bound = plain.product(a, b, out)
    within(got, exact, bound + plain.STORED[out] * exact.abs())
    limit = 1e-6 if out == torch.float32 else (2.5e-3 if floats == 1 else 1.8e-3)
    off = got.double() - exact
    assert off.norm() <= limit * exact.norm(), (off.norm() / exact.norm()).item()
    assert (off.norm(dim=-1) <= 2 * limit * exact.norm(dim=-1)).all()


@pytest.mark.parametrize("size,types", shapes.FORWARD, ids=str)
def test_digits(size, types):
    W, T, inputs, outputs, more = size
    layer = Layer(W, inputs, outputs, **more)
    x_type, theta, out = (DTYPES[t] for t in types)
    a, x = layer.array(theta, std=0.3), randn((W, T, inputs), 2, x_type)
    got, _ = forward(layer, layer.plan(T), x, a, "none", None, out, before=False)
    check_digits(got, x, layer.matrix(a), out, types[:2].count("f32"))


@pytest.mark.parametrize("types", shapes.GRADIENT_TYPES, ids=str)
@pytest.mark.parametrize("size", shapes.GRADIENT_SIZES, ids=str)
def test_digits_of_gradients(size, types):
    W, T, inputs, outputs, more = size
    layer = Layer(W, inputs, outputs, **more)
    dout_type, x_type, theta, dx_type, grad_type = (DTYPES[t] for t in types)
    a, x, dout = layer.array(theta, std=0.3), randn((W, T, inputs), 2, x_type), randn((W, T, outputs), 3, dout_type)
    dx, grad = backward(layer, layer.plan(T), dout, x, a, "none", None, None, dx_type, a.to(grad_type), False)
    check_digits(dx, dout, layer.matrix(a).mT, dx_type, (types[0], types[2]).count("f32"))
    check_digits(layer.matrix(grad), x.mT, dout, grad_type, types[:2].count("f32"))


def test_digits_of_a_gradient_of_two_types():
    W, T, inputs, outputs, more = shapes.GRADIENT_SIZES[0]
    layer = Layer(W, inputs, outputs, **more)
    dout_type, x_type, theta, dx_type, grad_type = (DTYPES[t] for t in shapes.MIXED)
    a, x, dout = layer.array(theta, std=0.3), randn((W, T, inputs), 2, x_type), randn((W, T, outputs), 3, dout_type)
    _, grad = backward(layer, layer.plan(T), dout, x, a, "none", None, None, dx_type, a.to(grad_type), False)
    check_digits(layer.matrix(grad), x.mT, dout, grad_type, 1)


@pytest.mark.parametrize("types", shapes.GRADIENT_TYPES, ids=str)
@pytest.mark.parametrize("size", shapes.GRADIENT_SIZES, ids=str)
def test_gradients_added(size, types):
    check_gradient(size, types, "none", with_add=True, accumulate=True)


@pytest.mark.parametrize("room", shapes.BATCH_ROOMS)
@pytest.mark.parametrize("types", shapes.BATCH_TYPES, ids=str)
def test_gradients_through_an_activation_in_batches_of_workers(types, room):
    """Operands packed to a workspace that has room for one worker, or for some."""
    W, T, inputs, outputs, more = shapes.BATCHES
    layer = Layer(W, inputs, outputs, **more)
    dout_type, x_type, theta, dx_type, grad_type = (DTYPES[t] for t in types)
    a, x, dout = layer.array(theta, std=0.3), randn((W, T, inputs), 2, x_type), randn((W, T, outputs), 3, dout_type)
    before, old = randn((W, T, outputs), 4, dout_type), layer.array(grad_type, seed=6)
    plan = layer.plan(T, room)
    dx, grad = backward(layer, plan, dout, x, a, "silu", before, None, dx_type, old, False)
    of_dx, of_matrix, of_bias = plain.linear_gradient(dout, x, layer.matrix(a), before, "silu", None, dx_type, grad_type)
    within(dx, *of_dx)
    within(layer.matrix(grad), *plain.stored(*of_matrix, None, grad_type))
    within(layer.of_bias(grad), *plain.stored(*of_bias, None, grad_type))
    assert same_bits(layer.rest(grad), layer.rest(old))
    again = backward(layer, plan, dout, x, a, "silu", before, None, dx_type, old, False)
    assert same_bits(again[0], dx) and same_bits(again[1], grad)


@pytest.mark.parametrize("types", [shapes.WHOLE, shapes.FLOAT, shapes.SINGLE], ids=str)
def test_bad_numbers_stay_in_their_row_and_column(types):
    W, T, inputs, outputs, more = shapes.RANGE
    layer = Layer(W, inputs, outputs, **more)
    x_type, theta, out = (DTYPES[t] for t in types)
    a, x = layer.array(theta), randn((W, T, inputs), 2, x_type)
    x[0, 7, 3], x[1, T - 1, inputs - 1] = math.nan, math.inf
    layer.matrix(a)[0, inputs - 1, outputs - 1] = math.nan
    got, _ = forward(layer, layer.plan(T), x, a, "none", None, out, before=False)
    bad = torch.zeros(got.shape, dtype=torch.bool)
    bad[0, 7] = bad[1, T - 1] = True
    bad[0, :, outputs - 1] = True
    assert not got[bad].isfinite().any() and got[~bad].isfinite().all()


@pytest.mark.parametrize("types", [shapes.FLOAT, shapes.SINGLE], ids=str)
def test_operands_of_any_size(types):
    W, T, inputs, outputs, more = shapes.RANGE
    layer = Layer(W, inputs, outputs, **more)
    out = DTYPES[types[2]]
    plan = layer.plan(T)
    for size in (1e-15, 1e15):
        a, x = layer.array(torch.float32) * size, randn((W, T, inputs), 2) * size
        x[:, ::3] *= 1e-3
        got, _ = forward(layer, plan, x, a, "none", None, out, before=False)
        check_digits(got, x, layer.matrix(a), out, 2)
    zero, _ = forward(layer, plan, torch.zeros_like(x), a, "none", None, out, before=False)
    assert (zero == 0).all()
