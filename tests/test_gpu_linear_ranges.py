"""Large products whose operands have rows of very different sizes: what a padding position holds, or a row of nearly nothing, must not cost
other rows their digits. Every result is compared with its own row's size, in 64 bits."""
import pytest
import torch

import model_plain as plain
import product_shapes as shapes
from test_gpu_linear import DTYPES, Layer, backward, code, forward, nl, randn, same_bits, within

pytestmark = pytest.mark.gpu


def check_product(got, a, b, out):
    """got = a b with operands of 24 bits (float result) or 16 (bf16 result). Three bf16 parts leave 2^-24 of a number, and of their products
    twice 2^-24 is left out; two leave 2^-16 of each, and 2^-16 of the product. Six (three) products in binary32."""
    exact, sizes, k = a.double() @ b.double(), a.double().abs() @ b.double().abs(), a.shape[-1]
    rel = (6 * k + 8) * plain.U if out == torch.float32 else 3 * 2.0 ** -16 + (3 * k + 4) * plain.U
    within(got, exact, rel * sizes * plain.SLACK + plain.STORED[out] * exact.abs())
    if out == torch.float32:
        # the matrix cores add sixteen products at a time: 6 k / 16 roundings of random sign, less than 1e-6 at these sizes
        off, size = (got.double() - exact).norm(dim=-1), exact.norm(dim=-1)
        assert (off <= 1e-6 * size).all(), (off / size).max()


def rows_apart(x, how):
    """x with rows of worker 0 that lie far from the others; those of worker 1 stay."""
    x = x.float()
    if how == "one huge":
        x[0, 7] *= 1e30
    elif how == "one tiny":
        x[0, 7] *= 1e-15
    elif how == "falling":
        x[0] *= (10.0 ** -torch.linspace(0, 24, x.shape[1]))[:, None]
    return x


@pytest.mark.parametrize("how", ["one huge", "one tiny", "falling"])
@pytest.mark.parametrize("types", shapes.RANGE_TYPES, ids=str)
def test_rows_of_activations(types, how):
    W, T, inputs, outputs, more = shapes.RANGE
    layer = Layer(W, inputs, outputs, **more)
    x_type, theta, out = (DTYPES[t] for t in types)
    a, x = layer.array(theta, std=0.3), rows_apart(randn((W, T, inputs), 2), how).to(x_type)
    got, _ = forward(layer, layer.plan(T), x, a, "none", None, out, before=False)
    check_product(got, x, layer.matrix(a), out)


@pytest.mark.parametrize("how", ["one huge", "one tiny", "falling"])
@pytest.mark.parametrize("size", shapes.NARROW, ids=str)
def test_short_rows(size, how):
    W, T, inputs, outputs, more = size
    layer = Layer(W, inputs, outputs, **more)
    a, x = layer.array(torch.float32, std=0.3), rows_apart(randn((W, T, inputs), 2), how)
    got, _ = forward(layer, layer.plan(T), x, a, "none", None, torch.float32, before=False)
    check_product(got, x, layer.matrix(a), torch.float32)


@pytest.mark.parametrize("types", shapes.RANGE_TYPES, ids=str)
def test_rows_of_the_matrix(types):
    """One that belongs to an input that is zero everywhere."""
    W, T, inputs, outputs, more = shapes.RANGE
    layer = Layer(W, inputs, outputs, **more)
    x_type, theta, out = (DTYPES[t] for t in types)
    a, x = layer.array(theta, std=0.3), randn((W, T, inputs), 2, x_type)
    layer.matrix(a)[0, 11] *= 1e30
    x[0, :, 11] = 0
    got, _ = forward(layer, layer.plan(T), x, a, "none", None, out, before=False)
    check_product(got, x, layer.matrix(a), out)


@pytest.mark.parametrize("act", ["none", "relu"])
def test_padding_in_a_gradient(act):
    """Tokens whose x is anything and whose dout is zero: the matrix's gradient has none of them, dx zeros there. With relu dz is dout or zero."""
    W, T, inputs, outputs, more = shapes.RANGE
    layer = Layer(W, inputs, outputs, **more)
    a, x, dout = layer.array(torch.float32, std=0.3), randn((W, T, inputs), 2), randn((W, T, outputs), 3)
    x[0, 5::50] *= 1e25
    dout[0, 5::50] = 0
    dout[0, 6::50] *= 1e-12
    before = randn((W, T, outputs), 4) if act == "relu" else None
    dx, grad = backward(layer, layer.plan(T), dout, x, a, act, before, None, torch.float32, a, False)
    dz = dout if before is None else torch.where(before > 0, dout, 0.0)
    check_product(layer.matrix(grad), x.mT, dz, torch.float32)
    check_product(dx, dz, layer.matrix(a).mT, torch.float32)


@pytest.mark.parametrize("types", shapes.RANGE_TYPES, ids=str)
def test_bad_numbers_beside_rows_far_apart(types):
    """A NaN or an infinity makes its own row bad in a worker whose rows are far apart too; so does one next to binary32's end, which no bf16 but
    infinity is nearest to, not."""
    W, T, inputs, outputs, more = shapes.RANGE
    layer = Layer(W, inputs, outputs, **more)
    x_type, theta, out = (DTYPES[t] for t in types)
    a, x = layer.array(theta), rows_apart(randn((W, T, inputs), 2), "one huge").to(x_type)
    x[0, 30, 3], x[0, T - 1, inputs - 1] = float("nan"), float("inf")
    x[0, 60] = 0
    x[0, 60, 4] = torch.finfo(x_type).max
    layer.matrix(a)[0, 4] = 1e-9
    got, _ = forward(layer, layer.plan(T), x, a, "none", None, out, before=False)
    bad = torch.zeros((W, T), dtype=torch.bool)
    bad[0, 30] = bad[0, T - 1] = True
    assert not got[bad].isfinite().any() and got[~bad].isfinite().all()
    exact = (x[0, 60].double() @ layer.matrix(a)[0].double())
    assert ((got[0, 60].double() - exact).abs() <= 2 * plain.STORED[out] * exact.abs() + 2.0 ** -15 * exact.abs() * (out == torch.bfloat16) + 16 * plain.U * exact.abs()).all()


def test_lowest_numbers_that_meet_zeros():
    """A float operand beside a bf16 one, rounded to bf16: binary32's lowest number, nearest to -infinity, has to stay finite."""
    W, T, inputs, outputs, more = shapes.RANGE
    layer = Layer(W, inputs, outputs, **more)
    lowest = torch.finfo(torch.float32).min
    a, x, dout = layer.array(torch.bfloat16, std=0.3), randn((W, T, inputs), 2), randn((W, T, outputs), 3, torch.bfloat16)
    x[0, 5::50] = lowest
    dout[0, 5::50] = 0
    _, grad = backward(layer, layer.plan(T), dout, x, a, "none", None, None, torch.bfloat16, a, False)
    exact, bound = plain.product(x.mT, dout, torch.bfloat16)
    within(layer.matrix(grad), exact, bound + plain.STORED[torch.bfloat16] * exact.abs())
    a, x = layer.array(torch.float32, std=0.3), randn((W, T, inputs), 2, torch.bfloat16)
    layer.matrix(a)[0, 11] = lowest
    x[0, :, 11] = 0
    got, _ = forward(layer, layer.plan(T), x, a, "none", None, torch.bfloat16, before=False)
    exact, bound = plain.product(x, layer.matrix(a), torch.bfloat16)
    within(got, exact, bound + plain.STORED[torch.bfloat16] * exact.abs())


@pytest.mark.parametrize("types", shapes.RANGE_TYPES[::3], ids=str)
def test_captured_and_replayed_with_rows_near_and_far(types):
    """One graph, whose operands' rows lie near each other and far apart in turn, eager calls between."""
    W, T, inputs, outputs, more = shapes.RANGE
    layer = Layer(W, inputs, outputs, **more)
    x_type, theta_type, out_type = (DTYPES[t] for t in types)
    a = layer.array(theta_type, std=0.3)
    plan, theta, x = layer.plan(T), a.cuda(), randn((W, T, inputs), 2, x_type).cuda()
    out = torch.empty((W, T, outputs), dtype=out_type, device="cuda")
    step = lambda: nl.linear(plan, 1, x, code(x), theta, code(theta), T, out, code(out))  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay, how in enumerate(("", "one huge", "", "falling")):
        host = rows_apart(randn((W, T, inputs), 10 + replay), how).to(x_type)
        x.copy_(host)
        step()
        torch.cuda.synchronize()
        want = out.clone()
        for _ in range(2):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert same_bits(out, want)
        if how:
            check_product(out.cpu(), host, layer.matrix(a), out_type)
