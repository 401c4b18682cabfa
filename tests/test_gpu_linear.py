"""Matrices with bias, activation and residual and their gradient on the GPU, against the plain form in 64 bits."""
import math

import pytest
import torch

import model_plain as plain

pytestmark = pytest.mark.gpu
nl = pytest.importorskip("paper_2506_10911_amd")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


def code(t):
    return nl.BF16 if t.dtype == torch.bfloat16 else nl.F32


def same_bits(a, b):
    kind = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


def within(got, want, bound):
    off = (got.double() - want).abs() - bound
    assert not (off > 0).any() and not got.isnan().any(), off.max()


def randn(shape, seed, dtype=torch.float32, std=1.0):
    return (std * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(dtype)


class Layer:
    """A matrix in rows of NaN: behind `gap` elements, its rows `apart` elements further apart than they are long."""

    def __init__(self, W, inputs, outputs, bias=True, transposed=False, gap=0, apart=0):
        self.W, self.inputs, self.outputs, self.transposed = W, inputs, outputs, transposed
        self.rows, self.cols = (outputs, inputs) if transposed else (inputs, outputs)
        self.at, self.row_stride = gap, self.cols + apart
        end = gap + self.rows * self.row_stride
        self.bias = end + (gap & 1) if bias else -1
        self.stride = -(-(end + outputs + 3) // 64) * 64
        self.layer = (self.at, inputs, outputs, self.bias, transposed, self.row_stride)

    def plan(self, T, room=0):
        return nl.LinearPlan([(0, 1, 1), self.layer], self.stride, self.W, T, room)

    def array(self, dtype, seed=0, std=1.0):
        a = torch.full((self.W, self.stride), float("nan"))
        self.matrix(a).copy_(std * randn((self.W, self.inputs, self.outputs), seed))
        if self.bias >= 0:
            self.of_bias(a).copy_(std * randn((self.W, self.outputs), seed + 1))
        return a.to(dtype)

    def matrix(self, a):
        m = a.as_strided((self.W, self.rows, self.cols), (self.stride, self.row_stride, 1), self.at)
        return m.mT if self.transposed else m

    def of_bias(self, a):
        return a[:, self.bias:self.bias + self.outputs] if self.bias >= 0 else None

    def rest(self, a):
        a = a.clone()
        self.matrix(a).zero_()
        if self.bias >= 0:
            self.of_bias(a).zero_()
        return a


SIZES = [  # W, T, inputs, outputs, more of Layer
    (1, 1, 1, 1, {}), (2, 3, 5, 7, dict(gap=1)), (3, 61, 129, 33, {}), (1, 128, 128, 128, {}), (2, 130, 96, 192, dict(gap=8)),
    (1, 129, 64, 257, dict(bias=False)), (2, 100, 72, 40, dict(transposed=True)), (1, 257, 200, 264, dict(apart=8)), (2, 64, 33, 65, dict(transposed=True, apart=3)),
    (1, 40, 520, 24, dict(gap=4, bias=False)), (4, 1, 300, 150, {}), (1, 5, 1032, 136, {}), (1, 300, 256, 512, {}),
]
TYPES = [("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("f32", "bf16", "bf16"), ("bf16", "bf16", "f32")]


def forward(layer, plan, x, a, act, residual, out_dtype, before=True, in_place=False, stream=None):
    W, T = x.shape[:2]
    out = residual.cuda() if in_place else torch.full((W, T, layer.outputs), 9.0, dtype=out_dtype, device="cuda")
    more = out if in_place else (None if residual is None else residual.cuda())
    z = torch.full((W, T, layer.outputs), 9.0, dtype=out_dtype, device="cuda") if before else None
    nl.linear(plan, 1, x.cuda(), code(x), a.cuda(), code(a), T, out, code(out), activation=ACTS[act], residual=more, before=z, stream=stream)
    return out.cpu(), z.cpu() if before else None


def check_forward(size, types, act, with_residual):
    W, T, inputs, outputs, more = size
    layer = Layer(W, inputs, outputs, **more)
    x, theta, out = (DTYPES[t] for t in types)
    a, x = layer.array(theta, std=0.3), randn((W, T, inputs), 2, x)
    residual = randn((W, T, outputs), 3, out) if with_residual else None
    plan = layer.plan(T)
    got, before = forward(layer, plan, x, a, act, residual, out)
    wanted = plain.linear(x, layer.matrix(a), layer.of_bias(a), act, residual, out)
    within(got, *wanted[0])
    within(before, *wanted[1])
    again, _ = forward(layer, plan, x, a, act, residual, out, before=False, in_place=with_residual)
    assert same_bits(got, again)


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear(size, types):
    check_forward(size, types, "none", with_residual=size[1] % 2 == 0)


@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("act", list(ACTS))
def test_linear_with_activations(act, types, with_residual):
    check_forward((2, 70, 40, 72, {}), types, act, with_residual)


def test_activations_of_large_and_bad_numbers():
    """z itself as x, through a matrix of one: where the functions end, and what is no number."""
    z = torch.tensor([0.0, -0.0, 1e-20, -1e-20, 5.0, -5.0, 12.0, -12.0, 40.0, -40.0, 300.0, -300.0, 1e4, -1e4, 1e18, -1e18, 3e38])
    layer = Layer(1, 1, 1, bias=False)
    a = torch.ones((1, layer.stride))
    x = z.view(1, -1, 1)
    plan = layer.plan(len(z) + 2)
    for act in ACTS:
        got, _ = forward(layer, plan, x, a, act, None, torch.float32)
        want = plain.activation(act, z.double().clamp(-1e100, 1e100))[0]
        # functions of 4 U, of arguments whose rounding a tail of exp(-z^2 / 2) or less multiplies by z^2
        assert ((got.view(-1).double() - want).abs() <= 16 * plain.U * want.abs() * (1 + z.double().square().clamp(max=200)) + 1e-37).all(), act
        bad, _ = forward(layer, plan, torch.tensor([math.nan, 1.0]).view(1, 2, 1), a, act, None, torch.float32)
        assert bad[0, 0].isnan().all() and bad[0, 1].isfinite().all()


@pytest.mark.parametrize("types", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16")], ids=str)
def test_bad_numbers_stay_in_their_row_and_column(types):
    layer = Layer(2, 50, 70)
    x, theta, out = (DTYPES[t] for t in types)
    a, x = layer.array(theta), randn((2, 40, 50), 2, x)
    x[0, 7, 3] = math.nan
    x[1, 39, 49] = math.inf
    layer.matrix(a)[0, 49, 69] = math.nan
    got, _ = forward(layer, layer.plan(40), x, a, "none", None, out)
    bad = torch.zeros(got.shape, dtype=torch.bool)
    bad[0, 7] = bad[1, 39] = True
    bad[0, :, 69] = True
    assert not got[bad].isfinite().any() and got[~bad].isfinite().all()


def test_float_products_keep_their_digits():
    """Operands that differ from bf16 in their last bits, of every size that binary32 has room for."""
    layer = Layer(1, 64, 48, bias=False)
    for size in (1.0, 1e-12, 1e12):
        a, x = layer.array(torch.float32) * size, randn((1, 40, 64), 2) * size
        got, _ = forward(layer, layer.plan(40), x, a, "none", None, torch.float32)
        want, bound = plain.product(x, layer.matrix(a), torch.float32)
        within(got, want, bound)
        assert ((got.double() - want).norm() / want.norm()).item() < 4e-7


def backward(layer, plan, dout, x, a, act, before, add, dx_dtype, grad, accumulate, in_place=False, wants=(True, True), stream=None):
    W, T = dout.shape[:2]
    dx = None
    if wants[0]:
        dx = add.cuda() if in_place else torch.full((W, T, layer.inputs), 9.0, dtype=dx_dtype, device="cuda")
    more = dx if in_place else (None if add is None else add.cuda())
    grad = grad.cuda() if wants[1] else None
    nl.linear_gradient(plan, 1, dout.cuda(), code(dout), x.cuda() if wants[1] else None, code(x), a.cuda(), code(a), T, dx,
                       nl.BF16 if dx_dtype == torch.bfloat16 else nl.F32, grad, code(grad) if wants[1] else nl.F32, activation=ACTS[act],
                       before=None if before is None else before.cuda(), accumulate=accumulate, add=more if wants[0] else None, stream=stream)
    return None if dx is None else dx.cpu(), None if grad is None else grad.cpu()


def check_gradient(size, types, act, with_add, accumulate, room=0):
    W, T, inputs, outputs, more = size
    layer = Layer(W, inputs, outputs, **more)
    dout, x, theta, dx, grad = (DTYPES[t] for t in types)
    a, x, dout = layer.array(theta, std=0.3), randn((W, T, inputs), 2, x), randn((W, T, outputs), 3, dout)
    before = randn((W, T, outputs), 4, dout.dtype) if act != "none" else None
    add = randn((W, T, inputs), 5, dx) if with_add else None
    old = layer.array(grad, seed=6)
    plan = layer.plan(T, room)
    got, of_weights = backward(layer, plan, dout, x, a, act, before, add, dx, old, accumulate)
    of_dx, of_matrix, of_bias = plain.linear_gradient(dout, x, layer.matrix(a), before, act, add, dx, grad)
    within(got, *of_dx)
    within(layer.matrix(of_weights), *plain.stored(*of_matrix, layer.matrix(old) if accumulate else None, grad))
    if layer.bias >= 0:
        within(layer.of_bias(of_weights), *plain.stored(*of_bias, layer.of_bias(old) if accumulate else None, grad))
    assert same_bits(layer.rest(of_weights), layer.rest(old))
    again, again_weights = backward(layer, plan, dout, x, a, act, before, add, dx, old, accumulate, in_place=with_add)
    assert same_bits(got, again) and same_bits(of_weights, again_weights)
    if dx == grad:
        assert same_bits(backward(layer, plan, dout, x, a, act, before, add, dx, old, accumulate, wants=(True, False))[0], got)
        assert same_bits(backward(layer, plan, dout, x, a, act, before, add, dx, old, accumulate, wants=(False, True))[1], of_weights)


GRADIENT_TYPES = [("f32", "f32", "f32", "f32", "f32"), ("bf16", "bf16", "f32", "bf16", "f32"), ("bf16", "bf16", "bf16", "bf16", "bf16"),
                  ("f32", "bf16", "f32", "bf16", "bf16"), ("bf16", "f32", "bf16", "f32", "f32")]


@pytest.mark.parametrize("types", GRADIENT_TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradient(size, types):
    check_gradient(size, types, "none", with_add=size[1] % 2 == 0, accumulate=size[2] % 2 == 0)


@pytest.mark.parametrize("accumulate,with_add", [(False, False), (True, True)])
@pytest.mark.parametrize("types", GRADIENT_TYPES, ids=str)
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_gradient_through_activations(act, types, accumulate, with_add):
    check_gradient((2, 70, 40, 72, {}), types, act, with_add, accumulate)


# Large products: what is packed and what is not, every tile, k shared out, edges within a tile, a stage and a vector.
LARGE = [  # W, T, inputs, outputs, more of Layer
    (1, 1, 16392, 16408, {}), (2, 20, 2600, 2704, dict(transposed=True)), (1, 31, 3001, 2999, {}), (1, 300, 1000, 1000, dict(gap=1)), (1, 520, 712, 776, {}),
    (2, 130, 1064, 1048, dict(transposed=True, apart=8)), (4, 2041, 72, 2056, {}), (1, 4099, 4100, 64, dict(bias=False)), (1, 64, 2056, 2072, {}),
    (3, 333, 515, 517, dict(transposed=True)),
]


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_large_linear(size, types):
    check_forward(size, types, "none" if size[1] % 2 else "gelu", with_residual=size[1] % 2 == 0)


@pytest.mark.parametrize("types", [("f32", "f32", "f32", "f32", "f32"), ("bf16", "bf16", "f32", "bf16", "f32"), ("bf16", "bf16", "bf16", "bf16", "bf16")], ids=str)
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_large_gradient(size, types):
    check_gradient(size, types, "none" if size[1] % 2 else "silu", with_add=size[1] % 2 == 0, accumulate=size[2] % 2 == 0)


@pytest.mark.parametrize("types", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "bf16")], ids=str)
@pytest.mark.parametrize("size", [(1, 1024, 4096, 2048, {}), (1, 1030, 4104, 2051, dict(gap=1))], ids=str)
def test_large_linear_joined_in_vectors(size, types):
    """Results of 2^18 vectors and more whose k is shared out, with and without rows that end within a vector."""
    check_forward(size, types, "silu", with_residual=True)


@pytest.mark.parametrize("types", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "f32", "bf16")], ids=str)
def test_large_products_keep_bad_numbers_to_their_row_and_column(types):
    layer = Layer(2, 712, 776)
    x, theta, out = (DTYPES[t] for t in types)
    a, x = layer.array(theta), randn((2, 300, 712), 2, x)
    x[0, 7, 3] = math.nan
    x[1, 299, 711] = math.inf
    layer.matrix(a)[0, 711, 775] = math.nan
    got, _ = forward(layer, layer.plan(300), x, a, "none", None, out)
    bad = torch.zeros(got.shape, dtype=torch.bool)
    bad[0, 7] = bad[1, 299] = True
    bad[0, :, 775] = True
    assert not got[bad].isfinite().any() and got[~bad].isfinite().all()


def test_large_products_of_any_size():
    """Float operands of every size that binary32 has room for, and of sizes that lie far apart."""
    layer = Layer(1, 712, 776, bias=False)
    for size in (1e-15, 1e15):
        a, x = layer.array(torch.float32) * size, randn((1, 520, 712), 2) * size
        x[:, ::3] *= 1e-3
        got, _ = forward(layer, layer.plan(520), x, a, "none", None, torch.float32)
        within(got, *plain.product(x, layer.matrix(a), torch.float32))
    zero, _ = forward(layer, layer.plan(520), torch.zeros((1, 520, 712)), a, "none", None, torch.float32)
    assert (zero == 0).all()


def test_gradient_in_batches_of_workers():
    """A workspace that has room for one worker, or for two of five."""
    check_gradient((5, 70, 40, 72, {}), GRADIENT_TYPES[0], "gelu", True, True, room=1)
    check_gradient((5, 70, 40, 72, {}), GRADIENT_TYPES[1], "silu", True, False, room=4 * (70 * 72 * 4 + 4096))
    check_gradient((5, 300, 520, 456, {}), GRADIENT_TYPES[0], "gelu", True, False, room=1)
    check_gradient((5, 300, 520, 456, {}), GRADIENT_TYPES[1], "gelu", True, False, room=8 << 20)


def test_gradient_of_activations_is_that_of_differences():
    """Of z by z, through a matrix of one."""
    z = torch.cat([torch.linspace(-6, 6, 49), torch.tensor([-30.0, 30.0])])
    layer = Layer(1, 1, 1, bias=False)
    a = torch.ones((1, layer.stride))
    for act in ("gelu", "gelu_tanh", "silu"):
        dx, _ = backward(layer, layer.plan(len(z)), torch.ones((1, len(z), 1)), z.view(1, -1, 1), a, act, z.view(1, -1, 1), None, torch.float32, a, False)
        ends = [plain.activation(act, z.double() + step)[0] for step in (1e-4, -1e-4)]
        # third derivatives below 2: 1e-8 of them, and the result's own roundings
        assert ((ends[0] - ends[1]) / 2e-4 - dx.view(-1).double()).abs().max() < 1e-5


@pytest.mark.parametrize("value", [0.0, -0.0])
def test_slope_of_relu_at_zero(value):
    layer = Layer(1, 1, 1, bias=False)
    a = torch.ones((1, layer.stride))
    dx, _ = backward(layer, layer.plan(1), torch.ones((1, 1, 1)), torch.ones((1, 1, 1)), a, "relu", torch.full((1, 1, 1), value), None, torch.float32, a, False)
    assert dx.item() == 0.0


def test_no_tokens():
    layer = Layer(2, 10, 6)
    a = layer.array(torch.float32)
    theta, got = a.cuda(), a.cuda()
    plan = layer.plan(4)
    nl.linear(plan, 1, None, nl.F32, theta, nl.F32, 0, None, nl.F32)
    nl.linear_gradient(plan, 1, None, nl.F32, None, nl.F32, theta, nl.F32, 0, None, nl.F32, got, nl.F32, accumulate=True)
    assert same_bits(got.cpu(), a)
    nl.linear_gradient(plan, 1, None, nl.F32, None, nl.F32, theta, nl.F32, 0, None, nl.F32, got, nl.F32, activation=nl.ACT_GELU)
    assert (layer.matrix(got.cpu()) == 0).all() and (layer.of_bias(got.cpu()) == 0).all() and same_bits(layer.rest(got.cpu()), layer.rest(a))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_captured_and_on_another_stream(kind):
    layer = Layer(2, 96, 160)
    W, T, dtype = 2, 200, DTYPES[kind]
    theta, x, dout = layer.array(dtype).cuda(), randn((W, T, 96), 1, dtype).cuda(), randn((W, T, 160), 2, dtype).cuda()
    plan, number = layer.plan(T), code(theta)
    out, before, dx, grad = torch.empty_like(dout), torch.empty_like(dout), torch.empty_like(x), torch.zeros_like(theta)

    def both(stream=None):
        nl.linear(plan, 1, x, number, theta, number, T, out, number, activation=nl.ACT_GELU, before=before, stream=stream)
        nl.linear_gradient(plan, 1, dout, number, x, number, theta, number, T, dx, number, grad, number, activation=nl.ACT_GELU, before=before,
                           stream=stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for replay in range(3):
        x.copy_(randn((W, T, 96), 10 + replay, dtype))
        both()
        torch.cuda.synchronize()
        want = [t.clone() for t in (out, before, dx, grad)]
        for run in (graph.replay, lambda: both(stream=side)):
            for t in (out, before, dx, grad):
                t.zero_()
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
            assert all(same_bits(t, w) for t, w in zip((out, before, dx, grad), want))
