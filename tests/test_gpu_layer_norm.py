"""Layer norm and its gradient on the GPU, against the plain form in 64 bits."""
import math

import pytest
import torch

import model_plain as plain

pytestmark = pytest.mark.gpu
nl = pytest.importorskip("paper_2506_10911_amd")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


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


def arena(W, width, gap, bias, dtype, seed=0):
    """(array with NaN around weight and bias, weight's place, bias's place or -1, stride)"""
    at, behind = gap, gap + width + (3 if gap % 2 else 0)
    stride = -(-(behind + width + 5) // 64) * 64
    a = torch.full((W, stride), float("nan"))
    a[:, at:at + width] = 1 + 0.2 * randn((W, width), seed)
    if bias:
        a[:, behind:behind + width] = 0.3 * randn((W, width), seed + 1)
    return a.to(dtype), at, behind if bias else -1, stride


SIZES = [  # W, T, width, gap, bias
    (1, 1, 1, 0, True), (2, 3, 2, 1, True), (3, 5, 7, 0, False), (2, 61, 129, 0, True), (1, 9, 64, 4, True), (2, 33, 768, 0, True),
    (3, 4, 1000, 8, False), (2, 5, 1024, 2, True), (1, 6, 1025, 0, True), (2, 7, 2048, 0, True), (1, 5, 4096, 0, True), (1, 3, 4100, 4, True),
    (1, 2, 9000, 0, False), (2, 3, 16384, 0, True), (1, 3, 16385, 1, True), (2, 2, 20000, 0, True), (5, 2100, 24, 0, True), (1, 5000, 36, 0, True),
]


def run_norm(a, x, at, bias, stride, out_dtype, T=None, stats=True, stream=None, max_tokens=None, eps=EPS):
    W, T, width = x.shape
    plan = nl.LayerNormPlan([(0, None, 1), (at, bias, width)], stride, W, max_tokens or T)
    out = torch.full(x.shape, 9.0, dtype=out_dtype, device="cuda")
    kept = torch.full((W, T, 2), 9.0, device="cuda") if stats else None
    nl.layer_norm(plan, 1, x.cuda(), code(x), a.cuda(), code(a), T, eps, out, nl.BF16 if out_dtype == torch.bfloat16 else nl.F32,
                  stats=kept, stream=stream)
    return out.cpu(), kept.cpu() if stats else None


@pytest.mark.parametrize("x,theta,out", [("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "bf16"), ("bf16", "bf16", "f32")])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_norm(size, x, theta, out):
    W, T, width, gap, has_bias = size
    a, at, bias, stride = arena(W, width, gap, has_bias, DTYPES[theta])
    x = (randn((W, T, width), 2, std=1.5) + 0.5).to(DTYPES[x])
    got, stats = run_norm(a, x, at, bias, stride, DTYPES[out])
    (want, bound), (want_stats, stats_bound) = plain.layer_norm(x, a[:, at:at + width], a[:, bias:bias + width] if has_bias else None, EPS, DTYPES[out])
    within(got, want, bound)
    within(stats, want_stats, stats_bound)
    again, _ = run_norm(a, x, at, bias, stride, DTYPES[out], stats=False, max_tokens=T + 100)
    assert same_bits(got, again)


def test_norm_of_rows_far_from_zero():
    """The variance is that of the distances: a mean of 3000 beside a spread of 1 costs what x itself has lost."""
    a, at, bias, stride = arena(1, 768, 0, True, torch.float32)
    x = randn((1, 40, 768), 3) + 3000
    got, stats = run_norm(a, x, at, bias, stride, torch.float32)
    (want, bound), _ = plain.layer_norm(x, a[:, :768], a[:, bias:bias + 768], EPS, torch.float32)
    within(got, want, bound)
    assert (got.double() - want).abs().max() < 0.02


def test_norm_keeps_bad_rows_to_themselves():
    a, at, bias, stride = arena(2, 40, 0, True, torch.float32)
    x = randn((2, 9, 40), 4)
    clean, _ = run_norm(a, x, at, bias, stride, torch.float32)
    x[0, 3, 7], x[1, 0, 0], x[1, 8, 39] = math.nan, math.inf, -math.inf
    got, _ = run_norm(a, x, at, bias, stride, torch.float32)
    bad = torch.zeros((2, 9), dtype=torch.bool)
    bad[0, 3] = bad[1, 0] = bad[1, 8] = True
    assert got[bad].isnan().all() and same_bits(got[~bad], clean[~bad])


def test_norm_of_constant_rows():
    a, at, bias, stride = arena(1, 50, 0, True, torch.float32)
    x = torch.full((1, 3, 50), 2.5)
    got, stats = run_norm(a, x, at, bias, stride, torch.float32)
    assert torch.equal(got[0], a[:, bias:bias + 50].expand(3, 50)) and torch.equal(stats[0, :, 0], torch.full((3,), 2.5))


def gradient(a, at, bias, stride, dout, x, stats, dx_dtype, grad, accumulate, add=None, in_place=False, wants_grad=True, stream=None):
    W, T, width = x.shape
    plan = nl.LayerNormPlan([(at, bias, width)], stride, W, T)
    dx = add.cuda() if in_place else torch.full(x.shape, 9.0, dtype=dx_dtype, device="cuda")
    more = dx if in_place else (None if add is None else add.cuda())
    grad = grad.cuda() if wants_grad else None
    nl.layer_norm_gradient(plan, 0, dout.cuda(), code(dout), x.cuda(), code(x), a.cuda(), code(a), stats.cuda(), T, dx, code(dx), grad,
                           code(grad) if wants_grad else nl.F32, accumulate=accumulate, add=more, stream=stream)
    return dx.cpu(), grad.cpu() if wants_grad else None


def check_gradient(size, dout, x, theta, dx, grad, accumulate, with_add):
    W, T, width, gap, has_bias = size
    a, at, bias, stride = arena(W, width, gap, has_bias, DTYPES[theta])
    x = (randn((W, T, width), 2, std=1.5) + 0.5).to(DTYPES[x])
    dout = randn((W, T, width), 3, DTYPES[dout])
    add = randn((W, T, width), 4, DTYPES[dx]) if with_add else None
    old = arena(W, width, gap, has_bias, DTYPES[grad], seed=5)[0]
    stats = plain.layer_norm(x, a[:, at:at + width], None, EPS, torch.float32)[1][0].float()
    got, of_weights = gradient(a, at, bias, stride, dout, x, stats, DTYPES[dx], old, accumulate, add)
    (want, bound), *grads = plain.layer_norm_gradient(dout, x, a[:, at:at + width], stats, add, DTYPES[dx])
    within(got, want, bound)
    untouched = torch.ones(a.shape[1], dtype=torch.bool)
    for place, (value, off) in zip((at, bias), grads):
        if place < 0:
            continue
        part = slice(place, place + width)
        within(of_weights[:, part], *plain.stored(value, off, old[:, part] if accumulate else None, DTYPES[grad]))
        untouched[part] = False
    assert same_bits(of_weights[:, untouched], old[:, untouched])
    again, again_grad = gradient(a, at, bias, stride, dout, x, stats, DTYPES[dx], old, accumulate, add, in_place=with_add)
    assert same_bits(got, again) and same_bits(of_weights, again_grad)
    alone, _ = gradient(a, at, bias, stride, dout, x, stats, DTYPES[dx], old, accumulate, add, wants_grad=False)
    assert same_bits(got, alone)


@pytest.mark.parametrize("types", [("f32", "f32", "f32", "f32", "f32"), ("bf16", "bf16", "f32", "bf16", "f32"), ("bf16", "bf16", "bf16", "bf16", "bf16"),
                                   ("bf16", "f32", "bf16", "f32", "bf16")], ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradient(size, types):
    check_gradient(size, *types, accumulate=size[1] % 2 == 0, with_add=size[2] % 2 == 0)


@pytest.mark.parametrize("accumulate,with_add", [(False, False), (True, False), (False, True), (True, True)])
def test_gradient_added_and_written(accumulate, with_add):
    check_gradient((2, 50, 100, 0, True), "bf16", "bf16", "f32", "bf16", "f32", accumulate, with_add)


def test_gradient_is_that_of_differences():
    """Central differences of the norm in 64 bits."""
    W, T, width = 1, 2, 6
    a, at, bias, stride = arena(W, width, 0, True, torch.float32)
    x, dout = randn((W, T, width), 6), randn((W, T, width), 7)
    stats = plain.layer_norm(x, a[:, :width], None, EPS, torch.float32)[1][0].float()
    dx, grad = gradient(a, at, bias, stride, dout, x, stats, torch.float32, torch.zeros_like(a), False)

    def value(x, weight, b):
        return (plain.layer_norm(x, weight, b, EPS, torch.float32)[0][0] * dout.double()).sum().item()

    inputs = [x.double(), a[:, :width].double(), a[:, bias:bias + width].double()]
    for which, got in enumerate((dx, grad[:, :width], grad[:, bias:bias + width])):
        for i in range(inputs[which].numel()):
            ends = []
            for step in (1e-4, -1e-4):
                moved = [v.clone() for v in inputs]
                moved[which].view(-1)[i] += step
                ends.append(value(*moved))
            # third derivatives are at most some hundreds at these sizes: 1e-8 of them, and the float result
            assert abs((ends[0] - ends[1]) / 2e-4 - got.reshape(-1)[i].item()) < 2e-5


def test_no_tokens():
    a, at, bias, stride = arena(2, 10, 0, True, torch.float32)
    plan = nl.LayerNormPlan([(at, bias, 10)], stride, 2, 4)
    x = torch.zeros((2, 0, 10), device="cuda")
    grad = a.cuda()
    nl.layer_norm(plan, 0, None, nl.F32, grad, nl.F32, 0, EPS, None, nl.F32)
    theta = a.cuda()
    nl.layer_norm_gradient(plan, 0, x, nl.F32, x, nl.F32, theta, nl.F32, None, 0, x, nl.F32, grad, nl.F32, accumulate=True)
    assert same_bits(grad.cpu(), a)
    nl.layer_norm_gradient(plan, 0, x, nl.F32, x, nl.F32, theta, nl.F32, None, 0, x, nl.F32, grad, nl.F32)
    assert (grad[:, :10] == 0).all() and (grad[:, bias:bias + 10] == 0).all() and grad[:, bias + 10:].isnan().all()


def test_captured_and_on_another_stream():
    """Forward and gradient in one graph, replayed with new inputs and eager work between."""
    W, T, width = 2, 300, 200
    a, at, bias, stride = arena(W, width, 0, True, torch.float32)
    theta, x, dout = a.cuda(), randn((W, T, width), 1, torch.bfloat16).cuda(), randn((W, T, width), 2, torch.bfloat16).cuda()
    plan = nl.LayerNormPlan([(at, bias, width)], stride, W, T)
    out, dx, stats, grad = torch.empty_like(x), torch.empty_like(x), torch.empty((W, T, 2), device="cuda"), torch.zeros_like(theta)

    def both(stream=None):
        nl.layer_norm(plan, 0, x, nl.BF16, theta, nl.F32, T, EPS, out, nl.BF16, stats=stats, stream=stream)
        nl.layer_norm_gradient(plan, 0, dout, nl.BF16, x, nl.BF16, theta, nl.F32, stats, T, dx, nl.BF16, grad, nl.F32, stream=stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for replay in range(3):
        x.copy_(randn((W, T, width), 10 + replay, torch.bfloat16))
        both()
        torch.cuda.synchronize()
        want = [t.clone() for t in (out, dx, stats, grad)]
        for t in (out, dx, stats, grad):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same_bits(t, w) for t, w in zip((out, dx, stats, grad), want))
        for t in (out, dx, stats, grad):
            t.zero_()
        torch.cuda.synchronize()
        both(stream=side)
        torch.cuda.synchronize()
        assert all(same_bits(t, w) for t, w in zip((out, dx, stats, grad), want))
