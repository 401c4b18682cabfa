"""The operators of a replica's inner step together, as they are used: table lookup, norm, two matrices with activation and residual,
norm, the tied table as output head, the loss, and all of it backwards, for every worker at once; and arrays whose offsets
pass 32 bits."""
import math

import pytest
import torch

import model_plain as plain

pytestmark = pytest.mark.gpu
nl = pytest.importorskip("paper_2506_10911_amd")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


class Model:
    """Places of the tensors in a worker's row, in the order of a GPT-style block."""

    def __init__(self, W, vocab, width, hidden):
        self.W, self.vocab, self.width, self.hidden = W, vocab, width, hidden
        self.places, at = {}, 3                               # odd places
        for name, shape in (("table", (vocab, width)), ("w1", (width,)), ("b1", (width,)), ("up", (width, hidden)), ("up_b", (hidden,)),
                            ("down", (hidden, width)), ("down_b", (width,)), ("w2", (width,)), ("b2", (width,))):
            self.places[name] = (at, shape)
            at += math.prod(shape) + 1
        self.stride = -(-at // 64) * 64

    def views(self, array):
        return {name: array[:, at:at + math.prod(shape)].unflatten(1, shape) for name, (at, shape) in self.places.items()}

    def theta(self, dtype, seed=0):
        gen = torch.Generator().manual_seed(seed)
        a = torch.full((self.W, self.stride), float("nan"))
        for name, view in self.views(a).items():
            scale = 1.0 if name == "table" else (0.1 if len(view.shape) == 2 else 1 / math.sqrt(view.shape[1]))
            view.copy_(scale * torch.randn(view.shape, generator=gen) + (1.0 if name in ("w1", "w2") else 0.0))
        return a.to(dtype)


def exact(model, theta, tokens, targets, unit=0.0, gen=None):
    """(log_probs, gradients) in 64 bits of the mean loss of every worker. With `gen` everything that the operators store, forward and
    backward, is off by up to `unit` of itself."""
    class Stored(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return noisy(x)

        @staticmethod
        def backward(ctx, d):
            return noisy(d)

    def noisy(x):
        return x if gen is None else x * (1 + unit * (2 * torch.rand(x.shape, dtype=torch.float64, generator=gen) - 1))

    def norm(x, w, b):
        d = x - x.mean(-1, keepdim=True)
        return d * (d.square().mean(-1, keepdim=True) + EPS).rsqrt() * w[:, None] + b[:, None]

    keep = Stored.apply
    leaf = theta.double().nan_to_num(0.0).requires_grad_()
    v = model.views(leaf)
    x = keep(torch.stack([t[i] for t, i in zip(v["table"], tokens)]))
    z = keep(keep(norm(x, v["w1"], v["b1"])) @ v["up"] + v["up_b"][:, None])
    h = keep(keep(plain.activation("gelu", z)[0]) @ v["down"] + v["down_b"][:, None] + x)
    logits = keep(keep(norm(h, v["w2"], v["b2"])) @ v["table"].mT)
    there = targets >= 0
    lp = torch.where(there, logits.log_softmax(-1).gather(-1, targets.clamp(min=0)[..., None])[..., 0], 0.0)
    (-lp.sum() / targets.shape[1]).backward()
    return lp.detach(), leaf.grad


def run(model, plans, theta, tokens, targets, kind, buffers):
    """The same with the operators; gradients in buffers["grad"]."""
    embedding, norms, matrices, loss = plans
    W, T = tokens.shape
    k, b = (nl.BF16 if kind == torch.bfloat16 else nl.F32), buffers
    nl.embed_lookup(embedding, theta, k, tokens, nl.I64, T, 1.0, b["x"], k)
    nl.layer_norm(norms, 0, b["x"], k, theta, k, T, EPS, b["n1"], k, stats=b["s1"])
    nl.linear(matrices, 0, b["n1"], k, theta, k, T, b["a"], k, activation=nl.ACT_GELU, before=b["z"])
    nl.linear(matrices, 1, b["a"], k, theta, k, T, b["h"], k, residual=b["x"])
    nl.layer_norm(norms, 1, b["h"], k, theta, k, T, EPS, b["n2"], k, stats=b["s2"])
    nl.linear(matrices, 2, b["n2"], k, theta, k, T, b["logits"], k)
    nl.token_log_probs(loss, b["logits"], k, targets, nl.I64, T, b["lp"], norms=b["ln"])
    # backwards: the logits' gradient in their place, the residual branch's where it is added to
    nl.token_log_probs_gradient(loss, b["logits"], k, targets, nl.I64, T, b["ln"], b["by"], b["logits"], k)
    nl.linear_gradient(matrices, 2, b["logits"], k, b["n2"], k, theta, k, T, b["d"], k, b["grad"], k)
    nl.layer_norm_gradient(norms, 1, b["d"], k, b["h"], k, theta, k, b["s2"], T, b["dh"], k, b["grad"], k)
    nl.linear_gradient(matrices, 1, b["dh"], k, b["a"], k, theta, k, T, b["da"], k, b["grad"], k)
    nl.linear_gradient(matrices, 0, b["da"], k, b["n1"], k, theta, k, T, b["d"], k, b["grad"], k, activation=nl.ACT_GELU, before=b["z"])
    nl.layer_norm_gradient(norms, 0, b["d"], k, b["x"], k, theta, k, b["s1"], T, b["dh"], k, b["grad"], k, add=b["dh"])
    nl.embed_gradient(embedding, b["dh"], k, tokens, nl.I64, T, 1.0, b["grad"], k, accumulate=True)


def setup(W, T, vocab, width, hidden, kind):
    model = Model(W, vocab, width, hidden)
    theta = model.theta(kind)
    gen = torch.Generator().manual_seed(5)
    tokens, targets = (torch.randint(vocab, (W, T), generator=gen) for _ in range(2))
    targets[:, T - T // 8:] = -1
    p = {name: at for name, (at, _) in model.places.items()}
    plans = (nl.EmbeddingPlan(p["table"], vocab, width, model.stride, W, T),
             nl.LayerNormPlan([(p["w1"], p["b1"], width), (p["w2"], p["b2"], width)], model.stride, W, T),
             nl.LinearPlan([(p["up"], width, hidden, p["up_b"]), (p["down"], hidden, width, p["down_b"]), (p["table"], width, vocab, None, True)],
                           model.stride, W, T),
             nl.LogProbPlan(vocab, W, T))
    new = lambda *shape, dtype=kind: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    buffers = {name: new(W, T, width) for name in ("x", "n1", "h", "n2", "d", "dh")}
    buffers |= {name: new(W, T, hidden) for name in ("a", "z", "da")} | {name: new(W, T, 2, dtype=torch.float32) for name in ("s1", "s2")}
    buffers |= {name: new(W, T, dtype=torch.float32) for name in ("lp", "ln")}
    buffers |= {"logits": new(W, T, vocab), "grad": new(W, model.stride), "by": torch.full((W, T), -1.0 / T, device="cuda")}
    return model, theta, tokens, targets, plans, buffers


# binary32: sums of up to 300 numbers with some roundings each; bf16: what is stored, and operands that are rounded to it
UNITS = {"f32": 2.0 ** -17, "bf16": 2.0 ** -8}


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(3, 40, 61, 24, 72), (2, 300, 257, 64, 200), (1, 7, 33, 17, 31)], ids=str)
def test_inner_step(size, kind):
    """Twice what roundings of the full size at random signs do to the 64-bit result, the worst of three draws."""
    model, theta, tokens, targets, plans, buffers = setup(*size, DTYPES[kind])
    run(model, plans, theta.cuda(), tokens.cuda(), targets.cuda(), DTYPES[kind], buffers)
    lp, grad = exact(model, theta, tokens, targets)
    draws = [exact(model, theta, tokens, targets, UNITS[kind], torch.Generator().manual_seed(s)) for s in range(3)]
    worst = max((d[0] - lp).norm() for d in draws)
    assert (buffers["lp"].cpu().double() - lp).norm() <= 2 * worst + plain.U * lp.norm()
    got, noisy = model.views(buffers["grad"].cpu().double()), [model.views(d[1]) for d in draws]
    for name, want in model.views(grad).items():
        bound = 2 * max((n[name] - want).norm() for n in noisy) + 2 * plain.STORED[DTYPES[kind]] * want.norm()
        assert (got[name] - want).norm() <= bound, name


def test_inner_step_captured():
    """The whole chain as one graph, replayed with other tokens and weights, eager steps between; and two graphs of parts of it that
    share the plans' workspaces, one after the other."""
    model, theta, tokens, targets, plans, buffers = setup(2, 96, 131, 40, 88, torch.bfloat16)
    theta, tokens, targets = theta.cuda(), tokens.cuda(), targets.cuda()
    step = lambda: run(model, plans, theta, tokens, targets, torch.bfloat16, buffers)  # noqa: E731
    step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph in graphs:
        with torch.cuda.graph(graph):
            step()
    for replay in range(4):
        tokens.copy_(torch.randint(131, tokens.shape, device="cuda"))
        theta.mul_(0.99)
        buffers["grad"].zero_()
        step()
        torch.cuda.synchronize()
        want = {name: buffers[name].clone() for name in ("grad", "lp", "dh")}
        for graph in (graphs[replay % 2], graphs[1 - replay % 2]):
            for name in want:
                buffers[name].zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(buffers[name], value) for name, value in want.items())


# ---- offsets beyond 32 bits: the last rows of arrays of more than 2^32 bytes, or numbers ----

def test_log_probs_far_into_memory():
    W, T, vocab = 2, 33000, 65537                            # 4.3e9 logits
    logits = torch.empty((W, T, vocab), dtype=torch.bfloat16, device="cuda")
    logits.normal_(0.0, 2.0)
    tokens = torch.full((W, T), 65536, dtype=torch.int64, device="cuda")
    plan = nl.LogProbPlan(vocab, W, T, max_top=3)
    lp, ln = torch.zeros((W, T), device="cuda"), torch.zeros((W, T), device="cuda")
    ids, tops = torch.zeros((W, T, 3), dtype=torch.int32, device="cuda"), torch.zeros((W, T, 3), device="cuda")
    nl.token_log_probs(plan, logits, nl.BF16, tokens, nl.I64, T, lp, norms=ln, top=3, top_tokens=ids, top_log_probs=tops)
    rows = logits[1, -2:].cpu()
    want = plain.log_probs(rows, tokens[1, -2:].cpu())
    for name, got in (("log_probs", lp), ("norms", ln)):
        value, bound = want[name]
        assert ((got[1, -2:].cpu().double() - value).abs() <= bound).all()
    assert torch.equal(ids[1, -2:].cpu().long(), plain.top_tokens(rows, 3))
    nl.token_log_probs_gradient(plan, logits, nl.BF16, tokens, nl.I64, T, ln, torch.ones((W, T), device="cuda"), logits, nl.BF16)
    value, bound = plain.log_probs_gradient(rows, tokens[1, -2:].cpu(), ln[1, -2:].cpu(), torch.ones(2), None, None, torch.bfloat16)
    assert ((logits[1, -2:].cpu().double() - value).abs() <= bound).all()


def test_norms_far_into_memory():
    W, T, width = 2, 1100000, 2000                           # 4.4e9 numbers
    x = torch.empty((W, T, width), dtype=torch.bfloat16, device="cuda").normal_()
    theta = torch.ones((W, 2048), device="cuda")
    plan = nl.LayerNormPlan([(0, None, width)], 2048, W, T)
    out, stats = torch.zeros_like(x), torch.zeros((W, T, 2), device="cuda")
    nl.layer_norm(plan, 0, x, nl.BF16, theta, nl.F32, T, EPS, out, nl.BF16, stats=stats)
    last, weight = x[1:, -3:].cpu(), theta[1:, :width].cpu()
    (value, bound), _ = plain.layer_norm(last, weight, None, EPS, torch.bfloat16)
    assert ((out[1:, -3:].cpu().double() - value).abs() <= bound).all()
    dout = last.cuda()
    given = stats[1:, -3:].cpu()
    nl.layer_norm_gradient(plan, 0, out, nl.BF16, x, nl.BF16, theta, nl.F32, stats, T, x.new_empty(x.shape), nl.BF16, None, nl.F32)
    dx = torch.zeros_like(x)
    out[1:, -3:] = dout
    nl.layer_norm_gradient(plan, 0, out, nl.BF16, x, nl.BF16, theta, nl.F32, stats, T, dx, nl.BF16, None, nl.F32)
    (value, bound), *_ = plain.layer_norm_gradient(last, last, weight, given, None, torch.bfloat16)
    assert ((dx[1:, -3:].cpu().double() - value).abs() <= bound).all()


@pytest.mark.parametrize("inputs", [1024, 1001])
def test_matrices_far_into_memory(inputs):
    W, T, outputs = 5, 900000, 24                            # 4.6e9 numbers
    x = torch.empty((W, T, inputs), dtype=torch.bfloat16, device="cuda").normal_()
    stride = -(-(inputs * outputs) // 64) * 64
    theta = torch.empty((W, stride), dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.1)
    plan = nl.LinearPlan([(0, inputs, outputs)], stride, W, T)
    out = torch.zeros((W, T, outputs), dtype=torch.bfloat16, device="cuda")
    nl.linear(plan, 0, x, nl.BF16, theta, nl.BF16, T, out, nl.BF16)
    last, matrix = x[4:, -5:].cpu(), theta[4:, :inputs * outputs].cpu().view(1, inputs, outputs)
    (value, bound), _ = plain.linear(last, matrix, None, "none", None, torch.bfloat16)
    assert ((out[4:, -5:].cpu().double() - value).abs() <= bound).all()
    nl.linear_gradient(plan, 0, out, nl.BF16, None, nl.BF16, theta, nl.BF16, T, x, nl.BF16, None, nl.BF16)
    dlast = out[4:, -5:].cpu()
    value, bound = plain.product(dlast, matrix.mT, torch.bfloat16)
    assert ((x[4:, -5:].cpu().double() - value).abs() <= bound + plain.STORED[torch.bfloat16] * value.abs()).all()


def test_fewer_tokens_than_the_plans_take():
    W, width, outputs = 2, 72, 56
    stride = 64 * 65
    theta = torch.empty((W, stride), device="cuda").normal_(0.0, 0.2)
    plan, norms = nl.LinearPlan([(0, width, outputs), (0, width, outputs)], stride, W, 3000), nl.LayerNormPlan([(0, None, width)], stride, W, 3000)
    for T in (2999, 1, 257):
        x = torch.randn((W, T, width), generator=torch.Generator().manual_seed(T))
        out, normed = torch.zeros((W, T, outputs), device="cuda"), torch.zeros((W, T, width), device="cuda")
        nl.linear(plan, 1, x.cuda(), nl.F32, theta, nl.F32, T, out, nl.F32)
        nl.layer_norm(norms, 0, x.cuda(), nl.F32, theta, nl.F32, T, EPS, normed, nl.F32)
        value, bound = plain.product(x, theta[:, :width * outputs].cpu().view(W, width, outputs), torch.float32)
        assert ((out.cpu().double() - value).abs() <= bound + plain.U * value.abs()).all()
        (value, bound), _ = plain.layer_norm(x, theta[:, :width].cpu(), None, EPS, torch.float32)
        assert ((normed.cpu().double() - value).abs() <= bound).all()
