"""The inner step's operators over a replica arena, as cases that can be timed and checked.

Between two outer steps every worker trains its own row of the arena. Two parts of that inner step touch the
arena itself: the update of the weight matrices, whose direction is the momentum orthogonalised by
Newton-Schulz products, and the embedding table, which the forward pass looks tokens up in and the backward
pass adds their gradients to. A case is one call of one of the four entry points:

  orthogonalize  out = NS(x) for matrices of every worker's row: X_0 = x / (|x|_F + eps), then `steps` times
                 X <- a X + (b A + c A^2) X with A = X X^T (X stands on its short side)
  muon           momentum <- mu momentum + grad;  u = grad + mu momentum (Nesterov) or momentum;
                 theta <- (1 - lr wd) theta - lr scale NS(u)
  lookup         out[w, t] = scale table_w[token[w, t]], a row of zeros where the token is no row of the table
  gradient       grad_w[v] (+)= scale sum of dout[w, t] over the t with token[w, t] = v

Widths, vocabulary and replicas are those of `workloads/` (GPT-style blocks of 768/12/3072, 2048/24/8192 and
4096/32/16384, a vocabulary of 50257, sequences of 1024) or generic.
"""
import math

import numpy as np
import torch

own = False                     # whether run() calls the framework's operators or computes their plain forms

ALIGN_ELEMS = 64                # worker rows start at multiples of this many elements
COEFFICIENTS = ((3.4445, -4.7750, 2.0315),) * 5
EPS = 1e-7
LR, MU, WEIGHT_DECAY = 0.02, 0.95, 0.1
INIT_STD = 0.02                 # weights
DRIFT_STD = 5e-4                # how far the replicas have drifted apart
GRAD_STD = 1e-3
RANK = 32                       # a gradient is a few strong directions over a floor of noise
MOST_FLOPS = 4.2e13             # products of the largest listed case, every one counted whole
MOST_BYTES = 6e9
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _matrices(name, op, layout, W, x, out, **sizes):
    return dict(name=name, op=op, layout=layout, W=W, x=x, out=out, **sizes)


def _tokens(name, op, W, T, vocab, width, x, out, ids="i64", **more):
    return dict(name=name, op=op, W=W, T=T, vocab=vocab, width=width, x=x, out=out, ids=ids, **more)


def listed():
    return [
        # One attention projection of the 125M model by itself: a chain of short dependent products.
        _matrices("ortho_768_w1_bf16", "orthogonalize", "one", 1, "bf16", "bf16", rows=768, cols=768),
        # Odd shapes of every aspect, float throughout: adapters, a vector, a matrix as tall as it is thin.
        _matrices("ortho_ragged_w4_f32", "orthogonalize", "ragged", 4, "f32", "f32", count=12, least=1, most=1031),
        # Every head's slice of the 125M model's query projections by itself, eight replicas.
        _matrices("ortho_heads_w8_bf16", "orthogonalize", "heads", 8, "f32", "bf16", d=768, heads=12, blocks=12),
        # A toy model's matrices: the call itself is most of the time.
        _matrices("muon_toy_w4_f32", "muon", "gpt", 4, "f32", "f32", d=64, f=256, blocks=1, nesterov=True),
        # All matrices of the 125M model, two replicas with float weights.
        _matrices("muon_gpt125m_w2_f32", "muon", "gpt", 2, "f32", "f32", d=768, f=3072, blocks=12, nesterov=True),
        # One block of the 1.3B model on eight replicas with bf16 weights and gradients.
        _matrices("muon_block2048_w8_bf16", "muon", "gpt", 8, "bf16", "bf16", d=2048, f=8192, blocks=1, nesterov=True),
        # One block of the 6.8B model on two replicas: the largest.
        _matrices("muon_block4096_w2_bf16", "muon", "gpt", 2, "bf16", "bf16", d=4096, f=16384, blocks=1, nesterov=False),
        # A toy model's tokens, odd width and vocabulary.
        _tokens("lookup_toy_w4_f32", "lookup", 4, 61, 257, 129, "f32", "f32", ids="i32"),
        # The 125M model's tokens of one micro-batch of eight sequences on every replica, activations in bf16.
        _tokens("lookup_gpt125m_w8_bf16", "lookup", 8, 8192, 50257, 768, "f32", "bf16"),
        # The toy model's backward pass.
        _tokens("gradient_toy_w4_f32", "gradient", 4, 61, 257, 129, "f32", "f32", ids="i32", accumulate=False),
        # The 125M model's tied table: the output head has left its gradient there, the lookup adds its own.
        _tokens("gradient_gpt125m_w8_tied", "gradient", 8, 8192, 50257, 768, "bf16", "f32", accumulate=True),
        # The 6.8B model's first stage, untied: thirty-two sequences, the whole table's gradient written.
        _tokens("gradient_6p8b_w2_bf16", "gradient", 2, 32768, 50257, 4096, "bf16", "bf16", accumulate=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["orthogonalize", "muon", "muon", "lookup", "gradient"])
    W = rng.choice([1, 2, 3, 4, 5, 8])
    if op in ("lookup", "gradient"):
        vocab, width = _log_int(rng, 2, 60000), _log_int(rng, 1, 4096)
        T = _log_int(rng, 1, 40000)
        x, out = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
        more = {} if op == "lookup" else dict(accumulate=rng.random() < 0.5)
        most = int(MOST_BYTES / 16 / (max(vocab, T) * width))
        return dict(op=op, W=max(1, min(W, most)), T=T, vocab=vocab, width=width, x=x, out=out,
                    ids=rng.choice(["i32", "i64"]), **more)
    kind = rng.choice(["f32", "bf16"])
    case = dict(op=op, layout=rng.choice(["one", "gpt", "heads", "ragged"]), W=W,
                x=rng.choice(["f32", "bf16"]) if op == "orthogonalize" else kind, out=kind)
    if op == "muon":
        case["nesterov"] = rng.random() < 0.5
    if case["layout"] == "one":
        case |= dict(rows=_log_int(rng, 1, 4096), cols=_log_int(rng, 1, 16384))
        if rng.random() < 0.5:
            case |= dict(rows=case["cols"], cols=case["rows"])
    elif case["layout"] == "gpt":
        d = _log_int(rng, 16, 2100)
        case |= dict(d=d, f=4 * d, blocks=rng.choice([1, 1, 2, 3]))
    elif case["layout"] == "heads":
        heads = rng.choice([2, 4, 6, 8, 12])
        case |= dict(d=heads * _log_int(rng, 8, 128), heads=heads, blocks=_log_int(rng, 1, 12))
    else:
        least = _log_int(rng, 1, 64)
        case |= dict(count=_log_int(rng, 2, 24), least=least, most=least + _log_int(rng, 32, 1500))
    while case["W"] > 1 and _whole_flops(case) > MOST_FLOPS:
        case["W"] -= 1
    return case


# ---------------------------------------------------------------------------
# Layouts
# ---------------------------------------------------------------------------

def _layout(case):
    """(matrices, worker_stride): every matrix of a worker's row as (offset, rows, cols, row_stride, scale)."""
    kind, found, at = case["layout"], [], 0

    def add(offset, rows, cols, row_stride):
        # a tall matrix takes longer steps, so that its outputs change by as much as a square one's
        found.append((offset, rows, cols, row_stride, math.sqrt(max(1.0, rows / cols))))

    if kind == "one":
        add(0, case["rows"], case["cols"], case["cols"])
        at = case["rows"] * case["cols"]
    elif kind == "gpt":
        d, f = case["d"], case["f"]
        for _ in range(case["blocks"]):
            at += 2 * d                                     # first norm
            for part in range(3):                           # queries, keys and values, side by side in one tensor
                add(at + part * d, d, d, 3 * d)
            at += 3 * d * d + 3 * d
            add(at, d, d, d)                                # output projection
            at += d * d + d + 2 * d
            add(at, d, f, f)
            at += d * f + f
            add(at, f, d, d)
            at += f * d + d
    elif kind == "heads":
        d, heads = case["d"], case["heads"]
        for _ in range(case["blocks"]):
            for h in range(heads):                          # one head's columns of a [d, d] projection
                add(at + h * (d // heads), d, d // heads, d)
            at += d * d
    else:                                                   # odd sizes, one to seven elements of nobody's between them
        rng = np.random.default_rng([7, case["count"], case["least"], case["most"]])
        lo, hi = math.log(case["least"]), math.log(case["most"])
        for _ in range(case["count"]):
            rows, cols = (int(round(math.exp(v))) for v in rng.uniform(lo, hi, size=2))
            add(at, rows, cols, cols)
            at += rows * cols + int(rng.integers(1, 8))
    return found, -(-at // ALIGN_ELEMS) * ALIGN_ELEMS


def _whole_flops(case):
    """Multiplications and additions of all products, each counted whole."""
    total = 0
    for _, rows, cols, _, _ in _layout(case)[0]:
        m, n = min(rows, cols), max(rows, cols)
        total += len(COEFFICIENTS) * (4 * m * m * n + 2 * m * m * m)
    return total * case["W"]


def _view(array, matrix):
    """One matrix of every worker, [W, rows, cols], over the arena's memory."""
    offset, rows, cols, row_stride, _ = matrix
    return array.as_strided((array.shape[0], rows, cols), (array.stride(0), row_stride, 1), array.storage_offset() + offset)


def _table(array, case):
    """The embedding table of every worker, [W, vocab, width]; it begins every worker's row."""
    return array[:, :case["vocab"] * case["width"]].unflatten(1, (case["vocab"], case["width"]))


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _directions(array, matrices, gen):
    """Adds to each matrix of noise a few directions, ever weaker, that hold about four fifths of it."""
    W = array.shape[0]
    for matrix in matrices:
        _, rows, cols, _, _ = matrix
        rank = min(RANK, rows, cols)
        weight = 1.0 / torch.arange(1, rank + 1, device="cuda", dtype=torch.float32)
        weight *= 2.0 * GRAD_STD / weight.square().sum().sqrt()
        left = torch.empty((W, rows, rank), device="cuda").normal_(0.0, 1.0, generator=gen) * weight
        right = torch.empty((W, rank, cols), device="cuda").normal_(0.0, 1.0, generator=gen)
        view = _view(array, matrix)
        view += left @ right


def _matrix_arrays(case, seed):
    matrices, stride = _layout(case)
    W, gen = case["W"], _generator(seed)

    def moving():
        array = torch.empty((W, stride), device="cuda").normal_(0.0, GRAD_STD, generator=gen)
        _directions(array, matrices, gen)
        return array

    if case["op"] == "orthogonalize":
        return matrices, stride, {"x": moving().to(TYPES[case["x"]])}
    base = torch.empty(stride, device="cuda").normal_(0.0, INIT_STD, generator=gen)
    theta = torch.empty((W, stride), device="cuda").normal_(0.0, DRIFT_STD, generator=gen).add_(base)
    return matrices, stride, {"theta": theta.to(TYPES[case["out"]]), "grad": moving().to(TYPES[case["x"]]),
                              "momentum": moving().mul_(3.0)}


def _weights(vocab):
    """Shares of the tokens in a text: a few carry most of it, most are rare."""
    p = 1.0 / (np.arange(vocab, dtype=np.float64) + 2.7)
    return p / p.sum()


def _padding(T):
    return T // 32              # positions at the end of a worker's tokens that hold none (-1)


def _token_arrays(case, seed):
    W, T, vocab, width, gen = case["W"], case["T"], case["vocab"], case["width"], _generator(seed)
    stride = -(-vocab * width // ALIGN_ELEMS) * ALIGN_ELEMS
    edges = torch.from_numpy(np.cumsum(_weights(vocab))).to("cuda")
    spot = torch.rand((W, T), device="cuda", dtype=torch.float64, generator=gen)
    tokens = torch.searchsorted(edges, spot).clamp_(max=vocab - 1)
    if _padding(T):
        tokens[:, T - _padding(T):] = -1
    arrays = {"tokens": tokens.to(torch.int32 if case["ids"] == "i32" else torch.int64)}
    if case["op"] == "lookup":
        table = torch.empty((W, stride), device="cuda").normal_(0.0, INIT_STD, generator=gen)
        return stride, arrays | {"table": table.to(TYPES[case["x"]])}
    dout = torch.empty((W, T, width), device="cuda").normal_(0.0, GRAD_STD, generator=gen)
    grad = torch.empty((W, stride), device="cuda").normal_(0.0, GRAD_STD, generator=gen)
    return stride, arrays | {"dout": dout.to(TYPES[case["x"]]), "grad": grad.to(TYPES[case["out"]])}


def _scale(case):
    return math.sqrt(case["width"])         # the lookup's rows come out near unit size


def prepare(case, seed):
    state = dict(case=case)
    if case["op"] in ("lookup", "gradient"):
        stride, arrays = _token_arrays(case, seed)
        if case["op"] == "lookup":
            arrays["out"] = torch.zeros((case["W"], case["T"], case["width"]), device="cuda", dtype=TYPES[case["out"]])
        if own:
            import paper_2506_10911_amd as nl
            state["plan"] = nl.EmbeddingPlan(0, case["vocab"], case["width"], stride, case["W"], case["T"])
    else:
        matrices, stride, arrays = _matrix_arrays(case, seed)
        if case["op"] == "orthogonalize":
            arrays["out"] = torch.zeros((case["W"], stride), device="cuda", dtype=TYPES[case["out"]])
        state["matrices"] = matrices
        if own:
            import paper_2506_10911_amd as nl
            state["plan"] = nl.MuonPlan(matrices, stride, case["W"])
    state["arrays"] = arrays
    return state


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    case, arrays = state["case"], state["arrays"]
    one_pass = {"orthogonalize": _orthogonalize, "muon": _muon, "lookup": _lookup, "gradient": _gradient}[case["op"]]
    return one_pass(case, arrays, state)


def _newton_schulz(u):
    """[N, rows, cols] float."""
    tall = u.shape[1] > u.shape[2]
    x = u.mT if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for a, b, c in COEFFICIENTS:
        g = x @ x.mT
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.mT if tall else x


def _by_shape(matrices):
    """Matrices of one shape go through the products together."""
    shapes = {}
    for matrix in matrices:
        shapes.setdefault(matrix[1:3], []).append(matrix)
    return shapes.values()


def _orthogonalize(case, arrays, state):
    x, out = arrays["x"], arrays["out"]
    if own:
        import paper_2506_10911_amd as nl
        nl.orthogonalize(state["plan"], x, nl.BF16 if case["x"] == "bf16" else nl.F32,
                         out, nl.BF16 if case["out"] == "bf16" else nl.F32, coefficients=COEFFICIENTS, eps=EPS)
        return out
    for alike in _by_shape(state["matrices"]):
        got = _newton_schulz(torch.cat([_view(x, m) for m in alike]).float())
        for m, part in zip(alike, got.split(x.shape[0])):
            _view(out, m).copy_(part)
    return out


def _muon(case, arrays, state):
    theta, grad, momentum = arrays["theta"], arrays["grad"], arrays["momentum"]
    if own:
        import paper_2506_10911_amd as nl
        nl.muon_step(state["plan"], theta, nl.BF16 if case["out"] == "bf16" else nl.F32,
                     grad, nl.BF16 if case["x"] == "bf16" else nl.F32, momentum,
                     (LR, MU, WEIGHT_DECAY), nesterov=case["nesterov"], coefficients=COEFFICIENTS, eps=EPS)
        return {"theta": theta, "momentum": momentum}
    for alike in _by_shape(state["matrices"]):
        g = torch.cat([_view(grad, m) for m in alike]).float()
        moved = torch.cat([_view(momentum, m) for m in alike]).mul_(MU).add_(g)
        got = _newton_schulz(g.add_(moved, alpha=MU) if case["nesterov"] else moved)
        for m, new, part in zip(alike, moved.split(theta.shape[0]), got.split(theta.shape[0])):
            _view(momentum, m).copy_(new)
            view = _view(theta, m)
            view.copy_(view.float() * (1.0 - LR * WEIGHT_DECAY) - (LR * m[4]) * part)
    return {"theta": theta, "momentum": momentum}


def _lookup(case, arrays, state):
    tokens, table, out = arrays["tokens"], arrays["table"], arrays["out"]
    if own:
        import paper_2506_10911_amd as nl
        nl.embed_lookup(state["plan"], table, nl.BF16 if case["x"] == "bf16" else nl.F32,
                        tokens, nl.I32 if case["ids"] == "i32" else nl.I64, case["T"], _scale(case),
                        out, nl.BF16 if case["out"] == "bf16" else nl.F32)
        return out
    worker = torch.arange(case["W"], device="cuda")[:, None]
    there = ((tokens >= 0) & (tokens < case["vocab"]))
    rows = _table(table, case)[worker, torch.where(there, tokens, 0).long()]
    return out.copy_(torch.where(there[:, :, None], rows.float() * _scale(case), 0.0))


def _gradient(case, arrays, state):
    tokens, dout, grad = arrays["tokens"], arrays["dout"], arrays["grad"]
    if own:
        import paper_2506_10911_amd as nl
        nl.embed_gradient(state["plan"], dout, nl.BF16 if case["x"] == "bf16" else nl.F32,
                          tokens, nl.I32 if case["ids"] == "i32" else nl.I64, case["T"], _scale(case),
                          grad, nl.BF16 if case["out"] == "bf16" else nl.F32, accumulate=case["accumulate"])
        return grad
    vocab, width = case["vocab"], case["width"]
    there = ((tokens >= 0) & (tokens < vocab))
    # one row more takes what belongs to no token
    row = torch.where(there, tokens.long() + vocab * torch.arange(case["W"], device="cuda")[:, None], case["W"] * vocab)
    sums = torch.zeros((case["W"] * vocab + 1, width), device="cuda")
    sums.index_add_(0, row.reshape(-1), dout.reshape(-1, width).float())
    sums = sums[:-1].view(case["W"], vocab, width).mul_(_scale(case))
    view = _table(grad, case)
    view.copy_(view.float().add_(sums) if case["accumulate"] else sums)
    return grad


# ---------------------------------------------------------------------------
# What a pass cannot do without, and what its outputs are
# ---------------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
    W = case["W"]
    if case["op"] in ("lookup", "gradient"):
        T, width, vocab = case["T"], case["width"], case["vocab"]
        real = T - _padding(T)
        distinct = float((1.0 - (1.0 - _weights(vocab)) ** real).sum())     # rows that come up, on average
        ids = T * size[case["ids"]]
        if case["op"] == "lookup":
            moved = distinct * width * size[case["x"]] + T * width * size[case["out"]]
        else:
            rows = 2 * distinct if case["accumulate"] else vocab
            moved = real * width * size[case["x"]] + rows * width * size[case["out"]]
        return {"bytes": W * (moved + ids), "flops": W * real * width}
    numbers, flops = 0, 0
    for _, rows, cols, _, _ in _layout(case)[0]:
        m, n = min(rows, cols), max(rows, cols)
        numbers += rows * cols
        # A and A^2 are symmetric: half of each is enough
        flops += len(COEFFICIENTS) * (m * m * n + m * m * m + 2 * m * m * n)
    a_number = size[case["x"]] + (size[case["out"]] if case["op"] == "orthogonalize" else 2 * size[case["out"]] + 8)
    return {"bytes": W * numbers * a_number, "flops": W * flops}


def exact(case, seed):
    if case["op"] == "lookup":
        return _exact_lookup(case, seed)
    if case["op"] == "gradient":
        return _exact_gradient(case, seed)
    matrices, stride, arrays = _matrix_arrays(case, seed)
    if case["op"] == "orthogonalize":
        out = torch.zeros((case["W"], stride), device="cuda", dtype=torch.float64)
        for w in range(case["W"]):
            for m in matrices:
                _view(out[w:w + 1], m)[0] = _exact_newton_schulz(_view(arrays["x"][w:w + 1], m)[0].double())
        return out
    theta, momentum = arrays["theta"].double(), arrays["momentum"].double()
    for w in range(case["W"]):
        for m in matrices:
            here = [_view(array[w:w + 1], m)[0] for array in (theta, arrays["grad"], momentum)]
            weight, g, mom = here[0], here[1].double(), here[2]
            mom.copy_(mom * MU + g)
            step = _exact_newton_schulz(mom * MU + g if case["nesterov"] else mom.clone())
            weight.sub_(LR * (WEIGHT_DECAY * weight + m[4] * step))
    return {"theta": theta, "momentum": momentum}


def _exact_newton_schulz(u):
    """The same odd polynomials of one matrix, by Horner's rule: ((c A + b) A + a) X on the short side."""
    if u.shape[0] > u.shape[1]:
        return _exact_newton_schulz(u.T.contiguous()).T
    x = u / (torch.linalg.matrix_norm(u) + EPS)
    unit = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for a, b, c in COEFFICIENTS:
        gram = x @ x.T
        x = (gram @ (c * gram + b * unit) + a * unit) @ x
    return x


def _exact_lookup(case, seed):
    stride, arrays = _token_arrays(case, seed)
    out = torch.zeros((case["W"], case["T"], case["width"]), device="cuda", dtype=torch.float64)
    for w in range(case["W"]):
        tokens = arrays["tokens"][w].long()
        real = tokens >= 0
        rows = arrays["table"][w][:case["vocab"] * case["width"]].view(case["vocab"], case["width"])
        out[w, real] = rows[tokens[real]].double() * _scale(case)
    return out


def _exact_gradient(case, seed):
    stride, arrays = _token_arrays(case, seed)
    vocab, width = case["vocab"], case["width"]
    out = arrays["grad"].double()
    for w in range(case["W"]):
        tokens = arrays["tokens"][w].long()
        real = tokens >= 0
        rows = out[w][:vocab * width].view(vocab, width)
        if not case["accumulate"]:
            rows.zero_()
        rows.index_add_(0, tokens[real], arrays["dout"][w, real].double() * _scale(case))
    return out
