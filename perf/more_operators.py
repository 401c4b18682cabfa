"""The rest of the inner step over a replica arena, as cases that can be timed and checked.

Between the embedding table's lookup and its gradient a replica's inner step runs through layer norms, matrices and the
loss. Their weights lie in the W stacked rows of the arena and their gradients go there. A case is one call of one of
six entry points:

  norm           out = (x - mean) rstd weight + bias along the width, with mean and rstd = 1 / sqrt(variance + eps)
  norm_gradient  dx = add + rstd (g - mean(g) - xh mean(g xh)) with xh = (x - mean) rstd, g = dout weight;
                 the weight's gradient (+)= sum over tokens of dout xh, the bias's (+)= sum of dout
  linear         out = act(x M + bias) + residual, and what stands before the activation
  linear_gradient  dz = dout act'(before); dx = add + dz M^T; the matrix's gradient (+)= x^T dz, the bias's (+)= sum of dz
  log_probs      log_probs = logits[token] - n with n = log sum exp(logits); entropy; the `top` largest logits' tokens and
                 log probabilities, the lower token first where logits are equal; 0 where the token is none of the vocabulary
  log_probs_gradient  dlogits = dlog_probs ([v = token] - p) - dentropy p (log p + entropy)

Widths, vocabulary and replicas are those of `workloads/` (GPT-style blocks of width 768, 2048 with 8192 and 4096 with
16384, a vocabulary of 50257, sequences of 1024) and of examples/inner_outer.py, or generic.
"""
import math

import numpy as np
import torch

own = False                     # whether run() calls the framework's operators or computes their plain forms

ALIGN_ELEMS = 64                # worker rows start at multiples of this many elements
EPS = 1e-5
INIT_STD = 0.02                 # weights of matrices
GRAD_STD = 1e-3
LOGIT_STD = 2.5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MOST_FLOPS = 2.1e12             # of a drawn case: less than the largest listed one's
MOST_BYTES = 1.5e9              # that a drawn case moves outside of products


def _norm(name, op, W, T, width, x, theta, out, **more):
    return dict(name=name, op=op, W=W, T=T, width=width, x=x, theta=theta, out=out, gap=0, bias=True, **more)


def _linear(name, op, W, T, inputs, outputs, x, theta, out, act, **more):
    return dict(name=name, op=op, W=W, T=T, inputs=inputs, outputs=outputs, x=x, theta=theta, out=out, act=act, gap=0, bias=True,
                transposed=False, **more)


def _logits(name, op, W, T, vocab, x, ids, **more):
    return dict(name=name, op=op, W=W, T=T, vocab=vocab, stride=-(-vocab // ALIGN_ELEMS) * ALIGN_ELEMS, x=x, ids=ids, **more)


def listed():
    return [
        # A toy model's norm, odd width, float throughout: the call itself is most of the time.
        _norm("norm_toy_w4_f32", "norm", 4, 61, 129, "f32", "f32", "f32"),
        # The 125M model's norm of one micro-batch of eight sequences on every replica, float weights, activations in bf16.
        _norm("norm_gpt125m_w8_bf16", "norm", 8, 8192, 768, "bf16", "f32", "bf16"),
        # Its backward pass, which takes the residual branch's gradient in and adds to what other micro-batches left.
        _norm("norm_gradient_gpt125m_w8", "norm_gradient", 8, 8192, 768, "bf16", "f32", "bf16", add=True, accumulate=True),
        # The 6.8B model's on two replicas, bf16 throughout.
        _norm("norm_gradient_6p8b_w2_bf16", "norm_gradient", 2, 8192, 4096, "bf16", "bf16", "bf16", add=False, accumulate=False),
        # The example's first matrix with its activation.
        _linear("linear_toy_w4_f32", "linear", 4, 256, 96, 192, "f32", "f32", "f32", "relu", before=True, residual=False),
        # A micro-batch through the 1.3B model's first matrix of a feed-forward block, eight replicas.
        _linear("linear_2048_w8_bf16", "linear", 8, 4096, 2048, 8192, "bf16", "bf16", "bf16", "gelu", before=True, residual=False),
        # One token through the 6.8B model's second matrix on two replicas: bound by reading it.
        _linear("linear_token_w2_bf16", "linear", 2, 1, 16384, 4096, "bf16", "bf16", "bf16", "none", before=False, residual=True),
        # Backward through the 125M model's queries, keys and values: float weights and gradients, activations in bf16.
        _linear("linear_gradient_768_w8", "linear_gradient", 8, 2048, 768, 2304, "bf16", "f32", "bf16", "none", grad="f32", add=False,
                accumulate=True),
        # Backward through the 6.8B model's first matrix of a feed-forward block on two replicas: the largest.
        _linear("linear_gradient_4096_w2_bf16", "linear_gradient", 2, 4096, 4096, 16384, "bf16", "bf16", "bf16", "gelu", grad="bf16",
                add=False, accumulate=False),
        # One position of every replica, with the likeliest alternatives: what an evaluation asks for token by token.
        _logits("log_probs_token_w4_f32", "log_probs", 4, 1, 50257, "f32", "i64", top=8, entropy=True),
        # A sequence of the 125M model on every replica, the rows padded to a multiple of 64: the loss.
        _logits("log_probs_gpt125m_w8_bf16", "log_probs", 8, 1024, 50257, "bf16", "i64", top=0, entropy=False),
        # And its gradient.
        _logits("log_probs_gradient_gpt125m_w8", "log_probs_gradient", 8, 1024, 50257, "bf16", "i64", out="bf16", entropy=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_gradient", "linear", "linear", "linear_gradient", "linear_gradient", "log_probs",
                     "log_probs_gradient"])
    W, types = rng.choice([1, 2, 3, 4, 5, 8]), ["f32", "bf16"]
    if op.startswith("norm"):
        width, T = _log_int(rng, 8, 12000), _log_int(rng, 1, 20000)
        W = max(1, min(W, int(MOST_BYTES / 24 / (T * width))))
        case = dict(op=op, W=W, T=T, width=width, x=rng.choice(types), theta=rng.choice(types), out=rng.choice(types),
                    gap=rng.choice([0, 0, 3]), bias=rng.random() < 0.8)
        if op == "norm_gradient":
            case |= dict(add=rng.random() < 0.5, accumulate=rng.random() < 0.5)
    elif op.startswith("linear"):
        inputs, outputs, T = _log_int(rng, 1, 8192), _log_int(rng, 1, 8192), _log_int(rng, 1, 8192)
        if rng.random() < 0.5:                              # widths of real layers are multiples of something
            inputs, outputs = (max(32, v // 32 * 32) for v in (inputs, outputs))
        kind = rng.choice([("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"),
                           ("f32", "bf16", "bf16")])
        case = dict(op=op, W=W, T=T, inputs=inputs, outputs=outputs, x=kind[0], theta=kind[1], out=kind[2],
                    act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), gap=rng.choice([0, 0, 0, 3]),
                    bias=rng.random() < 0.8, transposed=rng.random() < 0.3)
        if op == "linear":
            case |= dict(before=rng.random() < 0.5, residual=rng.random() < 0.5)
        else:
            case |= dict(grad=kind[1], add=rng.random() < 0.3, accumulate=rng.random() < 0.5)
        while case["W"] > 1 and work(case)["flops"] > MOST_FLOPS:
            case["W"] -= 1
    else:
        vocab, T = _log_int(rng, 2, 130000), _log_int(rng, 1, 4000)
        W = max(1, min(W, int(MOST_BYTES / 12 / (T * vocab))))
        case = dict(op=op, W=W, T=T, vocab=vocab, stride=vocab + rng.choice([0, 0, 1, -vocab % 64]), x=rng.choice(types),
                    ids=rng.choice(["i32", "i64"]), entropy=rng.random() < 0.5)
        if op == "log_probs":
            case["top"] = rng.choice([0, 0, 1, 5, 20])
        else:
            case["out"] = rng.choice(types)
    return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, shape, std, kind):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen).to(TYPES[kind])


def _padded(elements):
    return -(-elements // ALIGN_ELEMS) * ALIGN_ELEMS


def _norm_places(case):
    """(weight's offset, bias's offset or -1, worker_stride)"""
    at, width = case["gap"], case["width"]
    return at, at + width if case["bias"] else -1, _padded(at + 2 * width)


def _linear_places(case):
    """(matrix's offset, bias's offset or -1, worker_stride)"""
    at, size = case["gap"], case["inputs"] * case["outputs"]
    return at, at + size if case["bias"] else -1, _padded(at + size + case["outputs"])


def _vector(array, offset, width):
    """A vector of every worker, [W, 1, width], over the arena's memory."""
    return array[:, None, offset:offset + width]


def _matrix(array, case):
    """The matrix of every worker, [W, inputs, outputs], over the arena's memory."""
    part = array[:, case["gap"]:case["gap"] + case["inputs"] * case["outputs"]]
    if case["transposed"]:
        return part.unflatten(1, (case["outputs"], case["inputs"])).mT
    return part.unflatten(1, (case["inputs"], case["outputs"]))


def _norm_arrays(case, seed):
    gen, shape = _generator(seed), (case["W"], case["T"], case["width"])
    weight, bias, stride = _norm_places(case)
    theta = torch.empty((case["W"], stride), device="cuda").normal_(0.0, 0.1, generator=gen)
    theta[:, weight:weight + case["width"]] += 1.0
    x = torch.empty(shape, device="cuda").normal_(0.0, 1.5, generator=gen)
    x += torch.empty((case["W"], case["T"], 1), device="cuda").normal_(0.0, 0.3, generator=gen)
    arrays = dict(theta=theta.to(TYPES[case["theta"]]), x=x.to(TYPES[case["x"]]))
    if case["op"] == "norm_gradient":
        # what the forward pass left
        wide = arrays["x"].double()
        mean = wide.mean(-1)
        rstd = ((wide - mean[..., None]).square().mean(-1) + EPS).rsqrt()
        arrays["stats"] = torch.stack([mean, rstd], -1).float()
        arrays["dout"] = _normal(gen, shape, GRAD_STD, case["x"])
        arrays["add"] = _normal(gen, shape, GRAD_STD, case["out"]) if case["add"] else None
        arrays["grad"] = _normal(gen, (case["W"], stride), GRAD_STD, case["theta"])
    return arrays


def _linear_arrays(case, seed):
    gen, W, T = _generator(seed), case["W"], case["T"]
    stride = _linear_places(case)[2]
    arrays = dict(theta=_normal(gen, (W, stride), INIT_STD, case["theta"]),
                  x=_normal(gen, (W, T, case["inputs"]), 1.0, case["x"]))
    if case["op"] == "linear":
        arrays["residual"] = _normal(gen, (W, T, case["outputs"]), 1.0, case["out"]) if case["residual"] else None
    else:
        arrays["dout"] = _normal(gen, (W, T, case["outputs"]), GRAD_STD, case["x"])
        arrays["before"] = _normal(gen, (W, T, case["outputs"]), 1.0, case["x"]) if case["act"] != "none" else None
        arrays["add"] = _normal(gen, (W, T, case["inputs"]), GRAD_STD, case["out"]) if case["add"] else None
        arrays["grad"] = _normal(gen, (W, stride), GRAD_STD, case["grad"])
    return arrays


def _padding(T):
    return T // 32              # positions at the end of a worker's tokens that hold none (-1)


def _logit_arrays(case, seed):
    gen, W, T, vocab = _generator(seed), case["W"], case["T"], case["vocab"]
    edges = torch.from_numpy(np.cumsum(1.0 / (np.arange(vocab) + 2.7))).to("cuda")
    spot = torch.rand((W, T), device="cuda", dtype=torch.float64, generator=gen) * edges[-1]
    tokens = torch.searchsorted(edges, spot).clamp_(max=vocab - 1)
    logits = torch.empty((W, T, case["stride"]), device="cuda").normal_(0.0, LOGIT_STD, generator=gen)
    # a trained model's logits are larger at the tokens that come
    logits.scatter_add_(2, tokens[..., None], torch.full((W, T, 1), 6.0, device="cuda"))
    if _padding(T):
        tokens[:, T - _padding(T):] = -1
    arrays = dict(logits=logits.to(TYPES[case["x"]]), tokens=tokens.to(torch.int32 if case["ids"] == "i32" else torch.int64))
    if case["op"] == "log_probs_gradient":
        arrays["dlog_probs"] = torch.full((W, T), -1.0 / T, device="cuda")
        arrays["dentropy"] = _normal(gen, (W, T), 0.1 / T, "f32") if case["entropy"] else None
        # what the forward pass left
        wide = arrays["logits"][..., :vocab].float()
        largest = wide.amax(-1, keepdim=True)
        shares = wide.sub_(largest).exp_()
        total = shares.sum(-1, dtype=torch.float64)
        arrays["norms"] = (largest[..., 0].double() + total.log()).float()
        shares /= total[..., None]
        mean = (shares * arrays["logits"][..., :vocab]).sum(-1, dtype=torch.float64)
        arrays["entropy"] = (largest[..., 0].double() + total.log() - mean).float() if case["entropy"] else None
    return arrays


def _arrays(case, seed):
    make = {"norm": _norm_arrays, "linear": _linear_arrays, "log_probs": _logit_arrays}[case["op"].removesuffix("_gradient")]
    return make(case, seed)


def _empty(shape, kind):
    return torch.zeros(shape, device="cuda", dtype=TYPES[kind])


def prepare(case, seed):
    arrays, W, T = _arrays(case, seed), case["W"], case["T"]
    state = dict(case=case, arrays=arrays)
    if own:
        import paper_2506_10911_amd as nl
    if case["op"].startswith("norm"):
        weight, bias, stride = _norm_places(case)
        arrays["out"] = _empty((W, T, case["width"]), case["out"])
        if case["op"] == "norm":
            arrays["stats"] = _empty((W, T, 2), "f32")
        if own:
            state["plan"] = nl.LayerNormPlan([(weight, bias, case["width"])], stride, W, T)
    elif case["op"].startswith("linear"):
        matrix, bias, stride = _linear_places(case)
        forward = case["op"] == "linear"
        arrays["out"] = _empty((W, T, case["outputs"] if forward else case["inputs"]), case["out"])
        if forward:
            arrays["before"] = _empty((W, T, case["outputs"]), case["out"]) if case["before"] else None
        if own:
            state["plan"] = nl.LinearPlan([(matrix, case["inputs"], case["outputs"], bias, case["transposed"])], stride, W, T)
    else:
        if case["op"] == "log_probs":
            arrays["log_probs"], arrays["norms"] = _empty((W, T), "f32"), _empty((W, T), "f32")
            arrays["entropy"] = _empty((W, T), "f32") if case["entropy"] else None
            arrays["top_tokens"] = torch.zeros((W, T, case["top"]), device="cuda", dtype=torch.int32) if case["top"] else None
            arrays["top_log_probs"] = _empty((W, T, case["top"]), "f32") if case["top"] else None
        else:
            arrays["out"] = _empty((W, T, case["stride"]), case["out"])
        if own:
            state["plan"] = nl.LogProbPlan(case["vocab"], W, T, row_stride=case["stride"], max_top=case.get("top", 0))
    return state


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    one_pass = {"norm": _run_norm, "norm_gradient": _run_norm_gradient, "linear": _run_linear,
                "linear_gradient": _run_linear_gradient, "log_probs": _run_log_probs,
                "log_probs_gradient": _run_log_probs_gradient}[state["case"]["op"]]
    return one_pass(state["case"], state["arrays"], state)


def _given(**outputs):
    return {name: value for name, value in outputs.items() if value is not None}


def _run_norm(case, arrays, state):
    x, theta, out, stats = arrays["x"], arrays["theta"], arrays["out"], arrays["stats"]
    if own:
        import paper_2506_10911_amd as nl
        kinds = {"f32": nl.F32, "bf16": nl.BF16}
        nl.layer_norm(state["plan"], 0, x, kinds[case["x"]], theta, kinds[case["theta"]], case["T"], EPS, out, kinds[case["out"]],
                      stats=stats)
        return {"out": out, "stats": stats}
    weight, bias, _ = _norm_places(case)
    wide = x.float()
    mean = wide.mean(-1, keepdim=True)
    wide = wide - mean
    rstd = (wide.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = wide * rstd * _vector(theta, weight, case["width"]).float()
    if case["bias"]:
        y += _vector(theta, bias, case["width"]).float()
    return {"out": out.copy_(y), "stats": stats.copy_(torch.cat([mean, rstd], -1))}


def _put(array, offset, width, value, accumulate):
    """A vector's gradient to its place in every worker's row."""
    at = array[:, offset:offset + width]
    at.copy_(at.float() + value if accumulate else value)


def _run_norm_gradient(case, arrays, state):
    x, theta, stats, dout, add, grad, dx = (arrays[k] for k in ("x", "theta", "stats", "dout", "add", "grad", "out"))
    if own:
        import paper_2506_10911_amd as nl
        kinds = {"f32": nl.F32, "bf16": nl.BF16}
        nl.layer_norm_gradient(state["plan"], 0, dout, kinds[case["x"]], x, kinds[case["x"]], theta, kinds[case["theta"]], stats,
                               case["T"], dx, kinds[case["out"]], grad, kinds[case["theta"]], accumulate=case["accumulate"], add=add)
        return {"dx": dx, "grad": grad}
    weight, bias, _ = _norm_places(case)
    width = case["width"]
    mean, rstd = stats[..., :1], stats[..., 1:]
    xh = (x.float() - mean) * rstd
    d = dout.float()
    g = d * _vector(theta, weight, width).float()
    wide = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    dx.copy_(wide if add is None else wide + add.float())
    _put(grad, weight, width, (d * xh).sum(1), case["accumulate"])
    if case["bias"]:
        _put(grad, bias, width, d.sum(1), case["accumulate"])
    return {"dx": dx, "grad": grad}


def _activation(act, z):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if act == "gelu_tanh":      # (1 + tanh(u)) / 2 is 1 / (1 + exp(-2 u))
        return z / (1.0 + torch.exp(-math.sqrt(8.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(act, z):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if act == "gelu_tanh":
        s = 1.0 / (1.0 + torch.exp(-math.sqrt(8.0 / math.pi) * (z + 0.044715 * z * z * z)))
        return s + z * s * (1.0 - s) * math.sqrt(8.0 / math.pi) * (1.0 + 0.134145 * z * z)
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _run_linear(case, arrays, state):
    x, theta, residual, before, out = (arrays[k] for k in ("x", "theta", "residual", "before", "out"))
    if own:
        import paper_2506_10911_amd as nl
        kinds = {"f32": nl.F32, "bf16": nl.BF16}
        acts = {"none": nl.ACT_NONE, "relu": nl.ACT_RELU, "gelu": nl.ACT_GELU, "gelu_tanh": nl.ACT_GELU_TANH, "silu": nl.ACT_SILU}
        nl.linear(state["plan"], 0, x, kinds[case["x"]], theta, kinds[case["theta"]], case["T"], out, kinds[case["out"]],
                  activation=acts[case["act"]], residual=residual, before=before)
        return _given(out=out, before=before)
    z = x.float() @ _matrix(theta, case).float()
    if case["bias"]:
        z += _vector(theta, _linear_places(case)[1], case["outputs"]).float()
    y = _activation(case["act"], z)
    out.copy_(y if residual is None else y + residual.float())
    if before is not None:
        before.copy_(z)
    return _given(out=out, before=before)


def _run_linear_gradient(case, arrays, state):
    x, theta, dout, before, add, grad, dx = (arrays[k] for k in ("x", "theta", "dout", "before", "add", "grad", "out"))
    if own:
        import paper_2506_10911_amd as nl
        kinds = {"f32": nl.F32, "bf16": nl.BF16}
        acts = {"none": nl.ACT_NONE, "relu": nl.ACT_RELU, "gelu": nl.ACT_GELU, "gelu_tanh": nl.ACT_GELU_TANH, "silu": nl.ACT_SILU}
        nl.linear_gradient(state["plan"], 0, dout, kinds[case["x"]], x, kinds[case["x"]], theta, kinds[case["theta"]], case["T"],
                           dx, kinds[case["out"]], grad, kinds[case["grad"]], activation=acts[case["act"]], before=before,
                           accumulate=case["accumulate"], add=add)
        return {"dx": dx, "grad": grad}
    dz = dout.float() if before is None else dout.float() * _slope(case["act"], before.float())
    wide = dz @ _matrix(theta, case).float().mT
    dx.copy_(wide if add is None else wide + add.float())
    at, sums = _matrix(grad, case), x.float().mT @ dz
    at.copy_(at.float() + sums if case["accumulate"] else sums)
    if case["bias"]:
        _put(grad, _linear_places(case)[1], case["outputs"], dz.sum(1), case["accumulate"])
    return {"dx": dx, "grad": grad}


def _run_log_probs(case, arrays, state):
    logits, tokens, log_probs, entropy, norms = (arrays[k] for k in ("logits", "tokens", "log_probs", "entropy", "norms"))
    top, top_tokens, top_log_probs = case["top"], arrays["top_tokens"], arrays["top_log_probs"]
    if own:
        import paper_2506_10911_amd as nl
        nl.token_log_probs(state["plan"], logits, nl.BF16 if case["x"] == "bf16" else nl.F32, tokens,
                           nl.I32 if case["ids"] == "i32" else nl.I64, case["T"], log_probs, entropy=entropy, norms=norms, top=top,
                           top_tokens=top_tokens, top_log_probs=top_log_probs)
        return _given(log_probs=log_probs, norms=norms, entropy=entropy, top_tokens=top_tokens, top_log_probs=top_log_probs)
    vocab = case["vocab"]
    wide = logits[..., :vocab].float()
    largest = wide.amax(-1, keepdim=True)
    shares = (wide - largest).exp()
    total = shares.sum(-1, keepdim=True, dtype=torch.float64)       # next to 1 where one token is nearly certain
    norms.copy_((largest + total.log())[..., 0])
    there = (tokens >= 0) & (tokens < vocab)
    mine = wide.gather(2, torch.where(there, tokens, 0).long()[..., None])
    log_probs.copy_(torch.where(there, (mine - largest - total.log())[..., 0], 0.0))
    if entropy is not None:
        entropy.copy_((total.log() - (shares * (wide - largest)).sum(-1, keepdim=True) / total)[..., 0])
    if top:
        most, index = wide.sort(dim=-1, descending=True, stable=True)
        count = min(top, vocab)
        top_tokens.fill_(-1)
        top_log_probs.fill_(-math.inf)
        top_tokens[..., :count] = index[..., :count].int()
        top_log_probs[..., :count] = (most[..., :count] - largest - total.log()).float()
    return _given(log_probs=log_probs, norms=norms, entropy=entropy, top_tokens=top_tokens, top_log_probs=top_log_probs)


def _run_log_probs_gradient(case, arrays, state):
    logits, tokens, norms, dlog_probs, dentropy, entropy, dlogits = (
        arrays[k] for k in ("logits", "tokens", "norms", "dlog_probs", "dentropy", "entropy", "out"))
    if own:
        import paper_2506_10911_amd as nl
        kinds = {"f32": nl.F32, "bf16": nl.BF16}
        nl.token_log_probs_gradient(state["plan"], logits, kinds[case["x"]], tokens, nl.I32 if case["ids"] == "i32" else nl.I64,
                                    case["T"], norms, dlog_probs, dlogits, kinds[case["out"]], dentropy=dentropy, entropy=entropy)
        return dlogits
    vocab = case["vocab"]
    there = (tokens >= 0) & (tokens < vocab)
    by = torch.where(there, dlog_probs, 0.0)[..., None]
    logs = logits[..., :vocab].float() - norms[..., None]
    shares = logs.exp()
    wide = -by * shares
    index = torch.where(there, tokens, 0).long()[..., None]         # 1 - p there, also where p is next to 1
    wide.scatter_(2, index, by * -torch.expm1(logs.gather(2, index)))
    if dentropy is not None:
        wide -= dentropy[..., None] * shares * (logs + entropy[..., None])
    dlogits[..., :vocab].copy_(wide)
    return dlogits


# ---------------------------------------------------------------------------
# What a pass cannot do without, and what its outputs are
# ---------------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
    op, W, T = case["op"], case["W"], case["T"]
    if op.startswith("norm"):
        width, vectors = case["width"], case["width"] * (2 if case["bias"] else 1)
        if op == "norm":
            each = width * (size[case["x"]] + size[case["out"]]) + 8
            return {"bytes": W * (T * each + vectors * size[case["theta"]]), "flops": W * T * width * 8}
        each = width * (2 * size[case["x"]] + size[case["out"]] * (2 if case["add"] else 1)) + 8
        of_grad = vectors * size[case["theta"]] * (2 if case["accumulate"] else 1)
        return {"bytes": W * (T * each + width * size[case["theta"]] + of_grad), "flops": W * T * width * 14}
    if op.startswith("linear"):
        inputs, outputs = case["inputs"], case["outputs"]
        weights, vector = inputs * outputs * size[case["theta"]], outputs if case["bias"] else 0
        if op == "linear":
            rows = inputs * size[case["x"]] + outputs * size[case["out"]] * (1 + case["before"] + case["residual"])
            return {"bytes": W * (T * rows + weights + vector * size[case["theta"]]), "flops": 2 * W * T * inputs * outputs}
        rows = (inputs + outputs * (1 if case["act"] == "none" else 2)) * size[case["x"]] + inputs * size[case["out"]] * (1 + case["add"])
        of_grad = (inputs * outputs + vector) * size[case["grad"]] * (2 if case["accumulate"] else 1)
        return {"bytes": W * (T * rows + weights + of_grad), "flops": 4 * W * T * inputs * outputs}
    vocab, real = case["vocab"], T - _padding(T)
    if op == "log_probs":
        each = vocab * size[case["x"]] + size[case["ids"]] + 8 + (4 if case["entropy"] else 0) + 8 * case["top"]
        return {"bytes": W * T * each, "flops": W * T * vocab * 4}
    read = T if case["entropy"] else real           # a position without a token has a row of zeros
    moved = read * vocab * size[case["x"]] + T * vocab * size[case["out"]] + T * (size[case["ids"]] + (16 if case["entropy"] else 8))
    return {"bytes": W * moved, "flops": W * read * vocab * 4}


def exact(case, seed):
    arrays = _arrays(case, seed)
    return {"norm": _exact_norm, "norm_gradient": _exact_norm_gradient, "linear": _exact_linear,
            "linear_gradient": _exact_linear_gradient, "log_probs": _exact_log_probs,
            "log_probs_gradient": _exact_log_probs_gradient}[case["op"]](case, arrays)


def _exact_norm(case, arrays):
    out = torch.empty((case["W"], case["T"], case["width"]), device="cuda", dtype=torch.float64)
    stats = torch.empty((case["W"], case["T"], 2), device="cuda", dtype=torch.float64)
    weight, bias, _ = _norm_places(case)
    for w in range(case["W"]):
        x, row = arrays["x"][w].double(), arrays["theta"][w].double()
        rstd = (x.var(-1, correction=0) + EPS) ** -0.5
        stats[w, :, 0], stats[w, :, 1] = x.mean(-1), rstd
        out[w] = (x - x.mean(-1, keepdim=True)) * rstd[:, None] * row[weight:weight + case["width"]]
        if case["bias"]:
            out[w] += row[bias:bias + case["width"]]
    return {"out": out, "stats": stats}


def _exact_norm_gradient(case, arrays):
    """dx by the product with the Jacobian rstd (1 - 1/n - xh xh^T / n), from the statistics that are given."""
    weight, bias, _ = _norm_places(case)
    n, grad = case["width"], arrays["grad"].double()
    dx = torch.empty((case["W"], case["T"], n), device="cuda", dtype=torch.float64)
    for w in range(case["W"]):
        mean, rstd = arrays["stats"][w].double().unbind(-1)
        xh = (arrays["x"][w].double() - mean[:, None]) * rstd[:, None]
        d = arrays["dout"][w].double()
        g = d * arrays["theta"][w, weight:weight + n].double()
        dx[w] = (g - (g.sum(-1, keepdim=True) + xh * (g * xh).sum(-1, keepdim=True)) / n) * rstd[:, None]
        if case["add"]:
            dx[w] += arrays["add"][w].double()
        for at, value in ((weight, (d * xh).sum(0)), (bias, d.sum(0))):
            if at >= 0:
                grad[w, at:at + n] = value + (grad[w, at:at + n] if case["accumulate"] else 0.0)
    return {"dx": dx, "grad": grad}


def _exact_weights(row, case):
    """One worker's matrix as [inputs, outputs]."""
    part = row[case["gap"]:case["gap"] + case["inputs"] * case["outputs"]]
    return part.view(case["outputs"], case["inputs"]).T if case["transposed"] else part.view(case["inputs"], case["outputs"])


def _exact_activation(act, z):
    """(activation, its derivative): by the normal distribution, and by sigmoids in place of tanh."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "gelu":
        below = 0.5 * torch.erfc(-z / 2 ** 0.5)
        return z * below, below + z * (-0.5 * z ** 2).exp() / (2 * math.pi) ** 0.5
    by, cubic = (1.0, 0.0) if act == "silu" else (2 * (2 / math.pi) ** 0.5, 0.044715)
    s = torch.sigmoid(by * (z + cubic * z ** 3))
    return z * s, s + z * s * (1 - s) * by * (1 + 3 * cubic * z ** 2)


def _exact_linear(case, arrays):
    shape = (case["W"], case["T"], case["outputs"])
    out, before = (torch.empty(shape, device="cuda", dtype=torch.float64) for _ in range(2))
    bias = _linear_places(case)[1]
    for w in range(case["W"]):
        row = arrays["theta"][w].double()
        before[w] = arrays["x"][w].double() @ _exact_weights(row, case)
        if case["bias"]:
            before[w] += row[bias:bias + case["outputs"]]
        out[w] = _exact_activation(case["act"], before[w])[0]
        if case["residual"]:
            out[w] += arrays["residual"][w].double()
    return _given(out=out, before=before if case["before"] else None)


def _exact_linear_gradient(case, arrays):
    dx = torch.empty((case["W"], case["T"], case["inputs"]), device="cuda", dtype=torch.float64)
    grad, bias = arrays["grad"].double(), _linear_places(case)[1]
    for w in range(case["W"]):
        dz = arrays["dout"][w].double()
        if case["act"] != "none":
            dz = dz * _exact_activation(case["act"], arrays["before"][w].double())[1]
        dx[w] = dz @ _exact_weights(arrays["theta"][w].double(), case).T
        if case["add"]:
            dx[w] += arrays["add"][w].double()
        at = _exact_weights(grad[w], case)
        at.copy_(arrays["x"][w].double().T @ dz + (at if case["accumulate"] else 0.0))
        if case["bias"]:
            part = grad[w, bias:bias + case["outputs"]]
            part.copy_(dz.sum(0) + (part if case["accumulate"] else 0.0))
    return {"dx": dx, "grad": grad}


def _exact_log_probs(case, arrays):
    W, T, top = case["W"], case["T"], case["top"]
    log_probs, norms, entropy = (torch.zeros((W, T), device="cuda", dtype=torch.float64) for _ in range(3))
    top_tokens = torch.full((W, T, top), -1, device="cuda", dtype=torch.int32)
    top_log_probs = torch.full((W, T, top), -math.inf, device="cuda", dtype=torch.float64)
    for w in range(W):
        logits, tokens = arrays["logits"][w, :, :case["vocab"]].double(), arrays["tokens"][w].long()
        norms[w] = torch.logsumexp(logits, -1)
        logs = logits - norms[w][:, None]
        real = tokens >= 0
        log_probs[w, real] = logs[real, tokens[real]]
        entropy[w] = -(logs.exp() * logs).sum(-1)
        for k in range(min(top, case["vocab"])):            # the first of the largest, again and again
            most = logs.amax(-1, keepdim=True)
            index = torch.where(logs == most, torch.arange(case["vocab"], device="cuda"), case["vocab"]).amin(-1, keepdim=True)
            top_tokens[w, :, k:k + 1], top_log_probs[w, :, k:k + 1] = index.int(), most
            logs.scatter_(1, index, -math.inf)
    return _given(log_probs=log_probs, norms=norms, entropy=entropy if case["entropy"] else None,
                  top_tokens=top_tokens if top else None, top_log_probs=top_log_probs if top else None)


def _exact_log_probs_gradient(case, arrays):
    dlogits, vocab = torch.zeros((case["W"], case["T"], case["stride"]), device="cuda", dtype=torch.float64), case["vocab"]
    for w in range(case["W"]):
        tokens = arrays["tokens"][w].long()
        real = (tokens >= 0).nonzero()[:, 0]
        logs = arrays["logits"][w, :, :vocab].double() - arrays["norms"][w].double()[:, None]
        at = dlogits[w, :, :vocab]
        at[real] = -arrays["dlog_probs"][w, real].double()[:, None] * logs[real].exp()
        at[real, tokens[real]] += arrays["dlog_probs"][w, real].double()
        if case["entropy"]:
            at -= arrays["dentropy"][w].double()[:, None] * logs.exp() * (logs + arrays["entropy"][w].double()[:, None])
    return dlogits
