"""Plain implementations in 64 bits of layer norm, matrices and log probabilities, and what the kernels may be off by.

Nothing here imports the library: torch on the CPU, from the formulas of noloco.h. Every bound is a sum of roundings: U for an
operation in binary32 (half a step, relative to its result), STORED for a result's own type, and for a sum of n numbers n U
of the sum of their sizes. Second-order terms are covered by SLACK."""
import math

import torch

U = 2.0 ** -24
STORED = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
SLACK = 1.01
TINY = 1e-37            # binary32's range ends there: products below it may be lost


def additions(width):
    """Most additions one after the other in a row's sum: a thread's own, six steps of a wave, sixteen waves."""
    return 16 + 6 + 16 + math.ceil(width / 1024)


def layer_norm(x, weight, bias, eps, out_dtype):
    """((out, its bound), (stats, their bound)); x [W, T, n], weight and bias [W, n] or None."""
    x = x.double()
    n, adds = x.shape[-1], additions(x.shape[-1])
    weight = weight.double()[:, None]
    mean = x.mean(-1, keepdim=True)
    off_mean = (adds + 1) * U * x.abs().mean(-1, keepdim=True)
    d = x - mean
    off_d = off_mean + U * d.abs()
    var = d.square().mean(-1, keepdim=True)
    off_var = (2 * d.abs() * off_d + off_d.square()).mean(-1, keepdim=True) + (adds + 3) * U * var
    rstd = (var + eps).rsqrt()
    rel = 0.5 * off_var / (var + eps) + 4 * U
    scaled = d * rstd * weight
    y = scaled if bias is None else scaled + bias.double()[:, None]
    bound = (off_d * rstd * weight.abs() + scaled.abs() * (rel + 2 * U)) * SLACK + (U + STORED[out_dtype]) * y.abs() + TINY
    stats = torch.cat([mean, rstd], -1)
    return (y, bound), (stats, torch.cat([off_mean + U * mean.abs(), rstd * rel], -1) * SLACK + TINY)


def layer_norm_gradient(dout, x, weight, stats, add, dx_dtype):
    """((dx, bound), (weight's gradient, bound), (bias's, bound)), the last two sums over tokens, [W, n]."""
    d, x, mean, rstd = dout.double(), x.double(), stats[..., :1].double(), stats[..., 1:].double()
    n, adds, T = x.shape[-1], additions(x.shape[-1]), x.shape[1]
    xh = (x - mean) * rstd
    g = d * weight.double()[:, None]
    c1, c2 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    off_c1 = (adds + 2) * U * g.abs().mean(-1, keepdim=True)
    off_c2 = (adds + 5) * U * (g * xh).abs().mean(-1, keepdim=True)
    dx = rstd * (g - c1 - xh * c2)
    off = rstd * (U * g.abs() + off_c1 + xh.abs() * off_c2 + 5 * U * (g.abs() + c1.abs() + (xh * c2).abs()))
    if add is not None:
        dx = dx + add.double()
    bound = off * SLACK + (U + STORED[dx_dtype]) * dx.abs() + TINY
    grads = []
    for part in (d * xh, d):
        grads.append((part.sum(1), (T + 8) * U * part.abs().sum(1) * SLACK + TINY))
    return (dx, bound), *grads


def stored(value, bound, old, dtype):
    """A gradient as it is stored: added to `old` (None: written), rounded to its type."""
    if old is not None:
        value, bound = value + old.double(), bound + U * (value + old.double()).abs()
    return value, bound + STORED[dtype] * value.abs() * SLACK


def activation(name, z):
    """(act(z), act'(z)) in 64 bits."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "gelu":
        below = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * below, below + z * (-0.5 * z * z).exp() / math.sqrt(2 * math.pi)
    by, cubic = (1.0, 0.0) if name == "silu" else (2 * math.sqrt(2 / math.pi), 0.044715)
    s = torch.sigmoid(by * (z + cubic * z ** 3))
    return z * s, s + z * s * (1 - s) * by * (1 + 3 * cubic * z * z)


STEEPEST = 1.2          # |act'| of all of them
BENT = 1.3              # |act''|, of those that have one (2 / sqrt(2 pi) and less), but at a relu's step


def off_activation(z):
    """What evaluating act or act' in binary32 may add: some functions of 4 U each, with arguments up to z^2."""
    return 8 * U * (1 + z.abs()) * (1 + z * z)


def product(a, b, out_dtype):
    """(a @ b, bound) for a [.., m, k], b [.., k, n] as they are stored. A bf16 result: float operands are rounded to bf16. A float
    one: three bf16 a float operand, of whose products those of 2^-24 are left out, or two binary16 (2^-22 of a number, or 2^-40 of
    its worker's largest), of whose products that of the low halves, 2^-22, is left out; as many additions as there are products."""
    sizes = a.double().abs() @ b.double().abs()
    floats = [t.dtype == torch.float32 for t in (a, b)]
    k = a.shape[-1]
    if out_dtype == torch.bfloat16:
        rel = sum(STORED[torch.bfloat16] for f in floats if f) * SLACK + (k + 4) * U
        least = 0.0
    else:
        rel = ({0: 1, 1: 3, 2: 6}[sum(floats)] * k + 4) * U + 4 * U * sum(floats) + (4 * U if all(floats) else 0)
        least = 0.0
        if any(floats):
            largest = [t.double().abs().amax((-2, -1), keepdim=True) for t in (a, b)]
            least = 2.0 ** -40 * (largest[0] * b.double().abs().sum(-2, keepdim=True) + largest[1] * a.double().abs().sum(-1, keepdim=True))
    return a.double() @ b.double(), (rel * sizes + least) * SLACK + TINY * k


def linear(x, matrix, bias, act, residual, out_dtype):
    """((out, bound), (before, bound)); x [W, T, i], matrix [W, i, o], bias [W, o] or None."""
    z, off = product(x, matrix, out_dtype)
    if bias is not None:
        z = z + bias.double()[:, None]
        off = off + U * z.abs()
    y = activation(act, z)[0]
    bound = off * STEEPEST + (off_activation(z) if act not in ("none", "relu") else 0)
    if residual is not None:
        y = y + residual.double()
    return (y, bound * SLACK + (U + STORED[out_dtype]) * y.abs() + TINY), (z, off * SLACK + STORED[out_dtype] * z.abs() + TINY)


def linear_gradient(dout, x, matrix, before, act, add, dx_dtype, grad_dtype):
    """((dx, bound), (matrix's gradient, bound), (bias's, bound))"""
    dz, off = dout.double(), torch.zeros((), dtype=torch.float64)
    if act != "none":
        slope = activation(act, before.double())[1]
        dz = dz * slope
        off = dout.double().abs() * (off_activation(before.double()) if act != "relu" else 0) + U * dz.abs()
    kept = dout if act == "none" else dout.to(torch.float32)         # its type: what the products take it as

    def through(a, b, which, out_dtype):
        """A product with dz in place of operand `which`: the roundings of its type, and what it is off itself."""
        pair = [a, b]
        pair[which] = dz
        exact = pair[0].double() @ pair[1].double()
        pair[which] = dz.to(kept.dtype)           # off by a rounding of binary32 at most, which `off` has
        bound = product(*pair, out_dtype)[1]
        offs = [t.double().abs() for t in pair]
        offs[which] = off.expand_as(dz)
        return exact, bound * SLACK + offs[0] @ offs[1] + TINY

    dx, dx_bound = through(dout, matrix.mT, 0, dx_dtype)
    if add is not None:
        dx = dx + add.double()
    dx_bound = dx_bound * SLACK + (U + STORED[dx_dtype]) * dx.abs() + TINY
    of_matrix = through(x.mT, dout, 1, grad_dtype)
    T = dout.shape[1]
    of_bias = dz.sum(1), ((T + 4) * U * dz.abs().sum(1) + off.expand_as(dz).sum(1)) * SLACK + TINY
    return (dx, dx_bound), of_matrix, of_bias


def log_probs(logits, tokens):
    """{name: (value, bound)} of log_probs, norms, entropy, and all logits' log probabilities; logits [.., vocab] without NaN and
    +infinity, tokens [..]. A share exp(l - largest) is off by (|l - largest| + 20) 2^-23 of itself: the distance's rounding and its
    product with log2(e), the power, and the reference that it is taken from, up to 16 away."""
    l = logits.double()
    vocab = l.shape[-1]
    largest = l.amax(-1, keepdim=True)
    nothing = largest == -math.inf
    d = torch.where(nothing, -math.inf, l - torch.where(nothing, 0.0, largest))
    shares = d.exp()
    far = torch.where(shares > 0, d.abs(), 0.0)
    first = torch.zeros_like(shares).scatter_(-1, l.argmax(-1, keepdim=True), 1.0)
    rest = (shares * (1 - first)).sum(-1, keepdim=True)
    adds = math.ceil(vocab / 64) + 48
    off_rest = ((far + 20) * 2.0 ** -23 * shares * (1 - first)).sum(-1, keepdim=True) + adds * U * rest
    # a rest of 1 and more is taken from a sum that the largest is part of
    off_rest = off_rest + torch.where(rest > 0.9, (adds + 40) * U * (1 + rest), 0.0)
    total = torch.log1p(rest)
    off_total = off_rest / (1 + rest) + 3 * U * total
    norms = (largest + total)[..., 0]
    logs = torch.where(nothing, -math.inf, d - total)
    off_logs = off_total + 2 * U * far + 2 * U * torch.where(logs > -math.inf, logs.abs(), 0.0) + TINY
    spread = (shares * far).sum(-1, keepdim=True)
    off_spread = ((far + 20) * 2.0 ** -23 * shares * (far + 16)).sum(-1, keepdim=True) + adds * U * (shares * (far + 16)).sum(-1, keepdim=True) * \
        torch.where(rest > 0.9, 1.0, 0.0) + adds * U * spread
    entropy = total + spread / (1 + rest)
    off_entropy = off_total + off_spread / (1 + rest) + spread / (1 + rest) * off_rest / (1 + rest) + 4 * U * entropy
    there = (tokens >= 0) & (tokens < vocab)
    index = torch.where(there, tokens, 0).long()[..., None]
    mine, off_mine = logs.gather(-1, index)[..., 0], off_logs.gather(-1, index)[..., 0]
    zero = torch.zeros((), dtype=torch.float64)
    return {
        "log_probs": (torch.where(there, mine, zero), torch.where(there, off_mine, zero) * SLACK + TINY),
        "norms": (torch.where(nothing[..., 0], -math.inf, norms), off_total[..., 0] * SLACK + 2 * U * torch.where(nothing, 0.0, largest + total).abs()[..., 0] + TINY),
        "entropy": (torch.where(nothing[..., 0], 0.0, entropy[..., 0]), off_entropy[..., 0] * SLACK + TINY),
        "all": (logs, off_logs * SLACK),
    }


def top_tokens(logits, top):
    """The `top` largest logits' tokens, the lower first where they are equal, NaN as -infinity; -1 behind a small vocabulary."""
    l = torch.where(logits.isnan(), -math.inf, logits.double())
    order = l.sort(dim=-1, descending=True, stable=True)[1][..., :top]
    out = torch.full((*logits.shape[:-1], top), -1, dtype=torch.int64)
    out[..., :order.shape[-1]] = order
    return out


def log_probs_gradient(logits, tokens, norms, dlog_probs, dentropy, entropy, dtype):
    """(dlogits, bound) from the norms and entropies that are given."""
    vocab = logits.shape[-1]
    l, n = logits.double(), norms.double()[..., None]
    there = ((tokens >= 0) & (tokens < vocab))[..., None]
    by = torch.where(there, dlog_probs.double()[..., None], 0.0)
    nothing = (n == -math.inf)
    d = torch.where(nothing, -math.inf, l - torch.where(nothing, 0.0, n))
    p = d.exp()
    far = torch.where(p > 0, d.abs(), 0.0)
    off_p = p * (2 * far + 4) * 2.0 ** -23
    hit = torch.zeros_like(p).scatter_(-1, torch.where(there[..., 0], tokens, 0).long()[..., None], 1.0) * there
    value = by * (hit - p)
    # at the token -expm1(d): of its own size, not of 1
    off = by.abs() * torch.where(hit > 0, (U * far + 4 * U) * (1 - p).abs() + U * far * p, off_p + U * p)
    if dentropy is not None:
        de, h = dentropy.double()[..., None], entropy.double()[..., None]
        more = torch.where(p > 0, de * p * (torch.where(p > 0, d, 0.0) + h), 0.0)
        value = value - more
        off = off + de.abs() * (off_p * (far + h.abs()) + 4 * U * p * (far + h.abs())) + U * value.abs()
    value = torch.where(nothing, 0.0, value)
    return value, torch.where(nothing, 0.0, off) * SLACK + STORED[dtype] * value.abs() * SLACK + TINY
