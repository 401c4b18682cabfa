"""Plain implementations in 64 bits of the inner step's operators, and what the kernels may be off by.

Nothing here imports the library: torch on the CPU, from the formulas of noloco.h."""
import torch

COEFFICIENTS = ((3.4445, -4.7750, 2.0315),) * 5


def _noisy(x, unit, gen):
    """x with every number off by up to `unit` of itself, as a rounding leaves it."""
    return x if gen is None else x * (1 + unit * (2 * torch.rand(x.shape, dtype=torch.float64, generator=gen) - 1))


def newton_schulz(u, coefficients=COEFFICIENTS, eps=1e-7, unit=0.0, gen=None):
    """The orthogonalised u (float64, 2-d). With `gen`, everything that the kernels round (X_0, and A, P and X of every
    step) is off by up to `unit` of itself."""
    if u.shape[0] > u.shape[1]:
        return newton_schulz(u.T.contiguous(), coefficients, eps, unit, gen).T
    norm = u.square().sum().sqrt() + eps
    x = _noisy(u / norm if norm > 0 else torch.zeros_like(u), unit, gen)
    eye = torch.eye(x.shape[0], dtype=torch.float64)
    for a, b, c in coefficients:
        gram = _noisy(x @ x.T, unit, gen)
        poly = _noisy(a * eye + b * gram + c * gram @ gram, unit, gen)
        x = _noisy(poly @ x, unit, gen)
    return x


# One binary16 a number rounds by up to 2^-11 of it. A pair holds 22 bits, and its sums in binary32 are off by some
# roundings of 2^-24: 2^-21 covers both.
UNITS = {"f16": 2.0 ** -11, "pairs": 2.0 ** -21}
# Rounding to nearest with p significant bits: 2^-p of the number (bf16 has 8, binary32 24).
STORED = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def newton_schulz_bound(u, products, out_dtype, coefficients=COEFFICIENTS, eps=1e-7):
    """Most that the kernels' result may be off by in the 2-norm: twice what roundings of the full size, at random signs,
    do to the 64-bit result (the worst of three draws), and the rounding of the result itself."""
    exact = newton_schulz(u, coefficients, eps)
    worst = 0.0
    for seed in range(3):
        gen = torch.Generator().manual_seed(seed)
        worst = max(worst, (newton_schulz(u, coefficients, eps, UNITS[products], gen) - exact).norm().item())
    return exact, 2 * worst + STORED[out_dtype] * exact.norm().item() + 1e-12


def view(array, offset, rows, cols, row_stride):
    """One matrix of every worker, [W, rows, cols], over the arena's memory."""
    return array.as_strided((array.shape[0], rows, cols), (array.stride(0), row_stride, 1), array.storage_offset() + offset)


def lookup(table, tokens, scale, dtype):
    """table [W, vocab, width], tokens [W, T]: a binary32 product rounded once, which is exact to compare with."""
    there = (tokens >= 0) & (tokens < table.shape[1])
    rows = torch.stack([t[i] for t, i in zip(table.float(), torch.where(there, tokens, 0).long())])
    return torch.where(there[..., None], rows * torch.tensor(scale, dtype=torch.float32), torch.zeros(())).to(dtype)


def gradient(dout, tokens, scale, grad, accumulate):
    """(gradient, its bound) in 64 bits: a sum of n numbers in binary32 is off by at most n 2^-24 of the sum of their sizes;
    the product with the scale, the addition and the rounding to grad's type follow."""
    W, vocab, width = grad.shape
    scale = float(torch.tensor(scale, dtype=torch.float32))
    out = grad.double().clone() if accumulate else torch.zeros(grad.shape, dtype=torch.float64)
    sizes, counts = torch.zeros_like(out), torch.zeros((W, vocab, 1), dtype=torch.float64)
    for w in range(W):
        real = (tokens[w] >= 0) & (tokens[w] < vocab)
        index = tokens[w][real].long()
        out[w].index_add_(0, index, scale * dout[w][real].double())
        sizes[w].index_add_(0, index, abs(scale) * dout[w][real].double().abs())
        counts[w].index_add_(0, index, torch.ones((len(index), 1), dtype=torch.float64))
    unit = 2.0 ** -24
    return out, (counts + 2) * unit * sizes * 1.01 + (unit + STORED[grad.dtype]) * (out.abs() + sizes * counts * unit) + 1e-30
