"""Orthogonalisation and updates of matrices that go through a launch for each product, on the GPU, against 64-bit references."""
import functools

import pytest
import torch

import inner_plain as plain
from test_gpu_muon import DTYPES, code, filled, layout, owned, same_bits

pytestmark = pytest.mark.gpu
nl = pytest.importorskip("paper_2506_10911_amd")

# One binary16 a number rounds X_0 and four more X by up to 2^-11 of every number, a third of its square on average: at worst
# sqrt(5 / 3) 2^-11 = 0.00063 of the norm. What A and P lose beside their diagonals comes to it.
F16_OFF = 2.0 ** -10

PRODUCTS = {"f16": nl.PRODUCTS_F16, "pairs": nl.PRODUCTS_PAIRS}

# Shapes, workers, the first matrix's place, and what is planned for them in both formats: the tile, and whether X X^T is summed
# in parts (tests/test_inner_plans.py asks the planning for it).
PATHS = {
    "64": ([(260, 516), (516, 260, 300)], 2, 0, 64, False),
    "64 at odd places": ([(129, 333, 335), (333, 131)], 2, 3, 64, False),
    "64 in parts": ([(40, 4100), (1500, 90), (1, 70001)], 2, 0, 64, True),
    "128": ([(600, 604), (604, 600, 612)], 9, 0, 128, False),
    "128 at odd places": ([(600, 601, 611), (641, 600)], 9, 1, 128, False),
    "256": ([(1270, 1276), (1276, 1272)], 18, 0, 256, False),
    "256 at odd places": ([(1273, 1270, 1279)], 35, 5, 256, False),
}


def path(name):
    """(matrices, stride, W, tile, whether X X^T is summed in parts)"""
    shapes, W, first, tile, shared = PATHS[name]
    matrices, stride = layout(shapes, gap=4 if first == 0 else first, first=first)
    if first == 0:                                       # every matrix at a multiple of four
        at, moved = 0, []
        for _, rows, cols, row_stride, scale in matrices:
            moved.append((at, rows, cols, row_stride, scale))
            at = -(-(at + (rows - 1) * row_stride + cols) // 4) * 4 + 4
        matrices, stride = moved, -(-at // 64) * 64
    return matrices, stride, W, tile, shared


NARROW = [(4, 6000), (6000, 4), (4, 1024), (32, 512), (2000, 32)]


def parts(array, matrix):
    return plain.view(array, *matrix[:4]).cpu().double()


def check_narrow(matrices, which, W, seed):
    """Results of the matrices `which` of a plan of all of them: in binary16 to F16_OFF, as bf16 to that and their own rounding."""
    stride = max(-(-max(o + (r - 1) * s + c for o, r, c, s, _ in matrices) // 64) * 64, 64)
    x = filled(matrices, W, stride, torch.float32, seed=seed)
    d_x = x.cuda()
    plan = nl.MuonPlan(matrices, stride, W)
    got = torch.zeros((W, stride), device="cuda")
    nl.orthogonalize(plan, d_x, nl.F32, got, nl.F32, products=nl.PRODUCTS_F16)
    half = torch.zeros((W, stride), dtype=torch.bfloat16, device="cuda")
    nl.orthogonalize(plan, d_x, nl.F32, half, nl.BF16)
    for k in which:
        for w in range(W):
            exact = plain.newton_schulz(plain.view(x, *matrices[k][:4])[w].double())
            norm = exact.norm().item()
            what = f"{matrices[k][1]}x{matrices[k][2]} of worker {w}"
            off = (parts(got, matrices[k])[w] - exact).norm().item() / norm
            assert off <= F16_OFF, f"{what}: {off:.5f}"
            rounding = (exact.to(torch.bfloat16).double() - exact).norm().item() / norm
            off = (parts(half, matrices[k])[w] - exact).norm().item() / norm
            assert off <= (rounding ** 2 + F16_OFF ** 2) ** 0.5, f"{what} in bf16: {off:.5f}, its rounding {rounding:.5f}"


@pytest.mark.parametrize("narrow", NARROW, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("others", [1, 14])
def test_narrow_matrices_are_as_exact_beside_others(narrow, others):
    """All singular values of a matrix much longer than wide are alike, so that one rounding of A's diagonal is in all of
    them. 14 of 768 x 768 are enough for tiles of 128."""
    matrices, _ = layout([narrow] * 3 + [(768, 768)] * others)
    check_narrow(matrices, range(3), 1, seed=21)


def test_long_matrix_in_large_tiles():
    """52 matrices of 1024 x 1024 and a long one: tiles of 256."""
    matrices, _ = layout([(1024, 16384)] + [(1024, 1024)] * 52, gap=4)
    check_narrow(matrices, [0, 52], 1, seed=22)


def everywhere(matrices, W, stride, dtype, seed):
    """The same row for every worker: their results are the same bits, and one is compared with the formula."""
    return filled(matrices, 1, stride, dtype, seed=seed).expand(W, stride).contiguous()


def alike(got):
    for w in range(1, got.shape[0]):
        assert same_bits(got[w], got[0]), f"worker {w}"


@functools.lru_cache(maxsize=None)
def bounds(name, what, products):
    """Exact result and its bound (before it is stored) of every matrix of a path, from inputs of bf16 numbers."""
    matrices, stride, *_ = path(name)
    grad = filled(matrices, 1, stride, torch.bfloat16, seed=31)
    moved = filled(matrices, 1, stride, torch.float32, seed=32)
    found = []
    for m in matrices:
        g, mom = plain.view(grad, *m[:4])[0].double(), plain.view(moved, *m[:4])[0].double()
        mom = 0.9 * mom + g
        u = {"x": g, "momentum": mom, "nesterov": g + 0.9 * mom}[what]
        found.append(plain.newton_schulz_bound(u, products, torch.float32))
    return found


@pytest.mark.parametrize("products", PRODUCTS)
@pytest.mark.parametrize("name", PATHS)
def test_orthogonalize(name, products):
    matrices, stride, W, *_ = path(name)
    mask = owned(matrices, 1, stride)[0]
    for into in ("bf16", "f32"):
        x = everywhere(matrices, W, stride, torch.bfloat16, 31).to(DTYPES[into]).cuda()
        for out in ("f32", "bf16"):
            got = torch.full((W, stride), 7.0, dtype=DTYPES[out], device="cuda")
            nl.orthogonalize(nl.MuonPlan(matrices, stride, W), x, code(x.dtype), got, code(got.dtype), products=PRODUCTS[products])
            alike(got)
            row = got[:1].cpu()
            assert (row[0, ~mask] == 7.0).all()
            for m, (exact, bound) in zip(matrices, bounds(name, "x", products)):
                off = (plain.view(row, *m[:4])[0].double() - exact).norm().item()
                most = bound + (plain.STORED[DTYPES[out]] * exact.norm().item() if out == "bf16" else 0.0)
                assert off <= most, f"{m[1]}x{m[2]} {into} to {out}: off by {off:.3g}, at most {most:.3g}"


@pytest.mark.parametrize("products", PRODUCTS)
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("name", PATHS)
def test_muon_step(name, nesterov, products):
    """One update against the formula in 64 bits, weights about as large as the update."""
    matrices, stride, W, *_ = path(name)
    lr, mu, decay = 0.05, 0.9, 0.2
    mask = owned(matrices, 1, stride)
    g = everywhere(matrices, W, stride, torch.bfloat16, 31)
    moved = everywhere(matrices, W, stride, torch.float32, 32)
    weights = everywhere(matrices, W, stride, torch.bfloat16, 33)
    plan = nl.MuonPlan(matrices, stride, W)
    for theta, grad in (("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")):
        before = weights.to(DTYPES[theta])
        d_theta, d_moved = before.cuda(), moved.cuda()
        nl.muon_step(plan, d_theta, code(d_theta.dtype), g.to(DTYPES[grad]).cuda(), code(DTYPES[grad]), d_moved, (lr, mu, decay),
                     nesterov=nesterov, products=PRODUCTS[products])
        alike(d_theta)
        alike(d_moved)
        after, moved_after = d_theta[:1].cpu(), d_moved[:1].cpu()
        for a, b in ((after, before[:1]), (moved_after, moved[:1])):
            assert same_bits(torch.where(mask, torch.zeros_like(a), a), torch.where(mask, torch.zeros_like(b), b))
        for m, (exact, bound) in zip(matrices, bounds(name, "nesterov" if nesterov else "momentum", products)):
            at, scale = m[:4], m[4]
            gw, mw = plain.view(g, *at)[0].double(), plain.view(moved, *at)[0].double()
            mom = mu * mw + gw
            off = (plain.view(moved_after, *at)[0].double() - mom).abs()
            assert (off <= 2.0 ** -23 * (mu * mw.abs() + mom.abs()) + 2.0 ** -24 * mw.abs()).all()
            old = plain.view(before, *at)[0].double()
            want = (1 - lr * decay) * old - lr * scale * exact
            # binary32 operations on old and the step, the weight's rounding, and u's, which five steps multiply by at most 3.9 each
            most = (lr * scale * (bound + 3.9 ** 5 * 2.0 ** -23) + 3 * 2.0 ** -24 * (old.norm() + lr * scale * exact.norm())
                    + plain.STORED[DTYPES[theta]] * want.norm())
            off = (plain.view(after, *at)[0].double() - want).norm()
            assert off <= most, f"{m[1]}x{m[2]} theta {theta} grad {grad}: off by {off:.3g}, at most {most:.3g}"


@pytest.mark.parametrize("products", PRODUCTS)
@pytest.mark.parametrize("theta", ["f32", "bf16"])
def test_muon_step_of_small_matrices(theta, products):
    """The update of matrices that one workgroup takes, under the bound of the products that are asked for."""
    matrices, stride = layout([(48, 80), (80, 48, 90), (1, 77), (65, 65), (64, 96, 100)], gap=4)
    lr, mu, decay = 0.05, 0.9, 0.2
    weights = filled(matrices, 2, stride, DTYPES[theta], seed=41)
    g, moved = filled(matrices, 2, stride, torch.float32, seed=42), filled(matrices, 2, stride, torch.float32, seed=43)
    plan = nl.MuonPlan(matrices, stride, 2)
    got = {}
    for kind in (PRODUCTS[products], nl.PRODUCTS_AUTO):
        got[kind] = weights.cuda()
        nl.muon_step(plan, got[kind], code(DTYPES[theta]), g.cuda(), nl.F32, moved.cuda(), (lr, mu, decay), products=kind)
    assert products == "f16" or same_bits(got[PRODUCTS[products]].nan_to_num(), got[nl.PRODUCTS_AUTO].nan_to_num())
    after = got[PRODUCTS[products]].cpu()
    for m in matrices:
        at, scale = m[:4], m[4]
        for w in range(2):
            gw = plain.view(g, *at)[w].double()
            u = gw + mu * (mu * plain.view(moved, *at)[w].double() + gw)
            exact, bound = plain.newton_schulz_bound(u, products, torch.float32)
            old = plain.view(weights, *at)[w].double()
            want = (1 - lr * decay) * old - lr * scale * exact
            most = (lr * scale * (bound + 3.9 ** 5 * 2.0 ** -23) + 3 * 2.0 ** -24 * (old.norm() + lr * scale * exact.norm())
                    + plain.STORED[DTYPES[theta]] * want.norm())
            off = (plain.view(after, *at)[w].double() - want).norm()
            assert off <= most, f"{m[1]}x{m[2]}: off by {off:.3g}, at most {most:.3g}"


@pytest.mark.parametrize("eps", [0.0, 1e-7])
@pytest.mark.parametrize("products", PRODUCTS)
@pytest.mark.parametrize("name", ["64", "64 in parts", "128", "256 at odd places"])
def test_zeros_and_bad_numbers_stay_in_their_matrix(name, products, eps):
    matrices, stride, W, *_ = path(name)
    x = filled(matrices, W, stride, torch.float32, seed=51).cuda()
    plan = nl.MuonPlan(matrices, stride, W)

    def run(into):
        out = torch.zeros((W, stride), device="cuda")
        nl.orthogonalize(plan, into, nl.F32, out, nl.F32, eps=eps, products=PRODUCTS[products])
        return out

    clean, bad = run(x), x.clone()
    first, last = matrices[0], matrices[-1]
    plain.view(bad, *first[:4])[0].zero_()
    plain.view(bad, *last[:4])[1, last[1] - 1, 3] = float("nan")
    spoiled = {(0, 0): "zero", (len(matrices) - 1, 1): "nan"}
    if W > 2:
        plain.view(bad, *first[:4])[2, first[1] - 1, first[2] - 1] = float("inf")
        plain.view(bad, *last[:4])[W - 1, 0, 0] = float("-inf")
        spoiled |= {(0, 2): "nan", (len(matrices) - 1, W - 1): "nan"}
    got, after = run(bad), run(x)
    for k, m in enumerate(matrices):
        for w in range(W):
            part = plain.view(got, *m[:4])[w]
            kind = spoiled.get((k, w))
            if kind == "zero":
                assert (part == 0).all()
            elif kind == "nan":
                assert part.isnan().all()
            else:
                assert same_bits(part, plain.view(clean, *m[:4])[w])
    # what the workspace holds of them does not reach the next call
    assert same_bits(after, clean)


@pytest.mark.parametrize("name", ["64", "64 in parts", "128"])
def test_sizes_of_numbers_do_not_matter(name):
    """Numbers whose squares leave binary32's range, either way."""
    matrices, stride, W, *_ = path(name)
    x = everywhere(matrices, W, stride, torch.bfloat16, 31).float()
    plan = nl.MuonPlan(matrices, stride, W)
    for factor in (2.0 ** -100, 2.0 ** 100):
        got = torch.zeros((W, stride), device="cuda")
        nl.orthogonalize(plan, (x * factor).cuda(), nl.F32, got, nl.F32, eps=0.0)
        alike(got)
        row = got[:1].cpu()
        # an eps of 1e-7 beside norms above 0.08 is 1.3e-6 of them, a common factor that the steps multiply by at most ten
        for m, (exact, bound) in zip(matrices, bounds(name, "x", "pairs")):
            assert (plain.view(row, *m[:4])[0].double() - exact).norm().item() <= bound + 10 * 1.3e-6 * exact.norm().item()


def test_offsets_beyond_32_bits():
    """Matrices more than 2^32 bytes and 2^31 elements from the array's start, updated in place."""
    stride, W = 1 << 30, 3
    at = stride - 260 * 516 - 4
    matrices = [(at, 260, 516, 516, 1.0), (12, 129, 300, 300, 1.0)]
    place = matrices[0][:4]
    small = filled([(0, 260, 516, 516, 1.0)], W, 260 * 516 + 48, torch.bfloat16, seed=61)
    here = plain.view(small, 0, 260, 516, 516)
    x = torch.zeros((W, stride), dtype=torch.bfloat16, device="cuda")
    plain.view(x, *place).copy_(here)
    plan = nl.MuonPlan(matrices, stride, W)
    got = torch.zeros((W, stride), dtype=torch.bfloat16, device="cuda")
    nl.orthogonalize(plan, x, nl.BF16, got, nl.BF16)
    results = plain.view(got, *place).cpu()
    for w in range(W):
        exact, bound = plain.newton_schulz_bound(here[w].double(), "f16", torch.bfloat16)
        assert (results[w].double() - exact).norm().item() <= bound
    # the momentum is what was orthogonalised, and the step of weights of zero the result
    momentum = torch.zeros((W, stride), device="cuda")
    theta = got.zero_()
    nl.muon_step(plan, theta, nl.BF16, x, nl.BF16, momentum, (1.0, 0.9, 0.0), nesterov=False)
    assert torch.equal(plain.view(momentum, *place).cpu(), here.float())
    assert same_bits(-plain.view(theta, *place).cpu(), results)
    assert (plain.view(theta, *matrices[1][:4]) == 0).all().item()


@pytest.mark.parametrize("name", ["64", "64 in parts", "128"])
def test_graph_of_an_update(name):
    matrices, stride, W, *_ = path(name)
    x = everywhere(matrices, W, stride, torch.float32, 71).nan_to_num().cuda()
    plan = nl.MuonPlan(matrices, stride, W)
    theta, moved = torch.zeros((W, stride), device="cuda"), torch.zeros((W, stride), device="cuda")
    e_theta, e_moved = theta.clone(), moved.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nl.muon_step(plan, theta, nl.F32, x, nl.F32, moved, (0.1, 0.9, 0.1))
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        nl.muon_step(plan, e_theta, nl.F32, x, nl.F32, e_moved, (0.1, 0.9, 0.1))
        assert same_bits(theta.cpu(), e_theta.cpu()) and same_bits(moved.cpu(), e_moved.cpu())


def test_small_matrices_round_their_first_x_once():
    """One step of 2 x^5, whose slope is five times itself: X_0 is off by one rounding, 2^-11, and X and the result's store by
    another. The number and the row's length are such that two roundings of X_0 go the same way (to 0.0019 together)."""
    n, w = 989, 1.0004663467407227
    signs = torch.randint(0, 2, (1, n), generator=torch.Generator().manual_seed(81)) * 2.0 - 1.0
    x = torch.zeros((1, 1024))
    x[:, :n] = signs * w
    plan = nl.MuonPlan([(0, 1, n), (1023, 1, 1)], 1024, 1)
    got = torch.zeros((1, 1024), device="cuda")
    nl.orthogonalize(plan, x.cuda(), nl.F32, got, nl.F32, coefficients=((0.0, 0.0, 2.0),), eps=0.0, products=nl.PRODUCTS_F16)
    want = 2.0 * signs.double() / n ** 0.5
    off = (got[:, :n].cpu().double() / want - 1.0).abs().max().item()
    assert off <= 6 * 2.0 ** -11 * 1.01, f"{off:.5f}"


@pytest.mark.parametrize("eps", [0.0, 1e-7])
def test_bad_numbers_of_small_matrices_in_binary16(eps):
    matrices, stride = layout([(70, 70), (9, 200), (200, 9), (64, 64)], gap=4)
    x = filled(matrices, 3, stride, torch.float32, seed=82).cuda()
    plan = nl.MuonPlan(matrices, stride, 3)

    def run(into):
        out = torch.zeros((3, stride), device="cuda")
        nl.orthogonalize(plan, into, nl.F32, out, nl.F32, eps=eps, products=nl.PRODUCTS_F16)
        return out

    clean, bad = run(x), x.clone()
    plain.view(bad, *matrices[0][:4])[1].zero_()
    plain.view(bad, *matrices[1][:4])[0, 8, 199] = float("inf")
    plain.view(bad, *matrices[2][:4])[1, 0, 0] = float("-inf")
    plain.view(bad, *matrices[3][:4])[2, 63, 3] = float("nan")
    bad_rows = plain.view(bad, *matrices[3][:4])[0]
    bad_rows.zero_()
    bad_rows[5, 7] = float("inf")                        # everything else is zero
    got = run(bad)
    for k, m in enumerate(matrices):
        for w in range(3):
            part = plain.view(got, *m[:4])[w]
            if (k, w) == (0, 1):
                assert (part == 0).all()
            elif (k, w) in ((1, 0), (2, 1), (3, 2), (3, 0)):
                assert part.isnan().all()
            else:
                assert same_bits(part, plain.view(clean, *m[:4])[w])
    assert same_bits(run(x), clean)


def test_sizes_of_numbers_do_not_matter_to_small_matrices_in_binary16():
    matrices, stride = layout([(30, 70), (64, 600)])
    x = filled(matrices, 1, stride, torch.float32, seed=83)
    plan = nl.MuonPlan(matrices, stride, 1)
    for factor in (1.0, 2.0 ** -100, 2.0 ** 100):
        got = torch.zeros((1, stride), device="cuda")
        nl.orthogonalize(plan, (x * factor).cuda(), nl.F32, got, nl.F32, eps=0.0, products=nl.PRODUCTS_F16)
        for m in matrices:
            exact, bound = plain.newton_schulz_bound(plain.view(x, *m[:4])[0].double(), "f16", torch.float32, eps=0.0)
            assert (plain.view(got.cpu(), *m[:4])[0].double() - exact).norm().item() <= bound
