"""Newton-Schulz orthogonalisation and the update built on it, on the GPU, against 64-bit references."""
import pytest
import torch

import inner_plain as plain

pytestmark = pytest.mark.gpu
nl = pytest.importorskip("paper_2506_10911_amd")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def code(dtype):
    return nl.BF16 if dtype == torch.bfloat16 else nl.F32


def layout(shapes, gap=3, first=0):
    """(offset, rows, cols, row_stride, scale) of matrices one after the other, `gap` elements of nobody's between them."""
    found, at = [], first
    for i, shape in enumerate(shapes):
        rows, cols = shape[:2]
        stride = shape[2] if len(shape) > 2 else cols
        found.append((at, rows, cols, stride, 1.0 + 0.25 * i))
        at += (rows - 1) * stride + cols + gap if rows and cols else 0
    return found, max(-(-at // 64) * 64, 64)


def filled(matrices, W, stride, dtype, seed=0, spread=0.0):
    """Noise in the matrices, NaN elsewhere (nobody's elements are not to be read)."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.full((W, stride), float("nan"))
    for offset, rows, cols, row_stride, _ in matrices:
        if rows and cols:
            m = torch.randn((W, rows, cols), generator=gen) * 1e-3
            if spread:                          # a few strong directions over the noise
                m += spread * torch.randn((W, rows, 2), generator=gen) @ torch.randn((W, 2, cols), generator=gen)
            plain.view(x, offset, rows, cols, row_stride).copy_(m)
    return x.to(dtype)


def owned(matrices, W, stride):
    mask = torch.zeros((W, stride), dtype=torch.bool)
    for offset, rows, cols, row_stride, _ in matrices:
        plain.view(mask, offset, rows, cols, row_stride).fill_(True)
    return mask


def same_bits(a, b):
    kind = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


def check(matrices, got, x, products, what=""):
    for offset, rows, cols, row_stride, _ in matrices:
        for w in range(x.shape[0]):
            u = plain.view(x[w:w + 1], offset, rows, cols, row_stride)[0].double()
            exact, bound = plain.newton_schulz_bound(u, products, got.dtype)
            off = (plain.view(got[w:w + 1], offset, rows, cols, row_stride)[0].double() - exact).norm().item()
            assert off <= bound, f"{what} {rows}x{cols} of worker {w}: off by {off:.3g}, at most {bound:.3g}"


SHAPES = [
    [(1, 1)], [(1, 300), (300, 1)], [(2, 3), (3, 2), (5, 5)], [(64, 64)], [(65, 63), (63, 65)], [(32, 200)],
    [(128, 96), (96, 128), (128, 129)], [(17, 1000), (1000, 17)], [(250, 260, 300)], [(40, 50, 51), (50, 40, 77)],
    [(260, 516)], [(516, 260)],
]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("into", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: "+".join("x".join(map(str, v)) for v in s))
def test_orthogonalize(shapes, into, out):
    matrices, stride = layout(shapes)
    x = filled(matrices, 2, stride, DTYPES[into])
    got = torch.full((2, stride), 7.0, dtype=DTYPES[out], device="cuda")
    plan = nl.MuonPlan(matrices, stride, 2)
    nl.orthogonalize(plan, x.cuda(), code(x.dtype), got, code(got.dtype))
    got = got.cpu()
    check(matrices, got, x, "pairs" if out == "f32" else "f16")
    assert (got[~owned(matrices, 2, stride)] == 7.0).all()


@pytest.mark.parametrize("rows,cols,W", [(512, 512, 24), (256, 768, 40), (768, 256, 40), (600, 600, 3), (130, 4100, 2)])
def test_large_and_many(rows, cols, W):
    """Sizes that take the large tiles, and launches of many matrices."""
    matrices, stride = layout([(rows, cols)])
    x = filled(matrices, W, stride, torch.float32, seed=3, spread=2e-3)
    plan = nl.MuonPlan(matrices, stride, W)
    for dtype, products in ((torch.bfloat16, "f16"), (torch.float32, "pairs")):
        got = torch.zeros((W, stride), dtype=dtype, device="cuda")
        nl.orthogonalize(plan, x.cuda(), nl.F32, got, code(dtype))
        got = got.cpu()
        some = [0, W // 2, W - 1]
        check(matrices, got[some], x[some], products)


@pytest.mark.parametrize("count", [40, 70])
def test_more_shapes_than_a_launch_takes(count):
    shapes = [(3 + i, 70 + 2 * i) for i in range(count)]
    matrices, stride = layout(shapes, gap=1)
    x = filled(matrices, 1, stride, torch.float32)
    plan = nl.MuonPlan(matrices, stride, 1)
    got = torch.zeros((1, stride), device="cuda")
    nl.orthogonalize(plan, x.cuda(), nl.F32, got, nl.F32)
    check(matrices, got.cpu(), x, "pairs")


def test_products_can_be_chosen():
    matrices, stride = layout([(90, 150)])
    x = filled(matrices, 1, stride, torch.float32)
    plan = nl.MuonPlan(matrices, stride, 1)
    got = torch.zeros((1, stride), device="cuda")
    nl.orthogonalize(plan, x.cuda(), nl.F32, got, nl.F32, products=nl.PRODUCTS_F16)
    check(matrices, got.cpu(), x, "f16")
    u = plain.view(x, *matrices[0][:4])[0].double()
    exact, tight = plain.newton_schulz_bound(u, "pairs", torch.float32)
    assert (plain.view(got.cpu(), *matrices[0][:4])[0].double() - exact).norm() > tight     # another product was taken
    half = torch.zeros((1, stride), dtype=torch.bfloat16, device="cuda")
    nl.orthogonalize(plan, x.cuda(), nl.F32, half, nl.BF16, products=nl.PRODUCTS_PAIRS)
    check(matrices, half.cpu(), x, "pairs")


@pytest.mark.parametrize("coefficients", [((1.5, -0.5, 0.0),) * 3, ((8.0, -22.0, 15.0), (1.9, -0.6, 0.05), (1.9, -1.3, 0.4)), ((2.0, -1.5, 0.5),)])
def test_other_coefficients(coefficients):
    matrices, stride = layout([(50, 130), (130, 50)])
    x = filled(matrices, 1, stride, torch.float32, seed=5)
    plan = nl.MuonPlan(matrices, stride, 1)
    got = torch.zeros((1, stride), device="cuda")
    nl.orthogonalize(plan, x.cuda(), nl.F32, got, nl.F32, coefficients=coefficients, eps=1e-3)
    for offset, rows, cols, row_stride, _ in matrices:
        u = plain.view(x, offset, rows, cols, row_stride)[0].double()
        exact, bound = plain.newton_schulz_bound(u, "pairs", torch.float32, coefficients, 1e-3)
        assert (plain.view(got.cpu(), offset, rows, cols, row_stride)[0].double() - exact).norm().item() <= bound


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("products", ["f16", "pairs"])
@pytest.mark.parametrize("shapes", [[(1, 1), (1, 70)], [(16, 64)], [(31, 2), (2, 31)], [(64, 64)], [(63, 97), (97, 63)], [(32, 200)], [(33, 300)]],
                         ids=lambda s: "+".join("x".join(map(str, v)) for v in s))
def test_small_matrices(shapes, products, out):
    matrices, stride = layout(shapes)
    x = filled(matrices, 3, stride, torch.float32, seed=9)
    plan = nl.MuonPlan(matrices, stride, 3)
    got = {}
    for kind in (nl.PRODUCTS_F16, nl.PRODUCTS_PAIRS, nl.PRODUCTS_AUTO):
        got[kind] = torch.zeros((3, stride), dtype=DTYPES[out], device="cuda")
        nl.orthogonalize(plan, x.cuda(), nl.F32, got[kind], code(DTYPES[out]), products=kind)
    check(matrices, got[nl.PRODUCTS_F16 if products == "f16" else nl.PRODUCTS_PAIRS].cpu(), x, products)
    assert same_bits(got[nl.PRODUCTS_AUTO], got[nl.PRODUCTS_PAIRS])


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", [[(1, 9001)], [(5000, 3)], [(70, 3201)], [(3500, 130, 137)], [(129, 3077)], [(40, 4100), (1500, 90), (200, 300)]],
                         ids=lambda s: "+".join("x".join(map(str, v)) for v in s))
def test_few_long_rows(shapes, out):
    matrices, stride = layout(shapes)
    x = filled(matrices, 2, stride, torch.float32, seed=12)
    plan = nl.MuonPlan(matrices, stride, 2)
    for kind, products in ((nl.PRODUCTS_F16, "f16"), (nl.PRODUCTS_PAIRS, "pairs")):
        got = [torch.full((2, stride), 3.0, dtype=DTYPES[out], device="cuda") for _ in range(2)]
        for g in got:
            nl.orthogonalize(plan, x.cuda(), nl.F32, g, code(DTYPES[out]), products=kind)
        check(matrices, got[0].cpu(), x, products)
        assert same_bits(*got)
        assert (got[0].cpu()[~owned(matrices, 2, stride)] == 3.0).all()


def test_one_large_matrix_takes_bf16_results_to_one_number():
    matrices, stride = layout([(16, 64), (128, 128)])
    x = filled(matrices, 1, stride, torch.bfloat16, seed=10)
    plan = nl.MuonPlan(matrices, stride, 1)
    got = [torch.zeros((1, stride), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    nl.orthogonalize(plan, x.cuda(), nl.BF16, got[0], nl.BF16)
    nl.orthogonalize(plan, x.cuda(), nl.BF16, got[1], nl.BF16, products=nl.PRODUCTS_F16)
    assert same_bits(*got)


def test_sizes_of_numbers_do_not_matter():
    """Gradients whose squares leave binary32's range, either way."""
    matrices, stride = layout([(30, 70)])
    x = filled(matrices, 1, stride, torch.float32)
    plan = nl.MuonPlan(matrices, stride, 1)
    for factor in (1.0, 2.0 ** -100, 2.0 ** 100):
        scaled = x * factor
        got = torch.zeros((1, stride), device="cuda")
        nl.orthogonalize(plan, scaled.cuda(), nl.F32, got, nl.F32, eps=0.0)
        u = plain.view(scaled, *matrices[0][:4])[0].double()
        exact, bound = plain.newton_schulz_bound(u, "pairs", torch.float32, eps=0.0)
        assert (plain.view(got.cpu(), *matrices[0][:4])[0].double() - exact).norm().item() <= bound


@pytest.mark.parametrize("eps", [0.0, 1e-7])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_zeros_and_bad_numbers_stay_in_their_matrix(out, eps):
    matrices, stride = layout([(70, 70), (70, 70), (9, 200), (200, 9)])
    x = filled(matrices, 3, stride, torch.float32)
    plan = nl.MuonPlan(matrices, stride, 3)
    clean = torch.zeros((3, stride), dtype=DTYPES[out], device="cuda")
    nl.orthogonalize(plan, x.cuda(), nl.F32, clean, code(clean.dtype), eps=eps)
    bad = x.clone()
    plain.view(bad, *matrices[0][:4])[1].zero_()
    plain.view(bad, *matrices[1][:4])[2, 69, 3] = float("nan")
    plain.view(bad, *matrices[2][:4])[0, 8, 199] = float("inf")
    plain.view(bad, *matrices[3][:4])[1, 0, 0] = float("-inf")
    got = torch.zeros((3, stride), dtype=DTYPES[out], device="cuda")
    nl.orthogonalize(plan, bad.cuda(), nl.F32, got, code(got.dtype), eps=eps)
    # and again: what the workspace holds of them does not reach the next call
    after = torch.zeros((3, stride), dtype=DTYPES[out], device="cuda")
    nl.orthogonalize(plan, x.cuda(), nl.F32, after, code(after.dtype), eps=eps)
    got, clean = got.cpu(), clean.cpu()
    for k, m in enumerate(matrices):
        for w in range(3):
            part, want = plain.view(got, *m[:4])[w], plain.view(clean, *m[:4])[w]
            if (k, w) == (0, 1):
                assert (part == 0).all()
            elif (k, w) in ((1, 2), (2, 0), (3, 1)):
                assert part.isnan().all()
            else:
                assert same_bits(part, want)
    assert same_bits(after.cpu(), clean)


def test_batches_and_repeats_do_not_change_a_bit():
    matrices, stride = layout([(100, 130), (70, 40), (64, 300), (300, 300)])
    x = filled(matrices, 5, stride, torch.float32).cuda()
    results = []
    for room in (0, 1, 3 << 20):
        plan = nl.MuonPlan(matrices, stride, 5, room)
        if room == 1:
            assert plan.info()["f32_batches"] > 1
        for _ in range(2):
            for dtype in (torch.float32, torch.bfloat16):
                got = torch.zeros((5, stride), dtype=dtype, device="cuda")
                nl.orthogonalize(plan, x, nl.F32, got, code(dtype))
                results.append(got.cpu())
    for got in results:
        assert same_bits(got, results[0] if got.dtype == torch.float32 else results[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(dtype):
    matrices, stride = layout([(100, 130), (130, 100, 111), (33, 33)])
    x = filled(matrices, 3, stride, DTYPES[dtype]).cuda()
    x[x.isnan()] = 3.0
    plan = nl.MuonPlan(matrices, stride, 3, 1)           # several batches
    got = torch.full_like(x, 3.0)
    nl.orthogonalize(plan, x, code(x.dtype), got, code(x.dtype))
    nl.orthogonalize(plan, x, code(x.dtype), x, code(x.dtype))
    assert same_bits(x.cpu(), got.cpu())


@pytest.mark.parametrize("first", [0, 1, 2, 5])
@pytest.mark.parametrize("theta,grad", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("nesterov", [False, True])
def test_muon_step(theta, grad, nesterov, first):
    """Three updates against the formula in 64 bits, in which the kernel's own momentum and weights of the step before stand."""
    matrices, stride = layout([(48, 80), (80, 48, 90), (1, 77), (65, 65)], gap=first or 4, first=first)
    W, lr, mu, decay = 2, 0.05, 0.9, 0.2
    weights = filled(matrices, W, stride, torch.float32, seed=1).mul(20).to(DTYPES[theta])
    moved = filled(matrices, W, stride, torch.float32, seed=2)
    plan = nl.MuonPlan(matrices, stride, W)
    d_theta, d_moved = weights.cuda(), moved.cuda()
    mask = owned(matrices, W, stride)
    for step in range(3):
        g = filled(matrices, W, stride, DTYPES[grad], seed=10 + step)
        before, moved_before = d_theta.cpu(), d_moved.cpu()
        nl.muon_step(plan, d_theta, code(d_theta.dtype), g.cuda(), code(g.dtype), d_moved, (lr, mu, decay), nesterov=nesterov)
        after, moved_after = d_theta.cpu(), d_moved.cpu()
        assert same_bits(torch.where(mask, torch.zeros_like(after), after), torch.where(mask, torch.zeros_like(before), before))
        for offset, rows, cols, row_stride, scale in matrices:
            at = (offset, rows, cols, row_stride)
            for w in range(W):
                gw, mw = plain.view(g, *at)[w].double(), plain.view(moved_before, *at)[w].double()
                mom = mu * mw + gw
                off = (plain.view(moved_after, *at)[w].double() - mom).abs()
                assert (off <= 2.0 ** -23 * (abs(mu) * mw.abs() + mom.abs()) + 2.0 ** -24 * mw.abs()).all()
                u = gw + mu * mom if nesterov else mom
                exact, bound = plain.newton_schulz_bound(u, "pairs" if theta == "f32" else "f16", torch.float32)
                old = plain.view(before, *at)[w].double()
                want = (1 - lr * decay) * old - lr * scale * exact
                # binary32 operations on old and the step, and the weight's rounding
                bound = lr * scale * bound + (3 * 2.0 ** -24) * (old.norm() + lr * scale * exact.norm()) + plain.STORED[DTYPES[theta]] * want.norm()
                # u itself is a binary32 number: rounded, it is off by 2^-23 of itself, which the steps multiply by at most 3.9 each
                bound += lr * scale * 3.9 ** 5 * 2.0 ** -23
                assert (plain.view(after, *at)[w].double() - want).norm() <= bound


def test_no_update_leaves_the_weights():
    matrices, stride = layout([(20, 30)])
    theta = filled(matrices, 1, stride, torch.float32).cuda()
    before, moved = theta.clone(), torch.zeros((1, stride), device="cuda")
    nl.muon_step(nl.MuonPlan(matrices, stride, 1), theta, nl.F32, torch.ones((1, stride), device="cuda"), nl.F32, moved, (0.0, 0.9, 0.5))
    assert same_bits(theta.cpu(), before.cpu())
    assert (plain.view(moved.cpu(), 0, 20, 30, 30) == 1).all()


def test_offsets_beyond_32_bits():
    """Matrices more than 2^32 bytes and 2^31 elements from the array's start."""
    stride, W = 1 << 30, 3
    matrices = [(stride - 70 * 90 - 5, 70, 90, 90, 1.0), (11, 64, 64, 64, 1.0)]
    x = torch.zeros((W, stride), dtype=torch.bfloat16, device="cuda")
    small = filled([(0, 70, 90, 90, 1.0)], W, 6336, torch.float32, seed=4).to(torch.bfloat16)
    plain.view(x, *matrices[0][:4]).copy_(plain.view(small, 0, 70, 90, 90))
    plan = nl.MuonPlan(matrices, stride, W)
    nl.orthogonalize(plan, x, nl.BF16, x, nl.BF16)
    got = plain.view(x, *matrices[0][:4]).cpu()
    for w in range(W):
        exact, bound = plain.newton_schulz_bound(plain.view(small, 0, 70, 90, 90)[w].double(), "f16", torch.bfloat16)
        assert (got[w].double() - exact).norm().item() <= bound
    assert (plain.view(x, *matrices[1][:4]) == 0).all().item()


def test_other_stream_and_graph():
    matrices, stride = layout([(100, 130), (64, 64)])
    x = filled(matrices, 2, stride, torch.float32).cuda()
    plan = nl.MuonPlan(matrices, stride, 2)
    want = torch.zeros((2, stride), device="cuda")
    nl.orthogonalize(plan, x, nl.F32, want, nl.F32)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = torch.zeros((2, stride), device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    nl.orthogonalize(plan, x, nl.F32, got, nl.F32, stream=side)
    side.synchronize()
    assert same_bits(got.cpu(), want.cpu())

    theta, moved = torch.zeros((2, stride), device="cuda"), torch.zeros((2, stride), device="cuda")
    e_theta, e_moved = theta.clone(), moved.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nl.muon_step(plan, theta, nl.F32, x, nl.F32, moved, (0.1, 0.9, 0.1))
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        nl.muon_step(plan, e_theta, nl.F32, x, nl.F32, e_moved, (0.1, 0.9, 0.1))
        assert same_bits(theta.cpu(), e_theta.cpu()) and same_bits(moved.cpu(), e_moved.cpu())


def test_no_matrices():
    plan = nl.MuonPlan([(0, 0, 5), (3, 4, 0)], 64, 2)
    x = torch.full((2, 64), 2.0, device="cuda")
    nl.orthogonalize(plan, x, nl.F32, x, nl.F32)
    assert (x == 2).all().item() and plan.info()["elements_per_worker"] == 0


def test_refusals_of_calls():
    matrices, stride = layout([(20, 30)])
    plan = nl.MuonPlan(matrices, stride, 1)
    x, y = torch.zeros((1, stride), device="cuda"), torch.zeros((1, stride), device="cuda")
    m = torch.zeros((1, stride), device="cuda")

    def refused(status, call, *args, **more):
        with pytest.raises(nl.NolocoError) as e:
            call(plan, *args, **more)
        assert e.value.status == status

    refused(1, nl.orthogonalize, None, nl.F32, y, nl.F32)
    refused(1, nl.orthogonalize, x, nl.F32, None, nl.F32)
    refused(2, nl.orthogonalize, x, 2, y, nl.F32)
    refused(2, nl.orthogonalize, x, nl.F32, x.data_ptr() + 256, nl.F32)             # overlap
    refused(2, nl.orthogonalize, x, nl.F32, x, nl.BF16)                             # in place, another type
    refused(5, nl.orthogonalize, x.data_ptr() + 4, nl.F32, y, nl.F32)
    refused(2, nl.orthogonalize, x, nl.F32, y, nl.F32, coefficients=())
    refused(2, nl.orthogonalize, x, nl.F32, y, nl.F32, coefficients=((1.5, float("nan"), 0.0),))
    refused(2, nl.orthogonalize, x, nl.F32, y, nl.F32, eps=-1.0)
    refused(2, nl.orthogonalize, x, nl.F32, y, nl.F32, products=3)
    refused(7, nl.orthogonalize, x, nl.F32, y, nl.F32, coefficients=((16.0, 0.0, 0.0),))
    refused(7, nl.orthogonalize, x, nl.F32, y, nl.F32, coefficients=((1.8, 0.0, 0.0),) * 2)
    refused(1, nl.muon_step, x, nl.F32, y, nl.F32, None, (0.1, 0.9, 0.0))
    refused(2, nl.muon_step, x, nl.F32, y, nl.F32, y, (0.1, 0.9, 0.0))
    refused(2, nl.muon_step, x, nl.F32, y, 7, m, (0.1, 0.9, 0.0))
    refused(5, nl.muon_step, x, nl.F32, y.data_ptr() + 2, nl.BF16, m, (0.1, 0.9, 0.0))
