"""Orthogonalisation and updates of matrices that go through a launch for each product, on the GPU, against 64-bit references."""
import pytest
import torch

import inner_plain as plain
from test_gpu_muon import code, filled, layout

pytestmark = pytest.mark.gpu
nl = pytest.importorskip("paper_2506_10911_amd")

# One binary16 a number rounds X_0 and four more X by up to 2^-11 of every number, a third of its square on average: at worst
# sqrt(5 / 3) 2^-11 = 0.00063 of the norm. What A and P lose beside their diagonals comes to it.
F16_OFF = 2.0 ** -10

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
