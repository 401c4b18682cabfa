"""Embedding lookup and gradient at the ends of what a plan takes."""
import pytest
import torch

from test_gpu_embedding import same_bits

pytestmark = pytest.mark.gpu
nl = pytest.importorskip("paper_2506_10911_amd")


def test_lookup_of_more_than_2_28_tokens():
    """More threads than one dimension of a launch holds."""
    W, T, vocab = 3, (1 << 28) // 3 + 5, 7
    table = torch.randn((W, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    tokens = torch.arange(W * T, dtype=torch.int32, device="cuda").remainder_(vocab + 1).view(W, T)
    got = torch.full((W, T, 1), 9.0, dtype=torch.bfloat16, device="cuda")
    nl.embed_lookup(nl.EmbeddingPlan(3, vocab, 1, 64, W, T), table, nl.BF16, tokens, nl.I32, T, 0.5, got, nl.BF16)
    for w in range(W):
        rows = torch.cat([table[w, 3:3 + vocab].float() * 0.5, torch.zeros(1, device="cuda")]).to(torch.bfloat16)
        for at in range(0, T, 1 << 24):
            part = slice(at, at + (1 << 24))
            assert same_bits(got[w, part, 0], rows[tokens[w, part].long()])


def test_as_many_workers_as_there_may_be():
    W, T, vocab, width = 65536, 3, 5, 4
    tables = torch.randn((W, 64), generator=torch.Generator().manual_seed(2))
    tokens = torch.randint(-1, vocab, (W, T), generator=torch.Generator().manual_seed(3))
    there = tokens >= 0
    plan = nl.EmbeddingPlan(8, vocab, width, 64, W, T)
    got = torch.empty((W, T, width), device="cuda")
    nl.embed_lookup(plan, tables.cuda(), nl.F32, tokens.cuda(), nl.I64, T, 2.0, got, nl.F32)
    rows = tables[:, 8:8 + vocab * width].view(W, vocab, width)
    want = rows[torch.arange(W)[:, None], tokens.clamp(min=0)] * 2.0 * there[..., None]
    assert torch.equal(got.cpu(), want)
    # whole numbers: their sums are exact
    dout = torch.randint(-8, 9, (W, T, width), generator=torch.Generator().manual_seed(4)).float()
    grad = torch.full((W, 64), 3.0, device="cuda")
    nl.embed_gradient(plan, dout.cuda(), nl.F32, tokens.cuda(), nl.I64, T, 1.0, grad, nl.F32)
    sums = torch.zeros((W * vocab, width)).index_add_(0, (tokens + vocab * torch.arange(W)[:, None])[there], dout[there])
    grad = grad.cpu()
    assert torch.equal(grad[:, 8:8 + vocab * width], sums.view(W, vocab * width))
    assert (grad[:, :8] == 3).all() and (grad[:, 8 + vocab * width:] == 3).all()


def test_the_widest_row_at_an_odd_place():
    width, T = 1 << 24, 40
    stride = 2 * width + 64
    plan = nl.EmbeddingPlan(1, 2, width, stride, 1, T)
    gen = torch.Generator(device="cuda").manual_seed(5)
    dout = torch.randint(-8, 9, (1, T, width), generator=gen, device="cuda", dtype=torch.int8).to(torch.bfloat16)
    tokens = torch.arange(T, dtype=torch.int32, device="cuda").div(39, rounding_mode="floor")[None]      # 39 of token 0, one of 1
    grad = torch.full((1, stride), 3.0, device="cuda")
    nl.embed_gradient(plan, dout, nl.BF16, tokens, nl.I32, T, 1.0, grad, nl.F32)
    assert torch.equal(grad[0, 1:1 + width], dout[0, :39].sum(0, dtype=torch.float32))
    assert torch.equal(grad[0, 1 + width:1 + 2 * width], dout[0, 39].float())
    assert grad[0, 0] == 3 and (grad[0, 1 + 2 * width:] == 3).all()
