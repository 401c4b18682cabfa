"""Embedding lookup and its gradient on the GPU, against plain references."""
import pytest
import torch

import inner_plain as plain

pytestmark = pytest.mark.gpu
nl = pytest.importorskip("paper_2506_10911_amd")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IDS = {"i32": torch.int32, "i64": torch.int64}


def code(dtype):
    return {torch.bfloat16: nl.BF16, torch.float32: nl.F32, torch.int32: nl.I32, torch.int64: nl.I64}[dtype]


def arena(W, vocab, width, offset, dtype, seed=0):
    """An array whose rows hold a table at `offset`, NaN around it, and a view of the tables."""
    stride = -(-(offset + vocab * width + 5) // 64) * 64
    a = torch.full((W, stride), float("nan"))
    a[:, offset:offset + vocab * width] = torch.randn((W, vocab * width), generator=torch.Generator().manual_seed(seed))
    return a.to(dtype), stride


def tables(a, vocab, width, offset):
    return a[:, offset:offset + vocab * width].unflatten(1, (vocab, width))


def draw_tokens(W, T, vocab, ids, kind="mixed", seed=1):
    gen = torch.Generator().manual_seed(seed)
    if kind == "one":
        return torch.full((W, T), vocab - 1).to(ids)
    if kind == "none":
        return torch.full((W, T), -1).to(ids)
    few = (torch.rand((W, T), generator=gen) ** 4 * vocab).long().clamp_(max=vocab - 1)       # a few come up often
    if kind == "mixed":
        few[torch.rand((W, T), generator=gen) < 0.1] = -1
        few[torch.rand((W, T), generator=gen) < 0.05] = vocab
    return few.to(ids)


def same_bits(a, b):
    kind = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


SIZES = [  # W, T, vocab, width, offset
    (1, 1, 1, 1, 0), (2, 5, 3, 7, 1), (3, 64, 100, 64, 0), (1, 33, 50, 129, 64), (2, 100, 1000, 260, 4), (4, 2049, 300, 48, 0),
    (2, 700, 65, 1028, 8), (1, 300, 20, 2100, 2),
]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("table", ["f32", "bf16"])
@pytest.mark.parametrize("ids", ["i32", "i64"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_lookup(size, ids, table, out):
    W, T, vocab, width, offset = size
    a, stride = arena(W, vocab, width, offset, DTYPES[table])
    tokens = draw_tokens(W, T, vocab, IDS[ids])
    plan = nl.EmbeddingPlan(offset, vocab, width, stride, W, T)
    got = torch.full((W, T, width), 9.0, dtype=DTYPES[out], device="cuda")
    nl.embed_lookup(plan, a.cuda(), code(a.dtype), tokens.cuda(), code(tokens.dtype), T, 1.7, got, code(got.dtype))
    assert same_bits(got.cpu(), plain.lookup(tables(a, vocab, width, offset), tokens, 1.7, DTYPES[out]))


def run_gradient(plan, dout, tokens, scale, grad, accumulate, stream=None):
    nl.embed_gradient(plan, dout, code(dout.dtype), tokens, code(tokens.dtype), tokens.shape[1], scale, grad, code(grad.dtype),
                      accumulate=accumulate, stream=stream)


def check_gradient(size, ids, into, out, accumulate, kind, scale=0.6):
    W, T, vocab, width, offset = size
    a, stride = arena(W, vocab, width, offset, DTYPES[out])
    dout = torch.randn((W, T, width), generator=torch.Generator().manual_seed(2)).to(DTYPES[into])
    tokens = draw_tokens(W, T, vocab, IDS[ids], kind)
    plan = nl.EmbeddingPlan(offset, vocab, width, stride, W, T)
    got = a.cuda()
    run_gradient(plan, dout.cuda(), tokens.cuda(), scale, got, accumulate)
    again = a.cuda()
    run_gradient(plan, dout.cuda(), tokens.cuda(), scale, again, accumulate)
    got, again = got.cpu(), again.cpu()
    assert same_bits(got, again)
    want, bound = plain.gradient(dout, tokens, scale, tables(a, vocab, width, offset), accumulate)
    mine = tables(got, vocab, width, offset).double()
    assert ((mine - want).abs() <= bound).all(), ((mine - want).abs() - bound).max()
    rest, before = got.clone(), a.clone()
    tables(rest, vocab, width, offset).zero_()
    tables(before, vocab, width, offset).zero_()
    assert same_bits(rest, before)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("into,out", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradient(size, into, out, accumulate):
    check_gradient(size, "i64" if size[0] % 2 else "i32", into, out, accumulate, "mixed")


@pytest.mark.parametrize("kind", ["one", "none", "few"])
@pytest.mark.parametrize("T", [1, 31, 32, 33, 64, 65, 2048, 2049, 5000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_long_and_missing_rows(T, kind, accumulate):
    """One token at every position (a sum over all chunks), none at all, and lengths about a chunk's and a sorted list's."""
    check_gradient((2, T, 70, 20, 0), "i32", "f32", "f32", accumulate, kind)


@pytest.mark.parametrize("T,vocab", [(40000, 200), (33000, 2), (70000, 5000)])
def test_gradient_of_many_tokens(T, vocab):
    """More sorted lists than one merge joins."""
    check_gradient((1, T, vocab, 8, 0), "i64", "f32", "f32", False, "mixed")


def test_gradient_of_a_vocabulary_beyond_21_bits():
    """Tokens that need more bits than the short sort keys have."""
    check_gradient((1, 3000, (1 << 21) + 77, 1, 0), "i64", "f32", "f32", False, "mixed")


def test_no_tokens():
    a, stride = arena(2, 10, 6, 0, torch.float32)
    plan = nl.EmbeddingPlan(0, 10, 6, stride, 2, 0)
    tokens, rows = torch.zeros((2, 0), dtype=torch.int64, device="cuda"), torch.zeros((2, 0, 6), device="cuda")
    got = a.cuda()
    nl.embed_lookup(plan, got, nl.F32, tokens, nl.I64, 0, 1.0, rows, nl.F32)
    run_gradient(plan, rows, tokens, 1.0, got, True)
    assert same_bits(got.cpu(), a)
    run_gradient(plan, rows, tokens, 1.0, got, False)
    assert (tables(got.cpu(), 10, 6, 0) == 0).all()


def test_fewer_tokens_than_the_plan_takes():
    W, vocab, width = 2, 40, 12
    a, stride = arena(W, vocab, width, 0, torch.float32)
    plan = nl.EmbeddingPlan(0, vocab, width, stride, W, 5000)
    for T in (4100, 3, 2500):
        dout = torch.randn((W, T, width), generator=torch.Generator().manual_seed(T))
        tokens = draw_tokens(W, T, vocab, torch.int32, seed=T)
        got = a.cuda()
        run_gradient(plan, dout.cuda(), tokens.cuda(), 1.0, got, False)
        want, bound = plain.gradient(dout, tokens, 1.0, tables(a, vocab, width, 0), False)
        assert ((tables(got.cpu(), vocab, width, 0).double() - want).abs() <= bound).all()


def test_tokens_that_are_no_rows():
    """Ids that would be rows if they were cut to 32 bits."""
    W, vocab, width = 1, 10, 4
    a, stride = arena(W, vocab, width, 0, torch.float32)
    tokens = torch.tensor([[0, 1 << 32, (1 << 32) + 3, -1, -(1 << 40), vocab, (1 << 63) - 1, -(1 << 63), 9]])
    plan = nl.EmbeddingPlan(0, vocab, width, stride, W, 9)
    got = torch.full((W, 9, width), 5.0, device="cuda")
    nl.embed_lookup(plan, a.cuda(), nl.F32, tokens.cuda(), nl.I64, 9, 1.0, got, nl.F32)
    assert same_bits(got.cpu(), plain.lookup(tables(a, vocab, width, 0), tokens, 1.0, torch.float32))
    grad = a.cuda()
    run_gradient(plan, torch.ones((W, 9, width), device="cuda"), tokens.cuda(), 2.0, grad, False)
    want = torch.zeros((W, vocab, width))
    want[0, [0, 9]] = 2.0
    assert torch.equal(tables(grad.cpu(), vocab, width, 0), want)


def test_bad_numbers_stay_in_their_row():
    W, T, vocab, width = 1, 200, 20, 8
    a, stride = arena(W, vocab, width, 0, torch.float32)
    tokens = draw_tokens(W, T, vocab, torch.int64)
    dout = torch.randn((W, T, width), generator=torch.Generator().manual_seed(5))
    hit, padding = int(tokens[0][(tokens[0] >= 0) & (tokens[0] < vocab)][7]), int((tokens[0] < 0).nonzero()[0])
    where = int((tokens[0] == hit).nonzero()[0])
    dout[0, where, 3] = float("nan")
    dout[0, padding] = float("inf")               # belongs to no row
    got = a.cuda()
    run_gradient(nl.EmbeddingPlan(0, vocab, width, stride, W, T), dout.cuda(), tokens.cuda(), 1.0, got, False)
    nan = tables(got.cpu(), vocab, width, 0).isnan()
    assert nan.nonzero().tolist() == [[0, hit, 3]]


def test_gradient_is_the_lookups():
    """Differences of a loss L = <lookup(table), dout> along random directions: L is linear, so one difference is its gradient."""
    W, T, vocab, width, scale = 2, 300, 50, 12, 1.25
    a, stride = arena(W, vocab, width, 0, torch.float32)
    tokens = draw_tokens(W, T, vocab, torch.int64)
    dout = torch.randn((W, T, width), generator=torch.Generator().manual_seed(3))
    plan = nl.EmbeddingPlan(0, vocab, width, stride, W, T)
    grad = a.cuda()
    run_gradient(plan, dout.cuda(), tokens.cuda(), scale, grad, False)
    grad = tables(grad.cpu(), vocab, width, 0).double()

    def loss(table):
        full = torch.zeros((W, stride))
        tables(full, vocab, width, 0).copy_(table)
        out = torch.empty((W, T, width), device="cuda")
        nl.embed_lookup(plan, full.cuda(), nl.F32, tokens.cuda(), nl.I64, T, scale, out, nl.F32)
        return (out.cpu().double() * dout.double()).sum().item()

    base = torch.zeros((W, vocab, width))
    for seed in range(4):
        way = torch.randn((W, vocab, width), generator=torch.Generator().manual_seed(100 + seed))
        size = (way.double().abs() * grad.abs()).sum().item()
        # rounding of the products, and of the sums behind every gradient
        assert abs((loss(way) - loss(base)) - (way.double() * grad).sum().item()) <= 2.0 ** -24 * (2 + T) * (size + 40 * T)


def test_offsets_beyond_32_bits():
    vocab, width, T = 300, 64, 500
    stride, W = 1 << 30, 3
    offset = stride - vocab * width
    a = torch.zeros((W, stride), dtype=torch.bfloat16, device="cuda")
    table = torch.randn((W, vocab, width), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    tables(a, vocab, width, offset).copy_(table)
    tokens = draw_tokens(W, T, vocab, torch.int32)
    plan = nl.EmbeddingPlan(offset, vocab, width, stride, W, T)
    got = torch.empty((W, T, width), device="cuda")
    nl.embed_lookup(plan, a, nl.BF16, tokens.cuda(), nl.I32, T, 3.0, got, nl.F32)
    assert same_bits(got.cpu(), plain.lookup(table, tokens, 3.0, torch.float32))
    dout = torch.randn((W, T, width), generator=torch.Generator().manual_seed(7))
    run_gradient(plan, dout.cuda(), tokens.cuda(), 1.0, a, True)
    want, bound = plain.gradient(dout, tokens, 1.0, table, True)
    assert ((tables(a, vocab, width, offset).cpu().double() - want).abs() <= bound).all()


def test_other_stream_and_graph():
    W, T, vocab, width = 2, 3000, 100, 32
    a, stride = arena(W, vocab, width, 0, torch.float32)
    tokens, dout = draw_tokens(W, T, vocab, torch.int64).cuda(), torch.randn((W, T, width), device="cuda")
    plan = nl.EmbeddingPlan(0, vocab, width, stride, W, T)
    want = a.cuda()
    run_gradient(plan, dout, tokens, 1.0, want, True)
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), a.cuda()
    side.wait_stream(torch.cuda.current_stream())
    run_gradient(plan, dout, tokens, 1.0, got, True, stream=side)
    side.synchronize()
    assert same_bits(got.cpu(), want.cpu())
    grad, eager = a.cuda(), a.cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_gradient(plan, dout, tokens, 1.0, grad, True)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        run_gradient(plan, dout, tokens, 1.0, eager, True)
        assert same_bits(grad.cpu(), eager.cpu())


def test_refusals():
    vocab, width, T = 10, 8, 4
    a, stride = arena(1, vocab, width, 0, torch.float32)
    a = a.cuda()
    plan = nl.EmbeddingPlan(0, vocab, width, stride, 1, T)
    tokens, rows = torch.zeros((1, T), dtype=torch.int64, device="cuda"), torch.zeros((1, T, width), device="cuda")

    def refused(status, call, *args, **more):
        with pytest.raises(nl.NolocoError) as e:
            call(plan, *args, **more)
        assert e.value.status == status

    refused(1, nl.embed_lookup, None, nl.F32, tokens, nl.I64, T, 1.0, rows, nl.F32)
    refused(1, nl.embed_lookup, a, nl.F32, None, nl.I64, T, 1.0, rows, nl.F32)
    refused(2, nl.embed_lookup, a, nl.F32, tokens, nl.I64, T + 1, 1.0, rows, nl.F32)
    refused(2, nl.embed_lookup, a, nl.F32, tokens, nl.I64, -1, 1.0, rows, nl.F32)
    refused(2, nl.embed_lookup, a, nl.F32, tokens, nl.F32, T, 1.0, rows, nl.F32)
    refused(2, nl.embed_lookup, a, nl.I32, tokens, nl.I64, T, 1.0, rows, nl.F32)
    refused(2, nl.embed_lookup, a, nl.F32, tokens, nl.I64, T, 1.0, a, nl.F32)               # overlap
    refused(5, nl.embed_lookup, a, nl.F32, tokens.data_ptr() + 4, nl.I64, T, 1.0, rows, nl.F32)
    refused(5, nl.embed_lookup, a, nl.F32, tokens, nl.I64, T, 1.0, rows.data_ptr() + 4, nl.F32)
    refused(5, nl.embed_gradient, rows, nl.F32, tokens, nl.I64, T, 1.0, a.data_ptr() + 16, nl.F32)
    refused(2, nl.embed_gradient, rows, nl.F32, tokens, nl.I64, T, 1.0, a, nl.F32, accumulate=2)
