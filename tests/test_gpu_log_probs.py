"""Log probabilities of tokens, entropy, alternatives and their gradient on the GPU, against the plain form in 64 bits."""
import math

import pytest
import torch

import model_plain as plain

pytestmark = pytest.mark.gpu
nl = pytest.importorskip("paper_2506_10911_amd")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IDS = {"i32": torch.int32, "i64": torch.int64}
LOWEST = torch.finfo(torch.float32).min


def code(t):
    return {torch.bfloat16: nl.BF16, torch.float32: nl.F32, torch.int32: nl.I32, torch.int64: nl.I64}[t.dtype]


def same_bits(a, b):
    kind = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


def within(got, want, bound):
    got, want = got.double(), want.double()
    fine = want.isfinite()
    assert torch.equal(got[~fine], want[~fine]), (got[~fine], want[~fine])
    off = (got - want).abs()[fine] - bound[fine]
    assert off.numel() == 0 or not (off > 0).any() and not got[fine].isnan().any(), off.max()


def draw(W, T, vocab, stride, dtype, ids, std=2.5, seed=0):
    gen = torch.Generator().manual_seed(seed)
    logits = torch.full((W, T, stride), float("nan"))
    logits[..., :vocab] = std * torch.randn((W, T, vocab), generator=gen)
    tokens = torch.randint(-1, vocab + 1, (W, T), generator=gen)          # -1 and vocab are padding
    return logits.to(dtype), tokens.to(ids)


def forward(logits, tokens, vocab, top=0, entropy=True, norms=True, max_tokens=None, max_top=None, stream=None):
    W, T, stride = logits.shape
    plan = nl.LogProbPlan(vocab, W, max_tokens or T, row_stride=stride, max_top=top if max_top is None else max_top)
    out = {"log_probs": torch.full((W, T), 9.0, device="cuda")}
    out["entropy"] = torch.full((W, T), 9.0, device="cuda") if entropy else None
    out["norms"] = torch.full((W, T), 9.0, device="cuda") if norms else None
    out["top_tokens"] = torch.full((W, T, top), -9, dtype=torch.int32, device="cuda") if top else None
    out["top_log_probs"] = torch.full((W, T, top), 9.0, device="cuda") if top else None
    nl.token_log_probs(plan, logits.cuda(), code(logits), tokens.cuda(), code(tokens), T, out["log_probs"], entropy=out["entropy"], norms=out["norms"],
                       top=top, top_tokens=out["top_tokens"], top_log_probs=out["top_log_probs"], stream=stream)
    return {k: v.cpu() for k, v in out.items() if v is not None}


def check(logits, tokens, vocab, top):
    got = forward(logits, tokens, vocab, top)
    rows = logits[..., :vocab]
    want = plain.log_probs(rows, tokens)
    for name in ("log_probs", "norms", "entropy"):
        within(got[name], *want[name])
    if top:
        order = plain.top_tokens(rows, top)
        assert torch.equal(got["top_tokens"].long(), order)
        there = order >= 0
        index = order.clamp(min=0)
        logs, bound = (t.gather(-1, index) for t in want["all"])
        within(got["top_log_probs"], torch.where(there, logs, -math.inf), torch.where(there, bound, 0.0))
    again = forward(logits, tokens, vocab, top, max_tokens=logits.shape[1] + 500, max_top=32)
    assert all(torch.equal(got[k].nan_to_num(7.0), again[k].nan_to_num(7.0)) for k in got if k != "norms") and same_bits(got["norms"], again["norms"])
    few = forward(logits, tokens, vocab, 0, entropy=False, norms=False)
    within(few["log_probs"], *want["log_probs"])           # another workgroup size may sum in another order


SIZES = [  # W, T, vocab, row_stride
    (1, 1, 1, 1), (2, 3, 2, 2), (1, 5, 7, 9), (3, 61, 129, 129), (2, 40, 1000, 1024), (1, 9, 1024, 1024), (2, 5, 1031, 1031), (1, 3, 4099, 4099),
    (2, 2, 16384, 16384), (1, 3, 16391, 16391), (1, 300, 16400, 16401), (4, 1, 50257, 50304), (1, 7, 50257, 50257), (2, 300, 5003, 5003), (1, 2, 65537, 65537),
    (1, 1, 200001, 200001), (1, 260, 66000, 66001),
]


@pytest.mark.parametrize("top", [0, 1, 5, 32])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_log_probs(size, dtype, top):
    W, T, vocab, stride = size
    logits, tokens = draw(W, T, vocab, stride, DTYPES[dtype], IDS["i32" if T % 2 else "i64"])
    check(logits, tokens, vocab, top)


@pytest.mark.parametrize("top", [0, 8])
@pytest.mark.parametrize("vocab", [40, 3000, 20011, 70001])
def test_masked_and_equal_logits(vocab, top):
    """Rows of -infinity and of the type's lowest value, whole and in part, equal logits, zeros of both signs."""
    logits, tokens = draw(1, 12, vocab, vocab, torch.float32, torch.int64, seed=3)
    row = logits[0]
    row[0] = -math.inf
    row[1, 1:] = -math.inf
    row[2, :vocab - 1] = -math.inf
    row[3, torch.arange(vocab) % 3 != 1] = -math.inf
    row[4] = LOWEST
    row[5, 5:] = LOWEST
    row[6] = 1.25
    row[7, ::2], row[7, 1::2] = 0.0, -0.0
    row[8] = torch.where(torch.arange(vocab) % 7 == 3, 4.0, -math.inf)
    row[9, vocab // 2] = 80.0
    row[10] -= 500
    row[11] += 3000
    tokens[0] = torch.tensor([0, 0, vocab - 1, 1, vocab - 1, 7, 3, 1, 3, vocab // 2, 0, -1])
    check(logits, tokens, vocab, top)


@pytest.mark.parametrize("vocab", [30, 3000, 50257, 70001])
def test_one_token_nearly_certain(vocab):
    """log(1 + rest) has the rest's digits: down to where the rest is 1e-30."""
    gaps = torch.tensor([5.0, 15.0, 30.0, 60.0])
    logits = torch.randn((1, 4, vocab), generator=torch.Generator().manual_seed(1))
    at = torch.tensor([[0, vocab - 1, vocab // 2, 1]])
    logits.scatter_(2, at[..., None], gaps[None, :, None] + math.log(vocab))
    got = forward(logits, at, vocab)
    want = plain.log_probs(logits, at)
    within(got["log_probs"], *want["log_probs"])
    # a share is off by (distance + 20) 2^-23, the sums by their additions
    limit = (60 + math.log(vocab) + 5 + 20) * 2.0 ** -23 + (vocab / 64 + 60) * plain.U
    assert ((got["log_probs"].double() / want["log_probs"][0] - 1).abs() <= limit).all()


def test_bad_numbers():
    """A NaN or +infinity makes its own row's results NaN; a NaN ranks as -infinity."""
    vocab = 5000
    logits, tokens = draw(1, 6, vocab, vocab, torch.float32, torch.int32, seed=4)
    tokens[0] = torch.tensor([1, 2, 3, 4, -1, 5])
    clean = forward(logits, tokens, vocab, 4)
    logits[0, 1, 77], logits[0, 3, 4999], logits[0, 4, 9] = math.nan, math.inf, math.nan
    got = forward(logits, tokens, vocab, 4)
    bad = torch.tensor([False, True, False, True, True, False])
    for name in ("entropy", "norms", "top_log_probs"):
        assert got[name][0, bad].isnan().all() and same_bits(got[name][0, ~bad], clean[name][0, ~bad])
    assert got["log_probs"][0, [1, 3]].isnan().all() and got["log_probs"][0, 4] == 0.0
    assert torch.equal(got["top_tokens"].long(), plain.top_tokens(logits, 4))
    only = torch.full((1, 1, 300), math.nan)
    got = forward(only, torch.zeros((1, 1), dtype=torch.int64), 300, 3)
    assert got["norms"].isnan().all() and torch.equal(got["top_tokens"][0, 0], torch.tensor([0, 1, 2], dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_alternatives_crowded_into_few_threads(dtype):
    """Large logits at a distance that puts them into the same threads, more of them than the first bound expects."""
    vocab = 65536
    place = torch.arange(vocab)
    rows = []
    for period, width in ((512, 8), (512, 16), (4096, 64), (2048, 8), (8192, 8)):
        rows.append(torch.where(place % period < width, 3.0 + (place % 1000) / 1000.0, (place % 977) / 977.0))
    logits = torch.stack(rows)[None].to(DTYPES[dtype])
    for top in (3, 32):
        check(logits, torch.zeros((1, len(rows)), dtype=torch.int64), vocab, top)


def gradient(logits, tokens, vocab, norms, dlog_probs, dentropy, entropy, dtype, in_place=False, stream=None):
    W, T, stride = logits.shape
    plan = nl.LogProbPlan(vocab, W, T, row_stride=stride)
    source = logits.cuda()
    out = source if in_place else torch.full((W, T, stride), 9.0, dtype=dtype, device="cuda")
    nl.token_log_probs_gradient(plan, source, code(logits), tokens.cuda(), code(tokens), T, norms.cuda(), dlog_probs.cuda(), out, code(out),
                                dentropy=None if dentropy is None else dentropy.cuda(), entropy=None if entropy is None else entropy.cuda(), stream=stream)
    return out.cpu()


def check_gradient(logits, tokens, vocab, dtype, with_entropy):
    W, T, _ = logits.shape
    exact = plain.log_probs(logits[..., :vocab], tokens)
    norms, entropy = exact["norms"][0].float(), exact["entropy"][0].float()
    gen = torch.Generator().manual_seed(9)
    dlog_probs = torch.randn((W, T), generator=gen)
    dlog_probs[(tokens < 0) | (tokens >= vocab)] = math.nan               # not read there
    dentropy = torch.randn((W, T), generator=gen) if with_entropy else None
    got = gradient(logits, tokens, vocab, norms, dlog_probs, dentropy, entropy if with_entropy else None, dtype)
    want, bound = plain.log_probs_gradient(logits[..., :vocab], tokens, norms, dlog_probs, dentropy, entropy, dtype)
    within(got[..., :vocab], want, bound)
    assert (got[..., vocab:] == 9.0).all()
    if dtype == logits.dtype:
        same = gradient(logits, tokens, vocab, norms, dlog_probs, dentropy, entropy if with_entropy else None, dtype, in_place=True)
        assert same_bits(same[..., :vocab], got[..., :vocab]) and same_bits(same[..., vocab:], logits[..., vocab:])


@pytest.mark.parametrize("with_entropy", [False, True])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradient(size, dtype, out, with_entropy):
    W, T, vocab, stride = size
    logits, tokens = draw(W, T, vocab, stride, DTYPES[dtype], IDS["i32" if T % 2 else "i64"])
    check_gradient(logits, tokens, vocab, DTYPES[out], with_entropy)


@pytest.mark.parametrize("with_entropy", [False, True])
def test_gradient_of_masked_rows(with_entropy):
    vocab = 300
    logits, tokens = draw(1, 6, vocab, vocab, torch.float32, torch.int64, seed=3)
    logits[0, 0] = -math.inf
    logits[0, 1, 1:] = -math.inf
    logits[0, 2, ::2] = -math.inf
    logits[0, 3] = LOWEST
    logits[0, 4, 100] = 60.0
    tokens[0] = torch.tensor([3, 0, 1, 5, 100, -1])
    check_gradient(logits, tokens, vocab, torch.float32, with_entropy)


def test_gradient_is_that_of_differences():
    vocab = 11
    logits, tokens = draw(1, 3, vocab, vocab, torch.float32, torch.int64, std=1.0, seed=5)
    tokens[0] = torch.tensor([2, 10, -1])
    weights, of_entropy = torch.tensor([[0.7, -1.3, 5.0]]), torch.tensor([[0.4, 0.0, -0.9]])
    exact = plain.log_probs(logits, tokens)
    got = gradient(logits, tokens, vocab, exact["norms"][0].float(), weights, of_entropy, exact["entropy"][0].float(), torch.float32)

    def value(l):
        want = plain.log_probs(l, tokens)
        return (want["log_probs"][0] * weights + want["entropy"][0] * of_entropy).sum().item()

    for i in range(logits.numel()):
        ends = []
        for step in (1e-4, -1e-4):
            moved = logits.double().clone()
            moved.view(-1)[i] += step
            ends.append(value(moved))
        assert abs((ends[0] - ends[1]) / 2e-4 - got.view(-1)[i].item()) < 1e-6


def test_no_tokens():
    plan = nl.LogProbPlan(10, 2, 4, max_top=2)
    nl.token_log_probs(plan, None, nl.F32, None, nl.I64, 0, None, top=2)
    nl.token_log_probs_gradient(plan, None, nl.F32, None, nl.I64, 0, None, None, None, nl.F32)


@pytest.mark.parametrize("T", [2, 300])
def test_captured_and_on_another_stream(T):
    """With parts that a second launch joins (few rows), and without."""
    W, vocab, top = 2, 30011, 6
    logits, tokens = draw(W, T, vocab, vocab, torch.bfloat16, torch.int64)
    logits, tokens = logits.cuda(), tokens.cuda()
    plan = nl.LogProbPlan(vocab, W, T, max_top=top)
    log_probs, norms, entropy = (torch.empty((W, T), device="cuda") for _ in range(3))
    top_tokens, top_log_probs = torch.empty((W, T, top), dtype=torch.int32, device="cuda"), torch.empty((W, T, top), device="cuda")
    dlogits, by = torch.empty_like(logits), torch.full((W, T), -1.0 / T, device="cuda")
    outs = (log_probs, norms, entropy, top_tokens, top_log_probs, dlogits)

    def both(stream=None):
        nl.token_log_probs(plan, logits, nl.BF16, tokens, nl.I64, T, log_probs, entropy=entropy, norms=norms, top=top, top_tokens=top_tokens,
                           top_log_probs=top_log_probs, stream=stream)
        nl.token_log_probs_gradient(plan, logits, nl.BF16, tokens, nl.I64, T, norms, by, dlogits, nl.BF16, dentropy=by, entropy=entropy, stream=stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for replay in range(3):
        logits.mul_(1.0 - 0.1 * replay)
        both()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for run in (graph.replay, lambda: both(stream=side)):
            for t in outs:
                t.fill_(3)
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
            assert all(same_bits(t, w) for t, w in zip(outs, want))
