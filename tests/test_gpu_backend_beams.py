"""Beam search's selection over beams and vocabulary against the definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def backend(rows, stream=None):
    from paper_2603_20661_b200.backend import Backend
    return Backend(max_rows=rows, device="cuda", stream=stream)


def exact(logits, totals, beams, keep):
    """(scores in 64 bits, parents, tokens), sorted; every score of a request, to tell neighbours apart."""
    rows, vocab = logits.shape
    x = logits.double()
    lost = torch.isnan(x).any(-1) | (x == math.inf).any(-1) | ~torch.isfinite(totals)
    score = torch.where(lost[:, None], -math.inf, torch.log_softmax(torch.where(lost[:, None], 0.0, x), -1) + totals.double()[:, None])
    score = torch.where(torch.isnan(score), -math.inf, score).view(rows // beams, beams * vocab)      # (a row of -infinity alone has no softmax)
    value, at = torch.sort(score, dim=-1, descending=True, stable=True)
    value, at = value[:, :keep], at[:, :keep]
    first = torch.arange(rows // beams, device="cuda")[:, None] * beams
    none = value == -math.inf
    return value, torch.where(none, -1, first + at // vocab), torch.where(none, -1, at % vocab)


def check(logits, totals, beams, keep, b=None):
    """Scores: fp32's rounding, and the sum's terms: 2^-21 each for the exponential and its argument (|x - max| 2^-24, which falls faster than the weight
    grows), (64 + 20) 2^-24 for their sum; all relative to the sum, so that is the error of its logarithm: 2^-20 + 2^-17.
    Candidates of one request swap only where their exact scores are nearer than that; there the parents decide by the same rule among themselves."""
    b = b or backend(logits.shape[0])
    score, parent, token = b.select_beams(logits, totals, beams=beams, keep=keep)
    b.sync()
    n = logits.shape[0] // beams
    assert score.shape == parent.shape == token.shape == (n, keep) and score.dtype == F32
    want, rows, tokens = exact(logits, totals, beams, keep)
    want, rows, tokens = (torch.cat([t, t.new_full((n, keep - t.shape[1]), v)], 1) for t, v in ((want, -math.inf), (rows, -1), (tokens, -1)))
    off = 2.0 ** -17 + 2.0 ** -20
    some = want > -math.inf
    assert torch.equal(score > -math.inf, some)
    assert ((score.double() - want).abs()[some] <= (2.0 ** -24 * want.abs() + off)[some]).all()
    assert (parent[~some] == -1).all() and (token[~some] == -1).all()
    same = (parent == rows) & (token == tokens)
    if not same.all():
        # where they differ, what was chosen scores what it says, by less than the two errors beside the place's own score, and nothing is chosen twice
        x = torch.log_softmax(logits.double(), -1) + totals.double()[:, None]
        at = torch.nonzero(~same)
        mine = x[parent[at[:, 0], at[:, 1]].long(), token[at[:, 0], at[:, 1]].long()]
        assert ((mine - want[at[:, 0], at[:, 1]]).abs() <= 2 * off).all()
        assert (parent[at[:, 0], at[:, 1]] != rows[at[:, 0], at[:, 1]]).all(), "candidates of one beam are in the logits' order"
    pairs = parent.long() * (1 << 32) + token
    for r in range(n):
        got = pairs[r][some[r]]
        assert got.unique().numel() == got.numel()
    return score, parent, token


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 31, 256, 1000, 4097, 32003, 131075])
@pytest.mark.parametrize("requests,beams,keep", [(1, 1, 1), (1, 4, 8), (3, 5, 11), (2, 32, 64), (7, 1, 33), (1, 2, 128)])
def test_types_and_sizes(dtype, vocab, requests, beams, keep):
    g = torch.Generator("cuda").manual_seed(vocab + keep)
    logits = (3.0 * torch.randn(requests * beams, vocab, generator=g, device="cuda")).to(dtype)
    totals = -5.0 * torch.rand(requests * beams, generator=g, device="cuda")
    check(logits, totals, beams, keep)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_first_step_dead_beams_and_masked_logits(dtype):
    """Beams without a hypothesis yet, rows under a grammar that leaves a few tokens or none."""
    g = torch.Generator("cuda").manual_seed(2)
    logits = torch.randn(12, 5003, generator=g, device="cuda").to(dtype)
    totals = torch.zeros(12, device="cuda")
    totals.view(3, 4)[:, 1:] = -math.inf
    check(logits, totals, 4, 8)
    logits[0, 3:] = -math.inf
    logits[4] = -math.inf
    logits[8, :] = -math.inf
    logits[8, [7, 4999]] = 1.0
    _, _, token = check(logits, totals, 4, 8)
    assert token[1].tolist() == [-1] * 8 and token[2].tolist() == [7, 4999] + [-1] * 6
    check(logits, torch.full((12,), -math.inf, device="cuda"), 4, 8)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [300, 9001, 70001])
def test_ties_go_to_the_lowest_row_and_token(dtype, vocab):
    """Constant rows, rows of two values, rows equal to one another: far more equal candidates than are kept."""
    logits = torch.zeros(4, vocab, device="cuda").to(dtype)
    totals = torch.tensor([-1.0, -1.0, -0.5, -0.5], device="cuda")
    _, parent, token = check(logits, totals, 4, 37)
    assert (parent == 2).all() and token[0].tolist() == list(range(37))
    logits[:, vocab // 2 :: 3] = 2.0
    _, parent, token = check(logits, totals, 2, 128)
    assert token[0, :40].tolist() == list(range(vocab // 2, vocab, 3))[:40] and (parent[0, : min(128, len(range(vocab // 2, vocab, 3)))] == 0).all()
    logits[:, 5], logits[:, 9] = -0.0, 0.0
    check(logits, totals, 1, 64)
    same = (2.0 * torch.randn(1, vocab, device="cuda")).to(dtype).expand(6, vocab).contiguous()
    _, parent, token = check(same, torch.zeros(6, device="cuda"), 6, 12)
    top = same[0].float().max()
    first = torch.nonzero(same[0].float() == top)[:, 0].tolist()
    want = [(r, t) for r in range(6) for t in first][:12]
    assert list(zip(parent[0].tolist(), token[0].tolist()))[: len(want)] == want


def test_best_ones_beside_one_another():
    """Sorted logits: the best of a row lie in one thread's or one warp's share."""
    for dtype in (F32, BF16):
        for step in (1, 8, 256, 2048):
            x = torch.full((2, 40000), -9.0, device="cuda")
            x[:, torch.arange(19) * step + 77] = torch.linspace(5.0, 1.0, 19, device="cuda").to(dtype).float()
            check(x.to(dtype), torch.tensor([0.0, -0.25], device="cuda"), 2, 24)
        x = torch.linspace(8.0, -8.0, 30000, device="cuda").expand(2, 30000).contiguous().to(dtype)
        check(x, torch.tensor([0.0, -0.1], device="cuda"), 2, 100)
        check(x.flip(1).contiguous(), torch.tensor([0.0, -0.1], device="cuda"), 1, 100)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("keep", [3, 40])
@pytest.mark.parametrize("vocab", [33000, 33001])
def test_many_rows_whose_slices_are_long(dtype, keep, vocab):
    """Enough rows that a block takes a whole one, tile by tile: rows that rise, fall, are constant, begin with nothing, and some at random."""
    g = torch.Generator("cuda").manual_seed(vocab + keep)
    x = torch.randn(600, vocab, generator=g, device="cuda")
    x[0::8] = torch.linspace(-6.0, 6.0, vocab, device="cuda")
    x[1::8] = torch.linspace(6.0, -6.0, vocab, device="cuda")
    x[2::8] = 0.5
    x[3::8, : vocab - 2000] = -math.inf
    x[4::8, :20000] = -math.inf
    x[5::8] = -math.inf
    x[5::8, vocab - 1] = 0.0
    x = x.to(dtype)
    totals = -3.0 * torch.rand(600, generator=g, device="cuda")
    totals[::13] = -math.inf
    check(x, totals, 3, keep)
    check(x, totals, 200, keep)


def test_large_and_unreal_logits():
    g = torch.Generator("cuda").manual_seed(4)
    x = torch.randn(6, 20003, generator=g, device="cuda")
    x[0] *= 1e30
    x[1] -= 3e4
    x[2, 777] = math.nan
    x[3, 19000] = math.inf
    x[4, 3000:] = math.nan                   # slices without a number
    totals = torch.tensor([0.0, -1.0, -1.0, -1.0, 0.0, math.nan], device="cuda")
    b = backend(6)
    score, parent, token = b.select_beams(x, totals, beams=1, keep=5)
    b.sync()
    assert (score[2:] == -math.inf).all() and (parent[2:] == -1).all() and (token[2:] == -1).all()
    check(x[:2].contiguous(), totals[:2].contiguous(), 1, 5)
    check(x, totals, 6, 9)
    check(x[:3], torch.tensor([math.inf, -1.0, 0.0], device="cuda"), 3, 9)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("offset,stride", [(0, 1009), (1, 1009), (3, 1024), (5, 1111)])
def test_strides_and_alignment(dtype, offset, stride):
    """Rows that begin anywhere in 16 bytes; what lies between them would win."""
    base = torch.full((offset + 6 * stride + 64,), 99.0, device="cuda").to(dtype)
    logits = base[offset : offset + 6 * stride].view(6, stride)[:, :1001]
    logits.copy_(torch.randn(6, 1001, device="cuda"))
    check(logits, torch.zeros(6, device="cuda"), 3, 10)


def test_repeats_bit_for_bit_and_leaves_tickets_clean():
    g = torch.Generator("cuda").manual_seed(6)
    logits, totals, b = torch.randn(64, 40001, generator=g, device="cuda").to(BF16), torch.zeros(64, device="cuda"), backend(64)
    first = b.select_beams(logits, totals, beams=4, keep=8)
    for beams, keep in ((4, 8), (8, 16), (64, 20), (4, 8)):
        got = b.select_beams(logits, totals, beams=beams, keep=keep)
    assert all(torch.equal(x, y) for x, y in zip(first, got))
    from paper_2603_20661_b200.backend import Backend                      # the tickets are those of shape_logits
    assert isinstance(b, Backend)
    out, token = b.shape_logits(logits, b.shaping())
    assert torch.equal(token, logits.float().argmax(-1).to(torch.int32))
    got = b.select_beams(logits, totals, beams=4, keep=8)
    b.sync()
    assert all(torch.equal(x, y) for x, y in zip(first, got))


def test_captured_and_replayed_and_on_another_stream():
    side = torch.cuda.Stream()
    b = backend(8, stream=side)
    logits, totals = torch.randn(8, 30011, device="cuda"), torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = b.select_beams(logits, totals, beams=4, keep=8)
    for seed in (1, 2):
        logits.copy_(torch.randn(8, 30011, generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = check(logits, totals, 4, 8)
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    eager = b.select_beams(logits, totals, beams=4, keep=8)
    junk = [torch.full((1 << 20,), 7.0, device="cuda") for _ in range(8)]  # the caller's stream reuses memory meanwhile
    b.sync()
    assert all(torch.equal(x, y) for x, y in zip(eager, want))
    del junk


def test_refusals():
    from paper_2603_20661_b200.binding import WwwsError
    b, x, t = backend(8), torch.zeros(8, 50, device="cuda"), torch.zeros(8, device="cuda")
    for args, more in (((x, t[:7]), dict(beams=4, keep=4)), ((x, t.double()), dict(beams=4, keep=4)), ((x, t), dict(beams=3, keep=4)), ((x, t), dict(beams=0, keep=4)), ((x, t), dict(beams=4, keep=0)),
                       ((x[0], t), dict(beams=4, keep=4)), ((x.double(), t), dict(beams=4, keep=4)), ((x.t(), t), dict(beams=4, keep=4)), ((x.cpu(), t), dict(beams=4, keep=4))):
        with pytest.raises(ValueError):
            b.select_beams(*args, **more)
    for args, more in (((x, t), dict(beams=4, keep=129)), ((torch.zeros(9, 5, device="cuda"), torch.zeros(9, device="cuda")), dict(beams=3, keep=2)),
                       ((torch.zeros(257, 5, device="cuda"), torch.zeros(257, device="cuda")), dict(beams=257, keep=2))):
        with pytest.raises(WwwsError):
            b.select_beams(*args, **more)
    none = b.select_beams(x[:0], t[:0], beams=4, keep=4)
    assert none[0].shape == (0, 4)
    b.sync()
