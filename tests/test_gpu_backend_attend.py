"""Attention over the paged cache against the definition in 64 bits: every type, cache kind and head layout, lengths from nothing to
several tiles, windows with sinks, pages in any order, garbage wherever no row may look."""
import math

import pytest
import torch

from tests.backend_cases import Case, attend_bound, attend_exact

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
DECODE = [(1, 1), (1, 2), (1, 15), (1, 16), (1, 17), (1, 32), (1, 33), (1, 64), (1, 129), (1, 1000), (0, 40), (1, 0), (0, 0)]
MIXED = [(1, 300), (5, 5), (16, 16), (3, 0), (17, 40), (0, 7), (33, 33), (40, 12), (2, 257)]
PROMPTS = [(128, 128), (129, 129), (255, 300), (64, 513), (1, 700), (300, 300), (7, 7), (31, 1200)]


def check(case, window=0, sinks=0, scale=None, stride_pad=0):
    got = case.attend(window, sinks, scale, stride_pad)
    case.backend.sync()
    want, weight, scores = attend_exact(case, window, sinks, scale)
    bound = attend_bound(case, want, weight, scores)
    assert torch.isfinite(got).all(), "a hidden key reached a result"
    off = (got.double() - want).abs() - bound
    assert (off <= 0).all(), f"off by {off.max().item():.3g} more than {bound.flatten()[off.argmax()].item():.3g} may be"


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,group", [(DECODE, 4), (MIXED, 1), (PROMPTS, 7)], ids=["decode", "mixed", "prompts"])
def test_types_and_lengths(cache, dtype, dim, lens, group):
    check(Case(lens, kv_heads=2, group=group, dim=dim, page=16, dtype=dtype, cache=cache, seed=1))


@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 13, 16])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_groups_and_pages(group, page):
    check(Case(MIXED + PROMPTS, kv_heads=3, group=group, dim=64, page=page, dtype=BF16, cache="16", seed=2))


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (16, 4), (33, 17), (100, 1), (128, 130), (250, 16), (5000, 3), (64, 100000)])
def test_windows_and_sinks(cache, window, sinks):
    check(Case(DECODE + MIXED + PROMPTS, kv_heads=1, group=4, dim=128, page=32, dtype=BF16, cache=cache, seed=3, window=window, sinks=sinks), window, sinks)


@pytest.mark.parametrize("lens", [[(1, 20000)], [(4, 9001)], [(1, 5000), (1, 30), (1, 17000)], [(600, 3000)], [(200, 9000)]], ids=str)
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_long_sequences_split_over_blocks(lens, cache):
    check(Case(lens, kv_heads=2, group=4, dim=128, page=64, dtype=BF16, cache=cache, seed=4))
    check(Case(lens, kv_heads=2, group=4, dim=128, page=64, dtype=BF16, cache=cache, seed=4, window=3000, sinks=5), 3000, 5)


@pytest.mark.parametrize("lens", [DECODE, PROMPTS], ids=["decode", "prompts"])
def test_strided_rows_and_other_scales(lens):
    case = Case(lens, kv_heads=2, group=4, dim=64, page=16, dtype=F16, cache="16", seed=5)
    check(case, scale=0.3, stride_pad=24)
    check(case, scale=-0.05, stride_pad=8)
    check(case, scale=0.0)


@pytest.mark.parametrize("cache", ["16", "int8"])
@pytest.mark.parametrize("lens", [[(1, 200)] * 3, [(150, 200)] * 2], ids=["decode", "prompts"])
def test_large_scores_keep_their_softmax(cache, lens):
    """Scores in the hundreds of both signs: the running maximum has to move, and no sum may overflow."""
    case = Case(lens, kv_heads=1, group=4, dim=64, page=16, dtype=BF16, cache=cache, seed=6, loud=30.0)
    check(case)


@pytest.mark.parametrize("lens", [[(1, 70), (1, 9)], [(4, 70), (3, 9)], [(70, 70), (140, 150)]], ids=["decode", "few", "prompts"])
def test_nan_row_of_a_quantised_cache_reaches_only_rows_that_see_it(lens):
    case = Case(lens, kv_heads=2, group=4, dim=64, page=16, dtype=BF16, cache="int8", seed=7)
    for place in (0, 64):
        case.k_scale[case.table[0, place // 16].item(), 1, place % 16] = math.nan
        case.v_scale[case.table[0, place // 16].item(), 0, place % 16] = math.nan
    window = 16                      # places 0 and 64 hidden from most rows
    got = case.attend(window, 0)
    case.backend.sync()
    q_len, kv = lens[0]
    for t in range(q_len):
        p = kv - q_len + t
        sees = any(p - window < j <= p for j in (0, 64))
        assert torch.isnan(got[t]).all() if sees else torch.isfinite(got[t]).all(), (t, p)
    assert torch.isfinite(got[q_len:]).all()


def test_repeats_bit_for_bit_and_leaves_tickets_clean():
    case = Case([(1, 4000), (1, 333), (1, 12000), (9, 700)], kv_heads=2, group=4, dim=128, page=64, dtype=BF16, cache="e4m3", seed=8)
    first = case.attend(0, 0).clone()
    for _ in range(20):
        assert torch.equal(case.attend(0, 0), first)


def test_another_stream_than_the_callers():
    side = torch.cuda.Stream()
    case = Case(MIXED + PROMPTS, kv_heads=2, group=4, dim=64, page=16, dtype=BF16, cache="16", seed=9, stream=side)
    torch.cuda.synchronize()
    got = case.attend(0, 0)
    junk = [torch.full((1 << 20,), 7.0, device="cuda") for _ in range(8)]       # the caller's stream reuses memory meanwhile
    case.backend.sync()
    want, weight, scores = attend_exact(case, 0, 0, None)
    assert ((got.double() - want).abs() <= attend_bound(case, want, weight, scores)).all()
    del junk


@pytest.mark.parametrize("lens", [[(1, 40), (1, 40)], [(40, 40), (130, 140)]], ids=["decode", "prompts"])
def test_bad_page_is_skipped_and_reported(lens):
    from paper_2603_20661_b200.binding import WwwsError
    case = Case(lens, kv_heads=1, group=4, dim=64, page=16, dtype=BF16, cache="16", seed=10)
    good = case.attend(0, 0).clone()
    case.table[0, 1] = case.n_pages
    got = case.attend(0, 0)
    with pytest.raises(WwwsError) as e:
        case.backend.sync()
    assert e.value.status == 8 and "page" in str(e.value)
    assert torch.equal(got[lens[0][0]:], good[lens[0][0]:]) and torch.isfinite(got).all()
    case.table[0, 1] = -1
    case.attend(0, 0)
    with pytest.raises(WwwsError):
        case.backend.sync()
    case.backend.sync()                                      # reported once


def test_sequence_beyond_the_bounds_is_skipped_and_reported():
    from paper_2603_20661_b200.binding import WwwsError
    case = Case([(1, 40), (1, 30)], kv_heads=1, group=4, dim=64, page=16, dtype=BF16, cache="16", seed=11)
    good = case.attend(0, 0).clone()
    case.kv_len[0] = 41                                      # above max_kv_len
    got = case.attend(0, 0)
    with pytest.raises(WwwsError) as e:
        case.backend.sync()
    assert e.value.status == 1
    assert torch.equal(got[1], good[1])


@pytest.mark.parametrize("q_len", [1, 200])
def test_pool_beyond_32_bit_offsets(q_len):
    """A pool of more than 2^32 bytes each for keys and values, the sequence's pages at its far end."""
    case = Case([(q_len, 300)], kv_heads=8, group=1, dim=128, page=128, dtype=BF16, cache="16", seed=12, extra_pages=17000)
    assert case.k.numel() * 2 > 1 << 32 and case.table[0].min().item() * 8 * 128 * 128 * 2 > 1 << 32
    check(case)


def test_refusals():
    from paper_2603_20661_b200.binding import WwwsError
    case = Case([(2, 20)], kv_heads=2, group=2, dim=64, page=16, dtype=BF16, cache="16", seed=13)
    b = case.backend
    with pytest.raises(ValueError):
        b.attend(case.cache, case.batch, case.q[:, :3])
    with pytest.raises(ValueError):
        b.attend(case.cache, case.batch, case.q.float())
    with pytest.raises(ValueError):
        b.attend(case.cache, case.batch, case.q[:1])
    with pytest.raises(ValueError):
        b.attend(case.cache, case.batch, case.q.transpose(0, 1).contiguous().transpose(0, 1))
    with pytest.raises(ValueError):
        b.bind_cache(case.k[:1], case.v)
    odd = torch.zeros(2 * 4 * 64 + 8, dtype=BF16, device="cuda")[1:2 * 4 * 64 + 1].view(2, 4, 64)      # 2 bytes off a 16-byte boundary
    with pytest.raises(WwwsError) as e:
        b.attend(case.cache, case.batch, odd)
    assert e.value.status == 1 and "aligned" in str(e.value)
    wide = torch.zeros(2, 4 * 64 + 4, dtype=BF16, device="cuda")[:, : 4 * 64].unflatten(1, (4, 64))
    with pytest.raises(WwwsError):
        b.attend(case.cache, case.batch, wide)
    with pytest.raises(WwwsError):
        b.attend(case.cache, case.batch, case.q, scale=math.inf)
    too_long = b.batch(case.q_start, case.kv_len, case.table, n_tokens=2, max_q_len=2, max_kv_len=33)
    with pytest.raises(WwwsError) as e:
        b.attend(case.cache, too_long, case.q)
    assert "page table" in str(e.value)
