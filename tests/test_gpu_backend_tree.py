"""Attention of drafted trees over the paged cache against the definition in 64 bits."""
import math
import random

import pytest
import torch

from tests.backend_cases import Case, attend_bound

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
FEW = [(1, 1), (2, 2), (7, 7), (8, 40), (3, 300), (5, 64), (0, 9), (1, 700), (6, 129), (0, 0), (3, 2)]
MANY = [(64, 64), (33, 200), (61, 1200), (16, 16), (1, 500), (9, 128), (40, 161), (40, 30)]
LONG = [(130, 130), (200, 700), (129, 400)]


def masks(lens, seed, kind="tree"):
    """Per sequence, per new token: whole numbers of bits."""
    rng = random.Random(seed)
    got = []
    for q, _ in lens:
        bits = []
        for t in range(q):
            if kind == "tree":
                parent = -1 if t == 0 or rng.random() < 0.1 else rng.randrange(t)
                bits.append((bits[parent] if parent >= 0 else 0) | 1 << t)
            elif kind == "chain":
                bits.append((2 << t) - 1)
            else:                                            # anything, later tokens' bits and none at all among them
                bits.append(rng.choice([0, rng.getrandbits(max(q, 1) + 40), rng.getrandbits(q), 1 << t, (1 << q) - 1]))
        got.append(bits)
    return got


def words_of(bits, most, spare=0):
    words = max(1, (most + 31) // 32 + spare)
    rows = [[(b >> 32 * w & 0xFFFFFFFF) for w in range(words)] for seq in bits for b in seq]
    return torch.tensor([[x - (1 << 32) if x >> 31 else x for x in r] for r in rows], dtype=torch.int32, device="cuda").view(-1, words)


def seen_of(q_len, kv, bits, window, sinks):
    """[q_len, kv] of truth values: the definition, one by one."""
    c = kv - q_len
    seen = torch.zeros(q_len, max(kv, 0), dtype=torch.bool)
    for t, b in enumerate(bits):
        mine = [j for j in range(t + 1) if b >> j & 1]
        depth = max(0, len(mine) - 1)
        for j in range(min(c, kv)):
            seen[t, j] = not window or j > c + depth - window or j < sinks
        for j in mine:
            if c + j >= 0:
                seen[t, c + j] = True
    return seen.cuda()


def exact(case, bits, window, sinks):
    out = torch.zeros(case.tokens, case.heads, case.dim, dtype=torch.float64, device="cuda")
    weight, scores = torch.zeros_like(out), torch.zeros(case.tokens, case.heads, dtype=torch.float64, device="cuda")
    at = 0
    for i, (q_len, kv) in enumerate(case.lens):
        if q_len and kv:
            k, v, seen = torch.nan_to_num(case.rows("k", i)), torch.nan_to_num(case.rows("v", i)), seen_of(q_len, kv, bits[i], window, sinks)
            for h in range(case.heads):
                q = case.q[at : at + q_len, h].double()
                kh, vh = k[h // case.group], v[h // case.group]
                x = (q @ kh.T * case.dim ** -0.5).masked_fill(~seen, -math.inf)
                top = x.amax(-1, keepdim=True)
                e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
                e = torch.nan_to_num(e / e.sum(-1, keepdim=True))
                out[at : at + q_len, h], weight[at : at + q_len, h] = e @ vh, e @ vh.abs()
                scores[at : at + q_len, h] = (q.abs() @ kh.abs().T * case.dim ** -0.5).masked_fill(~seen, 0.0).amax(-1)
        at += q_len
    return out, weight, scores


def check(case, bits, window=0, sinks=0, spare=0):
    tree = words_of(bits, max(q for q, _ in case.lens), spare)
    got = case.backend.attend(case.cache, case.batch, case.q, window=window, sinks=sinks, tree=tree)
    case.backend.sync()
    want, weight, scores = exact(case, bits, window, sinks)
    bound = attend_bound(case, want, weight, scores)
    assert torch.isfinite(got).all(), "a hidden key reached a result"
    off = (got.double() - want).abs() - bound
    assert (off <= 0).all(), f"off by {off.max().item():.3g} more than {bound.flatten()[off.argmax()].item():.3g} may be"
    return got, bound


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,group", [(FEW, 4), (FEW + MANY, 1), (MANY, 7), (LONG, 4)], ids=["few", "mixed", "many", "long"])
def test_types_and_lengths(cache, dtype, dim, lens, group):
    check(Case(lens, kv_heads=2, group=group, dim=dim, page=16, dtype=dtype, cache=cache, seed=1), masks(lens, 1))


@pytest.mark.parametrize("group", [1, 3, 8, 16])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_groups_pages_and_any_masks(group, page):
    lens = FEW + MANY + LONG
    check(Case(lens, kv_heads=1, group=group, dim=64, page=page, dtype=BF16, cache="16", seed=2), masks(lens, 2, "any"), spare=2)


@pytest.mark.parametrize("cache", ["16", "int8"])
@pytest.mark.parametrize("lens", [FEW, MANY + LONG], ids=["few", "many"])
@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (100, 1), (128, 130), (250, 16), (5000, 3)])
def test_windows_and_sinks(cache, lens, kind, window, sinks):
    # pages that a chain of the tokens would have left behind may still be seen by a token of a tree: none is taken out of the table
    check(Case(lens, kv_heads=1, group=4, dim=128, page=32, dtype=BF16, cache=cache, seed=3), masks(lens, 3, kind), window, sinks)


@pytest.mark.parametrize("lens", [[(8, 20000)], [(61, 17000)], [(4, 5000), (64, 9000)]], ids=str)
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("window", [0, 3000])
def test_long_contexts_split_over_blocks(lens, cache, window):
    check(Case(lens, kv_heads=2, group=4, dim=128, page=64, dtype=BF16, cache=cache, seed=4), masks(lens, 4), window, 5)


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("tokens", [30, 61])
def test_shares_of_a_few_tiles(cache, tokens):
    """Contexts so short that a block gets two or three tiles: each meets its rings, barriers and clock rates cold, and fresh backends meet cold caches as well."""
    lens = [(tokens, 3000)]
    for rep in range(4):
        case = Case(lens, kv_heads=2, group=4, dim=128, page=64, dtype=BF16, cache=cache, seed=13 + rep)
        bits = masks(lens, 13 + rep)
        for _ in range(3):
            check(case, bits)


@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_more_sequences_than_a_launch_takes(cache):
    lens = [(1 + 7 * k % 23, 23 + 11 * k % 90) for k in range(275)] + [(0, 40), (23, 23), (2, 130)]
    check(Case(lens, kv_heads=1, group=4, dim=64, page=16, dtype=F16, cache=cache, seed=6), masks(lens, 6))


@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("lens", [FEW, LONG], ids=["few", "long"])
def test_a_chain_is_attention_without_a_tree(cache, lens):
    """The masks of a chain hide what causal order hides."""
    case = Case(lens, kv_heads=2, group=4, dim=64, page=16, dtype=BF16, cache=cache, seed=5)
    for window, sinks in ((0, 0), (300, 4)):                 # (a window beyond every depth, whose start then goes by the same places)
        got, bound = check(case, masks(lens, 5, "chain"), window, sinks)
        plain = case.backend.attend(case.cache, case.batch, case.q, window=window, sinks=sinks)
        assert ((got.double() - plain.double()).abs() <= 2 * bound).all()        # each is within the bound of the same values


@pytest.mark.parametrize("dtype,dim", [(BF16, 128), (F16, 64)], ids=["bf16-128", "f16-64"])
@pytest.mark.parametrize("lens,group", [([(5, 90), (3, 200)], 4), ([(8, 40), (64, 400)], 4), ([(61, 61)], 7)], ids=str)
@pytest.mark.parametrize("what", [math.nan, math.inf], ids=str)
def test_a_value_that_is_no_number_reaches_the_tokens_that_see_it(dtype, dim, lens, group, what):
    case = Case(lens, kv_heads=2, group=group, dim=dim, page=16, dtype=dtype, cache="16", seed=6)
    bits = masks(lens, 6)
    want, weight, scores = exact(case, bits, 0, 0)
    bound = attend_bound(case, want, weight, scores)
    hurt = torch.zeros_like(want, dtype=torch.bool)
    at = 0
    for i, (q_len, kv) in enumerate(lens):
        for n, j in enumerate(sorted({0, q_len // 2, q_len - 1})):
            place, d = kv - q_len + j, (7 * n + 13 * i) % dim
            case.v[case.table[i, place // 16].item(), 1, place % 16, d] = what
            for t, b in enumerate(bits[i]):
                if b >> j & 1:
                    hurt[at + t, group:, d] = True
        at += q_len
    got = case.backend.attend(case.cache, case.batch, case.q, tree=words_of(bits, max(q for q, _ in lens)))
    case.backend.sync()
    assert torch.equal(~torch.isfinite(got), hurt)
    assert ((got.double() - want).abs() <= bound)[~hurt].all()


@pytest.mark.parametrize("lens", [[(5, 90)], [(64, 300)]], ids=str)
def test_a_key_that_is_not_a_number_and_a_scale_that_is_none(lens):
    for cache in ("16", "int8"):
        case = Case(lens, kv_heads=1, group=4, dim=64, page=16, dtype=BF16, cache=cache, seed=7)
        bits = masks(lens, 7)
        q_len, kv = lens[0]
        j = q_len // 2
        place = kv - q_len + j
        cell = (case.table[0, place // 16].item(), 0, place % 16)
        if cache == "16":
            case.k[cell][5] = math.nan
        else:
            case.k_scale[cell] = case.v_scale[cell] = math.nan
        got = case.backend.attend(case.cache, case.batch, case.q, tree=words_of(bits, q_len))
        case.backend.sync()
        for t, b in enumerate(bits[0]):
            assert torch.isnan(got[t]).all() if b >> j & 1 else torch.isfinite(got[t]).all(), t


@pytest.mark.parametrize("lens", [[(3, 40), (4, 90)], [(40, 40), (64, 140)]], ids=["few", "many"])
def test_bad_page_is_skipped_and_reported(lens):
    from paper_2603_20661_b200.binding import WwwsError
    case = Case(lens, kv_heads=1, group=4, dim=64, page=16, dtype=BF16, cache="16", seed=8)
    tree = words_of(masks(lens, 8), max(q for q, _ in lens))
    good = case.backend.attend(case.cache, case.batch, case.q, tree=tree).clone()
    case.table[0, 1] = -1
    got = case.backend.attend(case.cache, case.batch, case.q, tree=tree)
    with pytest.raises(WwwsError) as e:
        case.backend.sync()
    assert e.value.status == 8
    assert torch.equal(got[lens[0][0] :], good[lens[0][0] :]) and torch.isfinite(got).all()


def test_repeats_bit_for_bit():
    lens = [(8, 4000), (61, 12000), (5, 700)]
    case = Case(lens, kv_heads=2, group=4, dim=128, page=64, dtype=BF16, cache="e4m3", seed=9)
    tree = words_of(masks(lens, 9), 61)
    first = case.backend.attend(case.cache, case.batch, case.q, tree=tree).clone()
    for _ in range(10):
        assert torch.equal(case.backend.attend(case.cache, case.batch, case.q, tree=tree), first)
    case.backend.sync()


def test_captured_and_replayed():
    lens = [(8, 400), (40, 300)]
    side = torch.cuda.Stream()
    case = Case(lens, kv_heads=2, group=4, dim=64, page=16, dtype=BF16, cache="16", seed=10, stream=side)
    trees = [words_of(masks(lens, s), 40) for s in (10, 11)]
    tree = trees[0].clone()
    torch.cuda.synchronize()
    want = [case.backend.attend(case.cache, case.batch, case.q, tree=t) for t in trees]        # on the side stream
    case.backend.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = case.backend.attend(case.cache, case.batch, case.q, tree=tree)
    for t, w in zip(trees, want):
        tree.copy_(t)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, w)


def test_refusals():
    from paper_2603_20661_b200.binding import WwwsError
    case = Case([(40, 60), (3, 20)], kv_heads=2, group=2, dim=64, page=16, dtype=BF16, cache="16", seed=13)
    b = case.backend
    good = words_of(masks(case.lens, 1), 40)
    for bad in (good[:40], good.long(), good[:, 0], good.cpu(), good.t().contiguous().t()):
        with pytest.raises(ValueError):
            b.attend(case.cache, case.batch, case.q, tree=bad)
    with pytest.raises(WwwsError) as e:
        b.attend(case.cache, case.batch, case.q, tree=good[:, :1].contiguous())
    assert e.value.status == 1 and "tree_words" in str(e.value)
    assert torch.isfinite(b.attend(case.cache, case.batch, case.q, tree=good)).all()
    b.sync()
