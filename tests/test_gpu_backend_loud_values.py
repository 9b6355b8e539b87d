"""Over a quantised cache one value far larger than the others, which some rows see and others do not: how far it may take the others' results off."""
import pytest
import torch

from tests.backend_cases import Case, attend_bound, attend_exact
from tests.test_gpu_backend_tree import exact, masks, words_of
from tests.test_gpu_backend_tree_scales import faint_weights

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def shout(case, place_of, by):
    """Token place_of(context, q_len) of every sequence holds values `by` times as large."""
    for i, (q, kv) in enumerate(case.lens):
        place = place_of(kv - q, q)
        case.v_scale[case.table[i, place // case.page].item(), :, place % case.page] *= by


def check(case, got, want, weight, scores):
    """Within the bounds; what is beyond f16's largest number (65,504, next to which numbers are 32 apart) is infinite."""
    bound = attend_bound(case, want, weight, scores) + faint_weights(case)
    beyond = want.abs() >= 65504.0 - bound if case.dtype == F16 else torch.zeros_like(want, dtype=torch.bool)
    assert ((got.double() - want).abs() <= bound)[~beyond].all()
    assert (torch.isinf(got) | (got.abs() > 60000.0))[beyond].all()


# (`faint_weights` counts the largest value of all, seen or not.  The row kernel and the tile kernel carry 2^15 and 2^11 for a row's largest weight and lose less.)
@pytest.mark.parametrize("cache", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("drafts", [5, 40])
@pytest.mark.parametrize("by", [2.0 ** 10, 2.0 ** 16])
def test_a_loud_sibling(cache, dtype, drafts, by):
    lens = [(drafts, 300 + drafts), (drafts, drafts), (drafts, 61 + drafts)]
    case = Case(lens, kv_heads=2, group=4, dim=128, page=16, dtype=dtype, cache=cache, seed=drafts)
    shout(case, lambda context, q: context + 1, by)
    # token 1 has children, and siblings that do not see it
    bits = [[b & ~2 | (1 << t) if t % 2 == 0 else b | 2 for t, b in enumerate(m)] for m in masks(lens, drafts)]
    want, weight, scores = exact(case, bits, 0, 0)
    got = case.backend.attend(case.cache, case.batch, case.q, tree=words_of(bits, drafts))
    case.backend.sync()
    check(case, got, want, weight, scores)


@pytest.mark.parametrize("cache", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("new", [5, 100])
@pytest.mark.parametrize("by", [2.0 ** 10, 2.0 ** 16])
def test_a_loud_token_ahead(cache, dtype, new, by):
    lens = [(new, 300 + new), (new, new), (new, 61 + new)]
    case = Case(lens, kv_heads=2, group=4, dim=128, page=16, dtype=dtype, cache=cache, seed=new)
    shout(case, lambda context, q: context + q // 2, by)
    want, weight, scores = attend_exact(case, 0, 0, None)
    got = case.attend()
    case.backend.sync()
    check(case, got, want, weight, scores)
