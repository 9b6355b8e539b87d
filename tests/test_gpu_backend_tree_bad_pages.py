"""A page outside the pool hides its own keys and nothing else: values that are no numbers still reach the tokens that see them, in the same sequence
and in others that a block works on after it has met the page."""
import math

import pytest
import torch

from tests.backend_cases import Case
from tests.test_gpu_backend_tree import masks, words_of

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("drafts", [9, 40], ids=["one row tile", "two row tiles"])
@pytest.mark.parametrize("dtype,dim", [(BF16, 128), (F16, 64)], ids=["bf16-128", "f16-64"])
@pytest.mark.parametrize("what", [math.nan, math.inf], ids=str)
def test_values_that_are_no_numbers_beside_a_bad_page(drafts, dtype, dim, what):
    from paper_2603_20661_b200.binding import WwwsError
    # blocks take about thirty key tiles each: a block that meets a bad page goes on with more tiles, of this sequence and of the next
    lens = [(drafts, 2500 + 16 * i) for i in range(24)]
    case = Case(lens, kv_heads=8, group=4, dim=dim, page=32, dtype=dtype, cache="16", seed=3)
    bits = masks(lens, 3)
    tree = words_of(bits, drafts)

    def attend():
        out = case.backend.attend(case.cache, case.batch, case.q, tree=tree).clone()
        with pytest.raises(WwwsError) as e:
            case.backend.sync()
        assert e.value.status == 8
        return out

    for i in range(0, 24, 2):
        case.table[i, 1] = case.n_pages + i
    clean = attend()
    hurt = torch.zeros_like(clean, dtype=torch.bool)
    for i, (q_len, kv) in enumerate(lens):
        at, context = i * drafts, kv - q_len
        # in the tile of the bad page, in later tiles that every token sees, and among the drafts
        for n, place in enumerate((70, 700, 1500, context - 300, context + q_len // 2)):
            head, d = (n + i) % 8, (7 * n + 13 * i) % dim
            case.v[case.table[i, place // 32].item(), head, place % 32, d] = what
            for t, b in enumerate(bits[i]):
                if place < context or b >> (place - context) & 1:
                    hurt[at + t, 4 * head : 4 * head + 4, d] = True
    got = attend()
    assert torch.equal(~torch.isfinite(got), hurt)
    assert torch.equal(got[~hurt], clean[~hurt])
