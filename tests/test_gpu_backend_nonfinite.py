"""A value or key that is infinite or not a number reaches the rows that see it, in its own column (values) or in all (keys), and no other row."""
import math

import pytest
import torch

from tests.backend_cases import Case, attend_bound, attend_exact

pytestmark = pytest.mark.gpu


def sees(case, i, t, place, window, sinks):
    q_len, kv = case.lens[i]
    p = kv - q_len + t
    return place <= p and (not window or place > p - window or place < sinks)


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.float16, 64), (torch.bfloat16, 64)], ids=["bf16-128", "f16-64", "bf16-64"])
@pytest.mark.parametrize("lens,group", [([(5, 90), (3, 200)], 4), ([(2, 40), (9, 33)], 1), ([(70, 70), (300, 400)], 4), ([(130, 700)], 7), ([(600, 600)], 1)], ids=str)
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 0), (200, 3)])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf], ids=str)
def test_of_a_16_bit_cache(dtype, dim, lens, group, window, sinks, what):
    case = Case(lens, kv_heads=2, group=group, dim=dim, page=16, dtype=dtype, cache="16", seed=31, window=window, sinks=sinks)
    want, weight, scores = attend_exact(case, window, sinks, None)
    bound = attend_bound(case, want, weight, scores)
    hurt = torch.zeros_like(want, dtype=torch.bool)
    at = 0
    for i, (q_len, kv) in enumerate(lens):
        # new tokens' own places (the first, one amid them, the last but one), and one that the window leaves on the way
        for n, place in enumerate(sorted({kv - q_len, kv - q_len // 2 - 1, kv - 2, max(0, kv - q_len - 20)})):
            d = (7 * n + 13 * i) % dim
            page, slot = case.table[i, place // 16].item(), place % 16
            if page < 0:
                continue
            case.v[page, 1, slot, d] = what
            for t in range(q_len):
                if sees(case, i, t, place, window, sinks):
                    hurt[at + t, group:, d] = True
        at += q_len
    got = case.attend(window, sinks)
    case.backend.sync()
    assert torch.equal(~torch.isfinite(got), hurt)
    assert ((got.double() - want).abs() <= bound)[~hurt].all()


@pytest.mark.parametrize("lens,group", [([(5, 90)], 4), ([(70, 70), (300, 400)], 4)], ids=str)
def test_a_key_that_is_not_a_number(lens, group):
    case = Case(lens, kv_heads=2, group=group, dim=64, page=16, dtype=torch.bfloat16, cache="16", seed=32)
    want, weight, scores = attend_exact(case, 0, 0, None)
    bound = attend_bound(case, want, weight, scores)
    q_len, kv = lens[0]
    place = kv - q_len // 2 - 1
    case.k[case.table[0, place // 16].item(), 0, place % 16, 5] = math.nan
    got = case.attend(0, 0)
    case.backend.sync()
    hurt = torch.zeros_like(want, dtype=torch.bool)
    for t in range(q_len):
        hurt[t, :group] = sees(case, 0, t, place, 0, 0)
    assert torch.equal(torch.isnan(got), hurt)
    assert ((got.double() - want).abs() <= bound)[~hurt].all()
