"""Calls of more sequences than one launch of the tile kernel takes: prompts alone, and prompts among single tokens and idle sequences."""
import random

import pytest
import torch

from tests.backend_cases import Case, attend_bound, attend_exact
from tests.test_gpu_backend_attend import check

pytestmark = pytest.mark.gpu


def sequences(n, mixed):
    rng = random.Random(n)
    q = lambda: rng.choice([0, 1, 1, 3, 12, 40]) if mixed else rng.choice([40, 33])                  # noqa: E731
    return [(k, k + rng.choice([0, 0, 5, 60, 300])) for k in (q() for _ in range(n))]


@pytest.mark.parametrize("n", [32, 33, 70])
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("mixed", [False, True], ids=["prompts", "mixed"])
def test_sequences_are_taken_32_at_a_time(n, cache, mixed):
    check(Case(sequences(n, mixed), kv_heads=2, group=4, dim=128, page=32, dtype=torch.bfloat16, cache=cache, seed=n))


def test_offsets_are_checked_over_the_whole_call():
    """Only the call's first and last sequences, not those of each launch, have to meet its ends."""
    from paper_2603_20661_b200.binding import WwwsError
    lens = sequences(70, False)
    case = Case(lens, kv_heads=1, group=4, dim=64, page=16, dtype=torch.bfloat16, cache="16", seed=3)
    want, weight, scores = attend_exact(case, 0, 0, None)
    near = (lambda got, a, b: ((got.double() - want).abs() <= bound)[a:b].all())                     # (skipping one moves the cuts of the others' work)
    bound = attend_bound(case, want, weight, scores)
    case.q_start[70] -= 1
    got = case.attend()
    with pytest.raises(WwwsError) as e:
        case.backend.sync()
    assert e.value.status == 1
    assert near(got, 0, sum(q for q, _ in lens[:69]))
    case.q_start[70] += 1
    case.kv_len[40] = 1 << 20                                          # one sequence of the second launch breaks the bounds: it alone is skipped
    got = case.attend()
    with pytest.raises(WwwsError):
        case.backend.sync()
    a, b = sum(q for q, _ in lens[:40]), sum(q for q, _ in lens[:41])
    assert near(got, 0, a) and near(got, b, case.tokens)
