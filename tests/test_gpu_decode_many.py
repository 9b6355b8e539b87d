"""Single tokens of many sequences: the searches and sums of the row kernel run over more than one block's threads."""
import random

import pytest
import torch

from tests.backend_cases import Case
from tests.test_gpu_backend_attend import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [129, 300, 1200, 2048])
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_single_tokens_of_many_sequences(n, cache):
    rng = random.Random(n)
    lens = [(1, 1 + rng.choice([-1, 0, 0, 5, 16, 40])) for _ in range(n)]
    lens[n // 2] = (1, 700)
    check(Case(lens, kv_heads=1, group=4, dim=64, page=16, dtype=torch.bfloat16, cache=cache, seed=n))
