"""A page that a sliding window has left behind may already be someone else's: its table entry names nothing, and no kernel asks for it, whatever
the size of a kernel's tiles against that of a page."""
import pytest
import torch

from tests.backend_cases import Case
from tests.test_gpu_backend_attend import DECODE, MIXED, PROMPTS, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("window,sinks", [(1, 0), (20, 0), (20, 1), (33, 17), (100, 16), (112, 33)])
def test_pages_outside_the_window_are_not_looked_up(cache, dim, page, window, sinks):
    check(Case(DECODE + MIXED + PROMPTS + [(1, 100), (3, 100)], kv_heads=1, group=4, dim=dim, page=page, dtype=torch.bfloat16, cache=cache, seed=3, window=window,
               sinks=sinks), window, sinks)
