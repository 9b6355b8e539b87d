"""Prompts beside single tokens, short chunks and idle sequences: one kernel answers a call, whatever its sequences are."""
import random

import pytest
import torch

from tests.backend_cases import Case
from tests.test_gpu_backend_attend import check

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def sequences(n, seed):
    rng = random.Random(seed)
    new = lambda: rng.choice([0, 1, 1, 1, 2, 5, 17, 32, 33, 49, 64, 100])                            # noqa: E731
    lens = [(q, q + rng.choice([0, 3, 90, 500])) for q in (new() for _ in range(n))]
    return [(70, 130)] + lens[1:-1] + [(1, 257)]


def kernels_of(case, side, **how):
    """Launches of a call, counted in a capture that is not run."""
    runtime = pytest.importorskip("cuda.bindings.runtime")
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph, stream=side):
        case.attend(**how)
    status, _, n = runtime.cudaGraphGetNodes(runtime.cudaGraph_t(graph.raw_cuda_graph()))
    assert int(status) == 0
    return n


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("n,launches", [(2, 1), (22, 1), (32, 1), (33, 2), (70, 3)])
def test_a_kernel_for_all_of_a_launch(cache, n, launches):
    side = torch.cuda.Stream()
    case = Case(sequences(n, n), kv_heads=1, group=1, dim=64, page=32, dtype=BF16, cache=cache, seed=n, stream=side)
    torch.cuda.synchronize()
    assert kernels_of(case, side) == launches


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("kv_heads,group,dim,page", [(1, 1, 64, 32), (1, 4, 64, 16), (2, 7, 128, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 4)])
def test_mixed_batches(cache, dtype, kv_heads, group, dim, page, window, sinks):
    check(Case(sequences(22, 5), kv_heads=kv_heads, group=group, dim=dim, page=page, dtype=dtype, cache=cache, seed=5, window=window, sinks=sinks), window, sinks)


@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_many_answers_beside_a_prompt(cache):
    """The ordinary step of a peer that takes prompts in while it answers: single tokens, and a chunk of one prompt."""
    rng = random.Random(9)
    check(Case([(1, rng.randrange(1, 2000)) for _ in range(60)] + [(200, 900)], kv_heads=2, group=4, dim=128, page=16, dtype=BF16, cache=cache, seed=9))
