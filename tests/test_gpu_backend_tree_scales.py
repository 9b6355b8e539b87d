"""Attention of trees with other softmax scales than the default: none, a negative one, and queries so faint that a scale near 0 times them leaves fp32's range."""
import copy

import pytest
import torch

from tests.backend_cases import Case, attend_bound
from tests.test_gpu_backend_tree import exact, masks, words_of

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def faint_weights(case):
    """What `attend_bound` does not know of for bf16 backends: over a quantised cache the weights are f16, 2^11 or more for a row's largest, times the value's scale relative to
    at most twice the largest scale.  Below f16's normal range they are off by 2^-25, so each of kv keys adds, relative to a largest weight of 1 (and so to a sum of 1 or more),
    2^-25 / 2^11 * 2 of the largest scale times its code: 2^-35 of the largest value.  It counts where a column's other values are nearly all 0, as int8 codes may be."""
    if case.kind == "16":
        return 0.0
    most = max(case.rows("v", i).nan_to_num().abs().max().item() for i, (q, kv) in enumerate(case.lens) if kv)
    return max(kv for _, kv in case.lens) * 2.0 ** -35 * most


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("drafts", [5, 13, 40])
@pytest.mark.parametrize("faint", [1.0, 2.0 ** -12], ids=["", "faint"])
def test_scales(cache, dtype, drafts, faint):
    lens = [(drafts, 300 + drafts), (1, 200), (drafts, drafts), (0, 9), (2, 131)]
    case = Case(lens, kv_heads=2, group=4, dim=128, page=16, dtype=dtype, cache=cache, seed=drafts)
    case.q.mul_(faint)
    bits = masks(lens, drafts)
    tree = words_of(bits, drafts)
    # the definition with another scale is that with the default one over queries times their ratio, in 64 bits
    scaled = copy.copy(case)
    for scale in (0.0, -0.05, 0.3, 2.0 ** -120, -2.0 ** -126):
        scaled.q = case.q.double() * (scale * case.dim ** 0.5)
        want, weight, scores = exact(scaled, bits, 0, 0)
        got = case.backend.attend(case.cache, case.batch, case.q, scale=scale, tree=tree)
        case.backend.sync()
        assert torch.isfinite(got).all(), f"scale {scale}: a hidden key reached a result"
        assert ((got.double() - want).abs() <= attend_bound(case, want, weight, scores) + faint_weights(case)).all(), f"scale {scale}"
