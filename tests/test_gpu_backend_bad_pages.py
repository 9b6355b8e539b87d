"""Keys of a page outside the pool are hidden: the other keys share the softmax among themselves, as if the page were not there."""
import math

import pytest
import torch

from tests.backend_cases import Case, attend_bound

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def without_pages(case, window, sinks):
    """`attend_exact` with the keys of pages outside the pool hidden."""
    scale = case.dim ** -0.5
    out = torch.zeros(case.tokens, case.heads, case.dim, dtype=torch.float64, device="cuda")
    weight, scores = torch.zeros_like(out), torch.zeros(case.tokens, case.heads, dtype=torch.float64, device="cuda")
    at = 0
    for i, (q_len, kv) in enumerate(case.lens):
        if not (q_len and kv):
            at += q_len
            continue
        table = case.table[i].clone()
        there = (table >= 0) & (table < case.n_pages)
        case.table[i] = torch.where(there, table, -1)
        k, v = torch.nan_to_num(case.rows("k", i)), torch.nan_to_num(case.rows("v", i))
        case.table[i] = table
        p, j = torch.arange(kv - q_len, kv, device="cuda")[:, None], torch.arange(kv, device="cuda")
        seen = (j <= p) & there[j // case.page]
        if window:
            seen &= (j > p - window) | (j < sinks)
        for h in range(case.heads):
            q, kh, vh = case.q[at : at + q_len, h].double(), k[h // case.group], v[h // case.group]
            x = (q @ kh.T * scale).masked_fill(~seen, -math.inf)
            top = x.amax(-1, keepdim=True)
            e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
            e = torch.nan_to_num(e / e.sum(-1, keepdim=True))
            out[at : at + q_len, h], weight[at : at + q_len, h] = e @ vh, e @ vh.abs()
            scores[at : at + q_len, h] = ((q.abs() @ kh.abs().T) * scale).masked_fill(~seen, 0.0).amax(-1)
        at += q_len
    return out, weight, scores


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("dtype,dim", [(BF16, 128), (F16, 64)], ids=["bf16-128", "f16-64"])
@pytest.mark.parametrize("lens", [[(1, 40), (1, 600), (1, 16), (1, 2000)], [(5, 90), (2, 33)], [(40, 40), (130, 300), (200, 1500)]], ids=["decode", "few", "prompts"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 4)])
def test_keys_of_a_bad_page_are_hidden(cache, dtype, dim, lens, window, sinks):
    """Scores around -12: a key of zeros in the place of a hidden one would take nearly all the weight."""
    from paper_2603_20661_b200.binding import WwwsError
    case = Case(lens, kv_heads=2, group=4, dim=dim, page=16, dtype=dtype, cache=cache, seed=10, window=window, sinks=sinks)
    for p in (case.k.view(torch.int8),) if cache == "int8" else ():
        p.abs_()
    if cache == "16":
        case.k.abs_()
    elif cache == "e4m3":
        case.k.view(torch.uint8).bitwise_and_(0x7F)
    case.q.copy_(-case.q.abs() * 2)
    bad = {0: 0, 1: 1, 2: 0, 3: 50}
    for i, p in bad.items():
        if i < len(lens) and p < case.max_pages:
            case.table[i, p] = case.n_pages if i % 2 else -7
    case.table[len(lens) - 1, (lens[-1][1] - 1) // 16] = 1 << 30            # the page of the last token
    got = case.attend(window, sinks)
    with pytest.raises(WwwsError) as e:
        case.backend.sync()
    assert e.value.status == 8
    want, weight, scores = without_pages(case, window, sinks)
    assert torch.isfinite(got).all()
    off = (got.double() - want).abs() - attend_bound(case, want, weight, scores)
    assert (off <= 0).all(), off.max().item()
