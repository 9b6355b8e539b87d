"""Trees under host bounds far beyond what the sequences hold, as a program passes that knows no more than its page table's width."""
import pytest
import torch

from tests.backend_cases import Case, attend_bound
from tests.test_gpu_backend_tree import exact, masks, words_of

pytestmark = pytest.mark.gpu

WIDE = 1 << 22                                               # pages of a sequence, 2^29 tokens


def attend(case, tree, max_kv_len):
    from paper_2603_20661_b200.backend import Backend
    n = len(case.lens)
    b = Backend(n_heads=case.heads, n_kv_heads=case.kv_heads, head_dim=case.dim, page_tokens=case.page, n_pages=case.n_pages, max_seqs=n, max_tokens=case.tokens, max_pages=WIDE,
                dtype=case.dtype, cache=case.kind, device="cuda")
    table = torch.zeros(n, WIDE, dtype=torch.int32, device="cuda")
    table[:, : case.max_pages] = case.table
    batch = b.batch(case.q_start, case.kv_len, table, n_tokens=case.tokens, max_q_len=max(q for q, _ in case.lens), max_kv_len=max_kv_len)
    out = b.attend(b.bind_cache(case.k, case.v, case.k_scale, case.v_scale), batch, case.q, tree=tree)
    b.sync()
    return out


@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_bounds_do_not_change_what_a_call_does(cache):
    lens = [(40, 1000), (33, 500), (1, 77)]
    case = Case(lens, kv_heads=2, group=4, dim=128, page=128, dtype=torch.bfloat16, cache=cache, seed=1)
    tree = words_of(masks(lens, 1), 40)
    assert torch.equal(attend(case, tree, WIDE * 128), attend(case, tree, 1000))


def test_more_sequences_than_fit_a_launch_under_such_bounds():
    lens = [(100 - 7 * i, 300 + 31 * i) for i in range(12)]
    case = Case(lens, kv_heads=8, group=4, dim=64, page=128, dtype=torch.bfloat16, cache="16", seed=2)
    bits = masks(lens, 2)
    got = attend(case, words_of(bits, 100), WIDE * 128)
    want, weight, scores = exact(case, bits, 0, 0)
    assert ((got.double() - want).abs() <= attend_bound(case, want, weight, scores)).all()
