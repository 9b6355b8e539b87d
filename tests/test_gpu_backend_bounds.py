"""What does not fit a batch's bounds is refused or reported, and never passes unnoticed."""
import pytest
import torch

from tests.backend_cases import Case

pytestmark = pytest.mark.gpu


def small(lens=((1, 40), (1, 30)), **more):
    return Case(list(lens), **{**dict(kv_heads=1, group=4, dim=64, page=16, dtype=torch.bfloat16, cache="16", seed=11), **more})


def test_no_new_token_allowed_but_some_given():
    """max_q_len = 0 beside tokens: every sequence breaks the bounds, which the kernels report."""
    from paper_2603_20661_b200.binding import WwwsError
    case = small()
    batch = case.backend.batch(case.q_start, case.kv_len, case.table, n_tokens=2, max_q_len=0, max_kv_len=40)
    case.backend.attend(case.cache, batch, case.q)
    with pytest.raises(WwwsError) as e:
        case.backend.sync()
    assert e.value.status == 1
    assert torch.isfinite(case.attend()).all()
    case.backend.sync()

