"""After a wait inside `attend` ran out (its blocks then leave without taking their tickets), the next call starts clean.  Nothing is made to wait
here: the state that such a call leaves behind is written into the workspace."""
import pytest
import torch

from tests.backend_cases import Case

pytestmark = pytest.mark.gpu

ERR_TIMEOUT, TIMEOUT_BIT = 7, 16


@pytest.mark.parametrize("lens", [[(1, 9000), (1, 12000)], [(40, 6000)]], ids=["decode", "prompts"])
@pytest.mark.parametrize("left", [1, 3])
def test_tickets_start_at_zero_after_a_timeout(lens, left):
    from paper_2603_20661_b200.binding import WwwsError
    case = Case(lens, kv_heads=2, group=4, dim=64, page=64, dtype=torch.bfloat16, cache="16", seed=41)
    good = case.attend().clone()
    case.backend.sync()
    words = case.backend._ws[:4096].view(torch.int32)
    before = words.clone()
    assert (before[:960] == 0).all()                          # the error word and the tickets: left at zero by every call
    words[0] = TIMEOUT_BIT
    words[64:256] = left                                      # 256 bytes on: the tickets of the first blocks
    with pytest.raises(WwwsError) as e:
        case.backend.sync()
    assert e.value.status == ERR_TIMEOUT
    case.backend.sync()                                       # reported once
    assert (words[:960] == 0).all()
    for _ in range(3):
        assert torch.equal(case.attend(), good)
    case.backend.sync()
