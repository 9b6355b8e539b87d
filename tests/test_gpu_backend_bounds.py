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



@pytest.mark.parametrize("lens", [((1, 40), (1, 30)), ((40, 40), (40, 70)), ((40, 40), (1, 70))], ids=["decode", "prompts", "mixed"])
@pytest.mark.parametrize("kind", ["behind", "before"])
def test_tokens_that_no_sequence_holds_are_reported(lens, kind):
    from paper_2603_20661_b200.binding import WwwsError
    case = small(lens)
    good = case.attend()
    case.backend.sync()
    start = case.q_start.tolist()
    start = [start[0], start[1], start[2] - 1] if kind == "behind" else [1] + start[1:]
    batch = case.backend.batch(torch.tensor(start, dtype=torch.int32, device="cuda"), case.kv_len, case.table, n_tokens=case.tokens, max_q_len=max(q for q, _ in lens),
                               max_kv_len=max(kv for _, kv in lens))
    case.backend.attend(case.cache, batch, case.q)
    with pytest.raises(WwwsError) as e:
        case.backend.sync()
    assert e.value.status == 1 and "offsets" in str(e.value)
    assert torch.equal(case.attend(), good)
    case.backend.sync()


def test_windows_and_sinks_below_zero_are_refused():
    """They would wrap to bounds that hide nothing, or show everything."""
    case = small()
    for more in (dict(window=-1), dict(sinks=-1), dict(window=8, sinks=-4)):
        with pytest.raises(ValueError):
            case.attend(**more)


def test_records_of_another_configuration_are_refused():
    """A pool of fewer pages, a table of fewer columns or another kind of record would be read past its end.  Those of an equal backend are welcome."""
    case, same, longer, other = small(), small(), small([(1, 400), (1, 30)]), small(cache="int8")
    b = case.backend
    for cache, batch in ((longer.cache, case.batch), (other.cache, case.batch), (case.cache, longer.batch), (case.batch, case.cache), (b.shaping(), case.batch)):
        with pytest.raises(ValueError):
            b.attend(cache, batch, case.q)
        with pytest.raises(ValueError):
            b.append(cache, batch, case.q[:, :1], case.q[:, :1])
        with pytest.raises(ValueError):
            b.read(cache, batch, torch.zeros(3, dtype=torch.int32, device="cuda"), 0)
    with pytest.raises(ValueError):
        b.shape_logits(torch.zeros(2, 8, device="cuda"), case.batch)
    assert torch.equal(b.attend(same.cache, same.batch, same.q), case.attend())
    b.sync()
