"""A sequence whose new tokens end behind the call's arrays is skipped and reported by what writes the cache, as attention does."""
import pytest
import torch

from tests.backend_cases import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["16", "int8"])
@pytest.mark.parametrize("call", ["append", "rotate_append"])
@pytest.mark.parametrize("given", [23, 20], ids=["some of its tokens", "none of them"])
def test_a_sequence_that_ends_behind_the_tokens(cache, call, given):
    from paper_2603_20661_b200.binding import WwwsError
    case = Case([(20, 20), (5, 40)], kv_heads=2, group=2, dim=64, page=16, dtype=torch.bfloat16, cache=cache, seed=1)
    b, names = case.backend, [n for n in ("k", "v", "k_scale", "v_scale") if getattr(case, n) is not None]
    k, v = (torch.randn(25, 2, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    rotation = b.rotation(64)

    def write(n):
        batch = b.batch(case.q_start, case.kv_len, case.table, n_tokens=n, max_q_len=20, max_kv_len=40)
        if call == "append":
            b.append(case.cache, batch, k[:n], v[:n])
        else:
            b.rotate_append(case.cache, batch, case.q[:n], k[:n], v[:n], rotation)

    first = torch.zeros(case.n_pages, dtype=torch.bool, device="cuda")
    first[case.table[0, :2].long()] = True                   # the pages of the first sequence
    before = {n: getattr(case, n).view(torch.uint8).clone() for n in names}
    write(25)
    b.sync()
    whole = {n: getattr(case, n).view(torch.uint8).clone() for n in names}
    for n in names:
        getattr(case, n).view(torch.uint8).copy_(before[n])
    write(given)
    with pytest.raises(WwwsError) as e:
        b.sync()
    assert e.value.status == 1 and "offsets" in str(e.value)
    for n in names:
        now = getattr(case, n).view(torch.uint8)
        assert torch.equal(now[first], whole[n][first]) and not torch.equal(now[first], before[n][first]), n
        assert torch.equal(now[~first], before[n][~first]), n
