"""What a program does when the page pool has run out: it drops the sequence, or cuts it back to the pages it got."""
import pytest
import torch

from tests.test_gpu_backend_pages import backend, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
def test_places_without_a_page_are_let_go(in_place):
    from paper_2603_20661_b200.binding import WwwsError

    def short():
        b = backend(16, 4, 5, 4)
        refs, table, held, _ = b.fork(i32([0, 2, 0, 0]), i32([], 0, 5), i32([]), i32([-1]), i32([0]), i32([80]), in_place=in_place)
        with pytest.raises(WwwsError) as e:
            b.sync()
        assert e.value.status == 2 and table.tolist() == [[0, 2, 3, -1, -1]] and held.tolist() == [5] and refs.tolist() == [1, 2, 1, 1]
        return b, refs, table, held

    b, refs, table, held = short()
    refs, *_ = b.fork(refs, table, held, i32([]), i32([]), i32([]), in_place=in_place)
    b.sync()
    assert refs.tolist() == [0, 2, 0, 0]
    for source, keep in ((0, 48), (0, 33), (0, 0)):
        b, refs, table, held = short()
        refs, table, held, moves = b.fork(refs, table, held, i32([source]), i32([keep]), i32([0]), in_place=in_place)
        b.sync()
        pages = -(-keep // 16)
        assert table.tolist() == [[0, 2, 3][:pages] + [0] * (5 - pages)] and held.tolist() == [pages] and moves.tolist() == [[-1, -1, 0]]
        assert refs.tolist() == [int(pages > 0), 2, int(pages > 1), int(pages > 2)]
    for keep in (49, 64):                                    # a place without a page holds nothing to continue
        b, refs, table, held = short()
        _, table, _, moves = b.fork(refs, table, held, i32([0]), i32([keep]), i32([0]), in_place=in_place)
        with pytest.raises(WwwsError) as e:
            b.sync()
        assert e.value.status == 8 and table.tolist() == [[0, 2, 3, -1, 0]] and moves.tolist() == [[-1, -1, 0]]
