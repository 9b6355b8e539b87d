"""Pages of a paged cache under sequences that are forked, dropped, cut back and given room, against a count kept on the host."""
import random

import pytest
import torch

from tests.backend_cases import Case

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
i32 = lambda v, *shape: torch.tensor(v, dtype=torch.int32, device="cuda").view(*shape) if shape else torch.tensor(v, dtype=torch.int32, device="cuda")        # noqa: E731


def fork_on_host(refs, table, held, source, keep, room, page, width):
    """The definition, entry by entry.  Returns lists (refs, tables, held, moves) and whether the pool ran out."""
    refs = list(refs)
    for row, h in zip(table, held):
        for p in row[:h]:
            refs[p] -= 1
    new, ends = [], {}
    for i, (j, k) in enumerate(zip(source, keep)):
        new.append([])
        if j >= 0:
            new[i] = list(table[j][: k // page])
            for p in new[i]:
                refs[p] += 1
            if k % page:
                ends.setdefault(table[j][k // page], []).append(i)
    stays = {}
    for p, who in ends.items():
        if refs[p] == 0:
            stays[who[0]] = p
            refs[p] = 1
    free, short, moves, counts = [p for p, r in enumerate(refs) if r == 0], False, [], []
    for i, (j, k, r) in enumerate(zip(source, keep, room)):
        k = k if j >= 0 else 0
        counts.append(-(-max(k, r) // page))
        move = (-1, -1, 0)
        if i in stays:
            new[i].append(stays[i])
        elif k % page:
            move = (table[j][k // page], free[0] if free else -1, k % page)
        while len(new[i]) < counts[i]:
            short |= not free
            p = free.pop(0) if free else -1
            if p >= 0:
                refs[p] = 1
            new[i].append(p)
        moves.append(move)
        new[i] += [0] * (width - len(new[i]))
    return refs, new, counts, moves, short


def backend(page, n_pages, max_pages, max_seqs, stream=None, **more):
    from paper_2603_20661_b200.backend import Backend
    return Backend(**{**dict(n_heads=2, n_kv_heads=2, head_dim=64, page_tokens=page, n_pages=n_pages, max_seqs=max_seqs, max_tokens=8, max_pages=max_pages, dtype=BF16, device="cuda", stream=stream), **more})


def check(b, page, refs, table, held, source, keep, room, in_place=False):
    width = b.max_pages
    want = fork_on_host(refs, table, held, source, keep, room, page, width)
    before = i32(refs)
    got = b.fork(before, i32(table, len(table), width) if table else torch.zeros(0, width, dtype=torch.int32, device="cuda"), i32(held), i32(source), i32(keep), i32(room), in_place=in_place)
    if want[4]:
        from paper_2603_20661_b200.binding import WwwsError
        with pytest.raises(WwwsError) as e:
            b.sync()
        assert e.value.status == 2 and "pool" in str(e.value)
    else:
        b.sync()
    assert (got[0].data_ptr() == before.data_ptr()) == in_place
    if not in_place:
        assert before.tolist() == list(refs)
    assert got[0].tolist() == want[0]
    assert got[2].tolist() == want[2]
    assert got[1].tolist() == want[1] if source else got[1].shape[0] == 0
    assert [tuple(m) for m in got[3].tolist()] == want[3]
    return got


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("n_seqs,n_pages,width", [(1, 12, 4), (3, 60, 9), (40, 900, 33), (130, 9000, 70), (700, 20011, 20), (2048, 70001, 18)])
def test_steps_of_sequences_at_random(page, n_seqs, n_pages, width):
    """Several steps on end: continued, forked, cut back, dropped and new sequences, pages held by others."""
    rng = random.Random(n_seqs + page)
    b = backend(page, n_pages, width, 2048)
    outside = rng.sample(range(n_pages), min(n_pages // 20, 40))
    refs, table, held, length = [0] * n_pages, [], [], []
    for p in outside:
        refs[p] = rng.randrange(1, 3)
    for step in range(5):
        n = n_seqs if step != 2 else max(1, n_seqs // 2)
        source, keep, room = [], [], []
        for i in range(n):
            j = rng.randrange(len(table)) if table and rng.random() < 0.85 else -1
            if j >= 0 and i < len(table) and rng.random() < 0.5:
                j = i
            k = 0 if j < 0 else length[j] if rng.random() < 0.7 else rng.randrange(length[j] + 1)
            r = min(width * page, k + rng.choice([0, 1, 1, 1, page, rng.randrange(2 * page)])) if j >= 0 else rng.randrange(width * page // 2 + 1)
            source.append(j), keep.append(k), room.append(r)
        got = check(b, page, refs, table, held, source, keep, room, in_place=step % 2 == 1)
        refs, table, held = got[0].tolist(), got[1].tolist(), got[2].tolist()
        if any(p < 0 for row, h in zip(table, held) for p in row[:h]):
            return                                       # the pool ran out, as the smallest may
        length = [max(k if j >= 0 else 0, r) for j, k, r in zip(source, keep, room)]
        # every page is held as often as the tables and the others say
        count = [0] * n_pages
        for row, h in zip(table, held):
            for p in row[:h]:
                count[p] += 1
        assert all(r == c or p in outside and r > c for p, (r, c) in enumerate(zip(refs, count)))


def test_pages_that_are_shared_are_copied_before_they_are_written():
    b = backend(16, 12, 4, 8)
    # three sequences on one: full pages shared, the last one stays with the first and is copied for the others
    check(b, 16, [1, 1, 0, 1] + [0] * 8, [[3, 0, 1, 0]], [3], [0, 0, 0], [40, 40, 40], [41, 41, 49])
    # one ends inside a page that another holds whole: it is copied
    check(b, 16, [1, 1, 1] + [0] * 9, [[0, 1, 2, 0]], [3], [0, 0], [20, 32], [20, 32])
    # or that somebody else counts
    check(b, 16, [1, 2, 1] + [0] * 9, [[0, 1, 2, 0]], [3], [0], [20], [33])
    # two old ones that share a page, both cut back into it
    check(b, 16, [2, 2, 1, 1] + [0] * 8, [[0, 1, 2, 0], [0, 1, 3, 0]], [3, 3], [1, 0], [20, 25], [20, 25])
    # the freed page is the next one taken
    got = check(b, 16, [1, 1, 1] + [0] * 9, [[0, 1, 2, 0]], [3], [-1], [7], [5])
    assert got[1].tolist()[0][0] == 0


def test_nothing_old_nothing_new_and_an_empty_pool():
    b = backend(16, 5, 4, 4)
    check(b, 16, [0, 1, 0, 0, 2], [], [], [-1, -1], [0, 0], [17, 0])
    check(b, 16, [1, 1, 0, 0, 0], [[0, 1, 0, 0]], [2], [], [], [])
    check(b, 16, [1, 1, 0, 0, 0], [[0, 1, 0, 0]], [2], [0, 0, 0], [20, 20, 20], [40, 64, 20])            # runs out
    check(b, 16, [1, 1, 1, 1, 1], [[0, 1, 0, 0]], [2], [0, 0], [20, 20], [20, 20])                       # not even a copy's target


def test_bad_sequences_are_left_empty_and_reported():
    from paper_2603_20661_b200.binding import WwwsError
    b = backend(16, 12, 4, 8)
    refs, table, held = i32([1, 1, 1] + [0] * 9), i32([[0, 1, 2, 0]]), i32([3])
    for source, keep, room in (([0, 1], [40, 5], [41, 6]), ([0, 0], [40, 49], [41, 49]), ([0, 0], [40, -1], [41, 3]), ([0, -1], [40, 0], [41, 65]), ([0, -1], [40, 0], [41, -1])):
        got = b.fork(refs, table, held, i32(source), i32(keep), i32(room))
        with pytest.raises(WwwsError) as e:
            b.sync()
        assert e.value.status == 1
        assert got[2].tolist() == [3, 0] and got[1].tolist() == [[0, 1, 2, 0], [0, 0, 0, 0]] and got[0].tolist() == refs.tolist()
    got = b.fork(refs, i32([[0, 12, 2, 0]]), held, i32([0]), i32([40]), i32([40]))
    with pytest.raises(WwwsError) as e:
        b.sync()
    assert e.value.status == 8 and got[1].tolist() == [[0, 12, 2, 0]] and got[0].tolist() == refs.tolist()


LENS = [(5, 40), (1, 17), (20, 20), (33, 130), (0, 9), (3, 3)]


def layers(cache, dtype, page, kv_heads, dim, n=3):
    cases = [Case(LENS, kv_heads=kv_heads, group=1, dim=dim, page=page, dtype=dtype, cache=cache, seed=20 + i) for i in range(n)]
    for c in cases[1:]:
        c.table = cases[0].table
    return cases, cases[0].backend.caches([cases[0].backend.bind_cache(c.k, c.v, c.k_scale, c.v_scale) for c in cases])


def contents(cases):
    return [{n: getattr(c, n).clone() for n in ("k", "v", "k_scale", "v_scale") if getattr(c, n) is not None} for c in cases]


def same(x, y):
    return torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


@pytest.mark.parametrize("cache,dtype", [("16", BF16), ("16", F16), ("int8", BF16), ("e4m3", F16)])
@pytest.mark.parametrize("page,kv_heads,dim", [(16, 1, 64), (32, 8, 128), (128, 3, 64)])
def test_copy_pages(cache, dtype, page, kv_heads, dim):
    cases, caches = layers(cache, dtype, page, kv_heads, dim)
    n_pages = cases[0].n_pages
    order = random.Random(1).sample(range(n_pages), 6)
    moves = [(order[0], order[1], page), (-1, -1, 0), (order[0], order[2], 1), (order[3], order[4], page - 1), (order[3], order[5], 0)]
    want = contents(cases)
    for layer in want:
        for x in layer.values():
            for s, d, t in moves:
                if d >= 0:
                    x[d, :, :t] = x[s, :, :t].clone()
    cases[0].backend.copy_pages(caches, i32(moves))
    cases[0].backend.copy_pages(caches, torch.zeros(0, 3, dtype=torch.int32, device="cuda"))
    cases[0].backend.sync()
    for c, w in zip(cases, want):
        for name, x in w.items():
            assert same(getattr(c, name), x), name


@pytest.mark.parametrize("cache,dtype", [("16", BF16), ("16", F16), ("int8", F16), ("e4m3", BF16)])
@pytest.mark.parametrize("page,kv_heads,dim", [(16, 1, 64), (32, 8, 128), (64, 3, 64)])
def test_compact(cache, dtype, page, kv_heads, dim):
    cases, caches = layers(cache, dtype, page, kv_heads, dim)
    paths = [[0, 2, 3], [0], list(range(2, 20)), [1, 4, 5, 9, 15, 16, 17, 21, 31, 32], [], [2]]
    path = torch.full((len(LENS), 18), -7, dtype=torch.int32)
    for i, p in enumerate(paths):
        path[i, : len(p)] = torch.tensor(p, dtype=torch.int32)
    want = contents(cases)
    for layer, before in zip(want, contents(cases)):
        for name, x in layer.items():
            for i, ((q, kv), p) in enumerate(zip(LENS, paths)):
                cell = lambda place: (cases[0].table[i, place // page].item(), slice(None), place % page)        # noqa: E731
                for m, j in enumerate(p):
                    x[cell(kv - q + m)] = before[name][cell(kv - q + j)]
    cases[0].backend.compact(caches, cases[0].batch, path.cuda(), i32([len(p) for p in paths]))
    cases[0].backend.sync()
    for c, w in zip(cases, want):
        for name, x in w.items():
            assert same(getattr(c, name), x), name


def test_bad_moves_and_paths_move_nothing_and_are_reported():
    from paper_2603_20661_b200.binding import WwwsError
    cases, caches = layers("int8", BF16, 16, 2, 64, n=1)
    b, before = cases[0].backend, contents(cases)
    for moves, status in (([(cases[0].n_pages, 0, 3)], 8), ([(0, cases[0].n_pages, 3)], 8), ([(0, 1, 17)], 1), ([(-1, 1, 3)], 8)):
        b.copy_pages(caches, i32(moves))
        with pytest.raises(WwwsError) as e:
            b.sync()
        assert e.value.status == status
    none = [0] * len(LENS)
    for i, p in ((0, [0, 2, 2]), (0, [3, 1]), (0, [0, 5]), (1, [0, 1]), (0, [-1]), (4, [0])):
        path, n = torch.zeros(len(LENS), 3, dtype=torch.int32), list(none)
        path[i, : len(p)], n[i] = torch.tensor(p, dtype=torch.int32), len(p)
        b.compact(caches, cases[0].batch, path.cuda(), i32(n))
        with pytest.raises(WwwsError) as e:
            b.sync()
        assert e.value.status == 1
    for n in (-1, 4):
        b.compact(caches, cases[0].batch, torch.zeros(len(LENS), 3, dtype=torch.int32, device="cuda"), i32([n] + none[1:]))
        with pytest.raises(WwwsError):
            b.sync()
    for name, x in before[0].items():
        assert same(getattr(cases[0], name), x)


def test_more_layers_than_a_launch_holds():
    b = backend(16, 3, 1, 2)
    pools = [b.new_cache() for _ in range(70)]
    for i, c in enumerate(pools):
        c.tensors[0].fill_(float(i)), c.tensors[1].fill_(float(i))
        c.tensors[0][2].fill_(float(100 + i)), c.tensors[1][2].fill_(float(100 + i))
    b.copy_pages(b.caches(pools), i32([[2, 0, 5]]))
    batch = b.batch(i32([0, 4]), i32([16]), i32([[2]]), n_tokens=4, max_q_len=4, max_kv_len=16)
    for c in pools:
        c.tensors[0][2, :, 15].fill_(-1.0)
    b.compact(b.caches(pools), batch, i32([[3]]), i32([1]))
    b.sync()
    for i, c in enumerate(pools):
        assert (c.tensors[0][0, :, :5] == 100 + i).all() and (c.tensors[0][0, :, 5:] == i).all() and (c.tensors[0][1] == i).all()
        assert (c.tensors[0][2, :, 12] == -1.0).all() and (c.tensors[0][2, :, 13:15] == 100 + i).all()


def test_captured_and_replayed_and_on_another_stream():
    side = torch.cuda.Stream()
    b = backend(16, 40, 6, 8, stream=side)
    caches = b.caches([b.new_cache()])
    torch.cuda.synchronize()
    refs, table, held = i32([1, 1, 1] + [0] * 37), i32([[0, 1, 2, 0, 0, 0]]), i32([3])
    source, keep, room = i32([0, 0, 0]), i32([40, 33, 48]), i32([41, 41, 50])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = b.fork(refs, table, held, source, keep, room)
        b.copy_pages(caches, got[3])
    for k in ([40, 33, 48], [16, 40, 1]):
        keep.copy_(i32(k))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = fork_on_host(refs.tolist(), table.tolist(), [3], [0, 0, 0], k, [41, 41, 50], 16, 6)
        assert got[0].tolist() == want[0] and got[1].tolist() == want[1] and [tuple(m) for m in got[3].tolist()] == want[3]
    eager = b.fork(refs, table, held, source, keep, room)          # from the caller's stream, into the backend's
    b.sync()
    assert eager[0].tolist() == want[0]


def test_refusals():
    from paper_2603_20661_b200.binding import WwwsError
    b, other = backend(16, 12, 4, 2), backend(16, 12, 5, 2)
    refs, table, held, one = i32([0] * 12), i32([[0, 0, 0, 0]]), i32([0]), i32([0])
    for args in ((refs[:11], table, held, one, one, one), (refs, table[:, :3], held, one, one, one), (refs, table, i32([0, 0]), one, one, one), (refs, table, held, one, i32([0, 0]), one),
                 (refs, table, held, one, one, one.long()), (refs.float(), table, held, one, one, one), (refs, table.cpu(), held, one, one, one)):
        with pytest.raises(ValueError):
            b.fork(*args)
    with pytest.raises(WwwsError) as e:
        b.fork(refs, table, held, i32([0] * 3), i32([0] * 3), i32([0] * 3))
    assert e.value.status == 1 and "max_seqs" in str(e.value)
    caches = b.caches([b.new_cache()])
    with pytest.raises(ValueError):
        b.caches([backend(16, 13, 4, 2).new_cache()])
    with pytest.raises(ValueError):
        b.copy_pages(caches, i32([[0, 1]]))
    with pytest.raises(ValueError):
        b.copy_pages(b.new_cache(), i32([[0, 1, 1]]))
    batch = b.batch(i32([0, 1]), i32([1]), table, n_tokens=1, max_q_len=1, max_kv_len=1)
    with pytest.raises(ValueError):
        b.compact(caches, batch, i32([[0], [0]]), one)
    with pytest.raises(ValueError):
        b.compact(caches, other.batch(i32([0, 1]), i32([1]), i32([[0] * 5]), n_tokens=1, max_q_len=1, max_kv_len=1), i32([[0]]), one)
    with pytest.raises(WwwsError) as e:
        b.compact(caches, batch, torch.zeros(1, 2049, dtype=torch.int32, device="cuda"), one)
    assert "path_stride" in str(e.value)
    b.sync()
