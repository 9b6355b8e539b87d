"""The operators for drafts and beams together, as a provider uses them: what is in the cache after several steps of drafts accepted, or of beams
continued and dropped, is to the bit what the surviving text alone would have put there, and attention over it gives the same."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS, DIM, PAGE, VOCAB = 8, 2, 64, 16, 97
i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")        # noqa: E731


class World:
    """A backend of two layers over tables of queries, keys and values by token, so that a cached row follows from its token and its position alone."""

    def __init__(self, cache, max_seqs, max_tokens, seed):
        from paper_2603_20661_b200.backend import Backend
        g = torch.Generator("cuda").manual_seed(seed)
        self.b = Backend(n_heads=HEADS, n_kv_heads=KV_HEADS, head_dim=DIM, page_tokens=PAGE, n_pages=120, max_seqs=max_seqs, max_tokens=max_tokens, max_pages=9, max_rows=max_seqs, cache=cache, device="cuda")
        self.layers = [self.b.new_cache() for _ in range(2)]
        self.caches = self.b.caches(self.layers)
        self.tables = [[torch.randn(VOCAB, h, DIM, generator=g, device="cuda").to(torch.bfloat16) for h in (HEADS, KV_HEADS, KV_HEADS)] for _ in self.layers]
        weights = [1.0 + 0.2 * torch.randn(DIM, generator=g, device="cuda") for _ in range(2)]
        self.rotation = self.b.rotation(DIM, q_weight=weights[0], k_weight=weights[1])
        self.refs, self.table, self.held = torch.zeros(120, dtype=torch.int32, device="cuda"), torch.zeros(0, 9, dtype=torch.int32, device="cuda"), i32([])

    def fork(self, source, keep, room):
        self.refs, self.table, self.held, moves = self.b.fork(self.refs, self.table, self.held, i32(source), i32(keep), i32(room))
        self.b.copy_pages(self.caches, moves)

    def batch(self, new, lengths):
        starts = [sum(new[:i]) for i in range(len(new) + 1)]
        return self.b.batch(i32(starts), i32(lengths), self.table, n_tokens=starts[-1], max_q_len=max(new), max_kv_len=max(lengths))

    def write(self, batch, tokens, positions=None):
        """The new tokens' keys and values, in every layer; their queries, turned."""
        at = torch.tensor(tokens, device="cuda")
        return [self.b.rotate_append(c, batch, q[at], k[at], v[at], self.rotation, positions=positions) for c, (q, k, v) in zip(self.layers, self.tables)]

    def read(self, lengths):
        starts = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
        return [self.b.read(c, self.batch([0] * len(lengths), lengths), i32(starts), starts[-1]) for c in self.layers]


def check(world, texts, cache, seed):
    """The world's sequences hold `texts`, and nothing else is held; attention of one more token is that over a fresh backend with the texts alone."""
    fresh, n, lengths = World(cache, len(texts), 1000, seed), len(texts), [len(t) for t in texts]
    fresh.fork([-1] * n, [0] * n, [c + 1 for c in lengths])
    fresh.write(fresh.batch(lengths, lengths), [t for text in texts for t in text])
    world.fork(range(n), lengths, [c + 1 for c in lengths])
    for got, want in zip(world.read(lengths), fresh.read(lengths)):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    more = [c + 1 for c in lengths]
    for w in (world, fresh):
        batch = w.batch([1] * n, more)
        w.last = [w.b.attend(c, batch, q) for c, q in zip(w.layers, w.write(batch, [t[0] for t in texts]))]
        w.b.sync()
    assert all(torch.equal(x, y) for x, y in zip(world.last, fresh.last))
    pages = [p for row, h in zip(world.table.tolist(), world.held.tolist()) for p in row[:h]]
    assert world.refs.tolist() == [pages.count(p) for p in range(120)]
    world.fork([], [], [])
    world.b.sync()
    assert (world.refs == 0).all()


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
def test_drafts(cache):
    rng = random.Random(1)
    world = World(cache, 3, 300, 1)
    texts = [[rng.randrange(VOCAB) for _ in range(n)] for n in (5, 31, 48)]
    lengths = [len(t) for t in texts]
    world.fork([-1] * 3, [0] * 3, lengths)
    world.write(world.batch(lengths, lengths), [t for text in texts for t in text])
    for _ in range(6):
        new = [rng.randrange(1, 12) for _ in texts]
        parents = [[-1] + [rng.randrange(j) for j in range(1, q)] for q in new]
        tokens = [[rng.randrange(VOCAB) for _ in range(q)] for q in new]
        world.fork(range(3), lengths, [c + q for c, q in zip(lengths, new)])
        batch = world.batch(new, [c + q for c, q in zip(lengths, new)])
        masks, positions = [], []
        for c, ps in zip(lengths, parents):
            mine = []
            for j, p in enumerate(ps):
                mine.append((mine[p] if p >= 0 else 0) | 1 << j)
                positions.append(c + bin(mine[-1]).count("1") - 1)
            masks += [[m] for m in mine]
        queries = world.write(batch, [t for ts in tokens for t in ts], i32(positions))
        outs = [world.b.attend(c, batch, q, tree=i32(masks)) for c, q in zip(world.layers, queries)]
        assert all(torch.isfinite(o).all() for o in outs)
        # one path from the root is accepted: some node and its ancestors
        paths = []
        for ps in parents:
            node, path = rng.randrange(len(ps)), []
            while node >= 0:
                path.insert(0, node)
                node = ps[node]
            paths.append(path)
        most = max(len(p) for p in paths)
        world.b.compact(world.caches, batch, i32([p + [0] * (most - len(p)) for p in paths]), i32([len(p) for p in paths]))
        for text, ts, path in zip(texts, tokens, paths):
            text += [ts[j] for j in path]
        lengths = [len(t) for t in texts]
    world.b.sync()
    check(world, texts, cache, 1)


@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_beams(cache):
    g, beams, requests = torch.Generator("cuda").manual_seed(3), 4, 2
    rng = random.Random(2)
    world = World(cache, beams * requests, 300, 2)
    texts = [[rng.randrange(VOCAB) for _ in range(n)] for n in (17, 30)]
    world.fork([-1] * 2, [0] * 2, [17, 30])
    world.write(world.batch([17, 30], [17, 30]), texts[0] + texts[1])
    source, texts = [0] * beams + [1] * beams, [list(texts[i]) for i in [0] * beams + [1] * beams]
    totals = torch.zeros(beams * requests, device="cuda")
    for step in range(9):
        logits = 2.0 * torch.randn(beams * requests, VOCAB, generator=g, device="cuda")
        score, parent, token = world.b.select_beams(logits, totals, beams=beams, keep=beams)
        parent, token, totals = parent.flatten().tolist(), token.flatten().tolist(), score.flatten()
        source = [source[p] for p in parent] if step == 0 else parent
        texts = [list(texts[p]) for p in parent]
        lengths = [len(t) for t in texts]
        world.fork(source, lengths, [c + 1 for c in lengths])
        world.write(world.batch([1] * len(texts), [c + 1 for c in lengths]), token)
        for text, t in zip(texts, token):
            text.append(t)
    world.b.sync()
    check(world, texts, cache, 2)


def test_the_example_runs():
    from examples import answer_with_drafts
    drafted, best, scores = answer_with_drafts.main(["--requests", "3", "--beams", "3", "--most-new", "10", "--cache", "int8"])
    assert len(drafted) == len(best) == 3 and all(len(t) == 10 and all(0 <= x < 512 for x in t) for t in drafted + best)
    assert all(s <= 0.0 for s in scores)
