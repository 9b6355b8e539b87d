"""One provider answers requests with several drafted tokens a step, or with several beams each.

The decoder of `answer_requests` with norms of queries and keys per head and positions turned into them (`Backend.rotate_append`).  With drafts, a step
takes for each request a tree of tokens that followed the last ones earlier in its own text, attends over the cache and the tree in one call
(`Backend.attend` with `tree`), keeps the path that the model agrees with, moves its keys and values together (`Backend.compact`) and gives the
pages behind them back (`Backend.fork`).  With beams, a step keeps the best continuations over all beams and the vocabulary
(`Backend.select_beams`), continues their sequences (`Backend.fork`) and copies the pages that two of them would write (`Backend.copy_pages`).

    python examples/answer_with_drafts.py [--cache int8] [--requests 8] [--beams 4]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from examples.answer_requests import Decoder  # noqa: E402


class TurningDecoder(Decoder):
    """A decoder whose queries and keys are normed per head and turned by their positions."""

    def rotation(self, backend):
        ones = self.torch.ones(self.dim, device=self.device)
        return backend.rotation(self.dim, theta=10000.0, q_weight=ones, k_weight=ones)

    def step(self, backend, rotation, caches, batch, tokens, positions=None, tree=None):
        """Logits after every one of the batch's new tokens."""
        norm = lambda x: x * (x.float().square().mean(-1, keepdim=True) + 1e-6).rsqrt().to(x.dtype)                     # noqa: E731
        x, n = self.embed[tokens], self.heads * self.dim
        for layer, cache in enumerate(caches):
            qkv = norm(x) @ self.qkv[layer]
            k, v = qkv[:, n:].unflatten(1, (2, self.kv_heads, self.dim)).unbind(1)
            q = backend.rotate_append(cache, batch, qkv[:, :n].unflatten(1, (self.heads, self.dim)), k, v, rotation, positions=positions)
            x = x + backend.attend(cache, batch, q, tree=tree).flatten(1) @ self.out[layer]
        return norm(x) @ self.head


def drafted_tree(text, most, width=3):
    """Tokens that may follow `text`, as a tree: the last token itself, then what came after earlier ones like it.  (tokens, parents)"""
    tokens, parents = [text[-1]], [-1]
    for at in [i for i, t in enumerate(text[:-1]) if t == text[-1]][-width:]:
        node = 0
        for t in text[at + 1 : at + 4]:
            same = [j for j in range(len(tokens)) if parents[j] == node and tokens[j] == t]
            if not same and len(tokens) == most:
                break
            if not same:
                tokens.append(t), parents.append(node)
            node = same[0] if same else len(tokens) - 1
    return tokens, parents


class Pages:
    """The sequences of a backend as `fork` keeps them: counts of the pool, page tables, lengths."""

    def __init__(self, backend, torch):
        self.backend, self.torch, dev = backend, torch, backend.device
        self.refs = torch.zeros(backend.n_pages, dtype=torch.int32, device=dev)
        self.table = torch.zeros(0, backend.max_pages, dtype=torch.int32, device=dev)
        self.held = torch.zeros(0, dtype=torch.int32, device=dev)

    def go_on(self, source, keep, room, caches=None):
        """New sequence i continues the first keep[i] tokens of source[i] with room for room[i]; copies pages that two would write."""
        to = lambda v: self.torch.as_tensor(v, dtype=self.torch.int32, device=self.refs.device)                        # noqa: E731
        self.refs, self.table, self.held, moves = self.backend.fork(self.refs, self.table, self.held, to(source), to(keep), to(room))
        if caches is not None:
            self.backend.copy_pages(caches, moves)


class Answers:
    """Requests answered over one backend: prompts first, then with drafts or with beams."""

    def __init__(self, model, prompts, most_new, beams=1, page=16, cache="16", drafts=16):
        from paper_2603_20661_b200.backend import Backend
        self.model, self.torch, self.prompts, self.most_new, self.beams, self.drafts = model, model.torch, prompts, most_new, beams, drafts
        n, longest = len(prompts) * beams, max(len(p) for p in prompts) + most_new + drafts
        per = -(-longest // page)
        self.backend = Backend(n_heads=model.heads, n_kv_heads=model.kv_heads, head_dim=model.dim, page_tokens=page, n_pages=2 * n * per, max_seqs=n,
                               max_tokens=max(n * drafts, sum(len(p) for p in prompts)), max_pages=per, max_rows=n, cache=cache, device=model.device)
        self.layers = [self.backend.new_cache() for _ in range(model.layers)]
        self.caches, self.rotation, self.pages = self.backend.caches(self.layers), model.rotation(self.backend), Pages(self.backend, self.torch)

    def _i32(self, v):
        return self.torch.as_tensor(v, dtype=self.torch.int32, device=self.model.device)

    def _batch(self, new, lengths):
        starts = np.concatenate([[0], np.cumsum(new)])
        return self.backend.batch(self._i32(starts), self._i32(lengths), self.pages.table, n_tokens=int(starts[-1]), max_q_len=max(new), max_kv_len=max(lengths)), starts

    def _prompts(self, prompts):
        """Logits after each prompt but for its last token, which the first step brings."""
        lengths = [len(p) - 1 for p in prompts]
        self.pages.go_on([-1] * len(prompts), [0] * len(prompts), lengths)
        batch, _ = self._batch(lengths, lengths)
        self.model.step(self.backend, self.rotation, self.layers, batch, self.torch.as_tensor([t for p in prompts for t in p[:-1]], device=self.model.device))
        return lengths

    def with_drafts(self):
        """Greedy answers, several tokens a step where the drafts are right: (answers, steps)."""
        torch = self.torch
        lengths, texts, steps = self._prompts(self.prompts), [list(p) for p in self.prompts], 0
        rows = list(range(len(texts)))                           # the request of each sequence; one that is answered leaves, and gives its pages back
        while True:
            source = [i for i, r in enumerate(rows) if len(texts[r]) - len(self.prompts[r]) < self.most_new]
            if not source:
                break
            rows, lengths = [rows[i] for i in source], [lengths[i] for i in source]
            trees = [drafted_tree(texts[r], self.drafts) for r in rows]
            new = [len(t) for t, _ in trees]
            self.pages.go_on(source, lengths, [c + q for c, q in zip(lengths, new)])
            batch, starts = self._batch(new, [c + q for c, q in zip(lengths, new)])
            masks, depth = np.zeros((starts[-1], -(-max(new) // 32)), np.uint32), np.zeros(starts[-1], np.int32)
            for i, (_, parents) in enumerate(trees):
                for j, p in enumerate(parents):
                    row = starts[i] + j
                    if p >= 0:
                        masks[row], depth[row] = masks[starts[i] + p], depth[starts[i] + p] + 1
                    masks[row, j // 32] |= np.uint32(1 << j % 32)
            positions = self._i32(np.repeat(lengths, new) + depth)
            logits = self.model.step(self.backend, self.rotation, self.layers, batch, torch.as_tensor([t for ts, _ in trees for t in ts], device=self.model.device), positions=positions,
                                     tree=torch.from_numpy(masks.view(np.int32)).to(self.model.device))
            best = logits.float().argmax(-1).tolist()
            paths = []
            for i, (tokens, parents) in enumerate(trees):
                path = [0]
                while True:
                    want = best[starts[i] + path[-1]]
                    follow = [j for j in range(len(tokens)) if parents[j] == path[-1] and tokens[j] == want]
                    texts[rows[i]].append(want)
                    if not follow:
                        break
                    path.append(follow[0])
                paths.append(path)
            most = max(len(p) for p in paths)
            self.backend.compact(self.caches, batch, self._i32([p + [0] * (most - len(p)) for p in paths]), self._i32([len(p) for p in paths]))
            lengths = [c + len(p) for c, p in zip(lengths, paths)]
            steps += 1
        self.backend.sync()
        return [t[len(p) : len(p) + self.most_new] for t, p in zip(texts, self.prompts)], steps

    def with_beams(self):
        """The best answer of each request by beam search, and its score."""
        torch, k, dev = self.torch, self.beams, self.model.device
        first = self._prompts(self.prompts)
        n = len(self.prompts) * k
        lengths = [c for c in first for _ in range(k)]
        source = [r for r in range(len(self.prompts)) for _ in range(k)]
        totals = torch.full((len(self.prompts), k), -float("inf"), device=dev)
        totals[:, 0] = 0.0                                       # the beams are still one and the same
        totals, tokens = totals.flatten(), torch.as_tensor([self.prompts[r][-1] for r in source], device=dev)
        answers = torch.zeros(n, 0, dtype=torch.long, device=dev)
        for _ in range(self.most_new):
            self.pages.go_on(source, lengths, [c + 1 for c in lengths], self.caches)
            batch, _ = self._batch([1] * n, [c + 1 for c in lengths])
            logits = self.model.step(self.backend, self.rotation, self.layers, batch, tokens)
            score, parent, token = self.backend.select_beams(logits, totals, beams=k, keep=k)
            source, totals, tokens = parent.flatten().clamp(min=0), score.flatten(), token.flatten().long().clamp(min=0)
            answers = torch.cat([answers[source.long()], tokens[:, None]], 1)
            lengths = [c + 1 for c in lengths]
        self.backend.sync()
        return answers.view(len(self.prompts), k, -1)[:, 0].tolist(), totals.view(-1, k)[:, 0].tolist()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--cache", choices=("16", "int8", "e4m3"), default="16")
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--most-new", type=int, default=48)
    a = ap.parse_args(argv)
    import torch
    model, rng = TurningDecoder(vocab=512), np.random.default_rng(0)
    prompts = [rng.integers(0, 64, rng.integers(20, 200)).tolist() for _ in range(a.requests)]
    torch.cuda.synchronize()
    t = time.perf_counter()
    drafted, steps = Answers(model, prompts, a.most_new, cache=a.cache).with_drafts()
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    best, scores = Answers(model, prompts, a.most_new, beams=a.beams, cache=a.cache).with_beams()
    torch.cuda.synchronize()
    print(f"{len(prompts)} requests, {a.most_new} tokens each: with drafts {steps} steps in {t1 - t:.2f} s, with {a.beams} beams {a.most_new} steps in {time.perf_counter() - t1:.2f} s; "
          f"best score {max(scores):.2f}")
    return drafted, best, scores


if __name__ == "__main__":
    main()
