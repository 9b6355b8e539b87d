"""One provider of a simulated network answers the requests that were dispatched to it.

The simulator dispatches a batch of requests over a network of providers; this example takes the provider that got
the most of them and runs their token counts through a small decoder with random weights, the way a serving backend does:
prompts in chunks, then one token per request and step, all sequences together over one paged cache per layer
(`Backend.append`, `Backend.attend`), the next token from logits under a repetition penalty (`Backend.shape_logits`, a
temperature of zero).  Finished duels are judged under a mask that leaves three verdict tokens.  The measured rate stands
where `cap_true_tok_s` does in the simulator; here most of it is this script's lists and copies, not the operators.

    python examples/answer_requests.py [--cache int8] [--requests 24]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


class Decoder:
    """A decoder-only model of plain library products around the backend's operators (random weights)."""

    def __init__(self, vocab=4096, width=512, layers=2, heads=8, kv_heads=2, seed=0, device="cuda:0"):
        import torch
        g = torch.Generator(device).manual_seed(seed)
        self.torch, self.vocab, self.layers, self.heads, self.kv_heads, self.dim, self.device = torch, vocab, layers, heads, kv_heads, width // heads, device
        w = lambda *shape: (torch.randn(*shape, generator=g, device=device) * shape[0] ** -0.5).to(torch.bfloat16)      # noqa: E731
        self.embed = w(vocab, width) * vocab ** 0.5
        self.qkv = [w(width, (heads + 2 * kv_heads) * self.dim) for _ in range(layers)]
        self.out = [w(width, width) for _ in range(layers)]
        self.head = w(width, vocab)

    def step(self, backend, caches, batch, tokens, last):
        """Logits after the tokens `last` of the batch's new tokens."""
        norm = lambda x: x * (x.float().square().mean(-1, keepdim=True) + 1e-6).rsqrt().to(x.dtype)                     # noqa: E731
        x = self.embed[tokens]
        n = self.heads * self.dim
        for layer, cache in enumerate(caches):
            qkv = norm(x) @ self.qkv[layer]
            k, v = qkv[:, n:].unflatten(1, (2, self.kv_heads, self.dim)).unbind(1)
            backend.append(cache, batch, k, v)
            o = backend.attend(cache, batch, qkv[:, :n].unflatten(1, (self.heads, self.dim)))
            x = x + o.flatten(1) @ self.out[layer]
        return norm(x[last]) @ self.head


class Serving:
    """Sequences of one backend: their pages, lengths and tokens so far."""

    def __init__(self, model, prompts, most_new, page=32, cache="16", chunk=256):
        from paper_2603_20661_b200.backend import Backend
        torch = model.torch
        self.model, self.prompts, self.chunk, self.torch = model, prompts, chunk, torch
        n = len(prompts)
        need = [-(-(len(p) + most_new) // page) for p in prompts]
        self.backend = Backend(n_heads=model.heads, n_kv_heads=model.kv_heads, head_dim=model.dim, page_tokens=page, n_pages=sum(need), max_seqs=n,
                               max_tokens=max(n, n * chunk), max_pages=max(need), max_rows=n, dtype=torch.bfloat16, cache=cache, device=model.device)
        self.caches = [self.backend.new_cache() for _ in range(model.layers)]
        table = np.zeros((n, max(need)), np.int32)
        at = 0
        for i, k in enumerate(need):
            table[i, :k] = np.arange(at, at + k)
            at += k
        self.table = torch.from_numpy(table).to(model.device)
        self.done = [0] * n                      # tokens of each sequence in the cache
        self.answers = [[] for _ in range(n)]

    def _run(self, new):
        """One step over new tokens ({sequence: tokens}): logits after each sequence's last one."""
        torch, dev = self.torch, self.model.device
        n = len(self.prompts)
        q = [len(new.get(i, ())) for i in range(n)]
        for i in range(n):
            self.done[i] += q[i]
        starts = np.concatenate([[0], np.cumsum(q)]).astype(np.int32)
        to = lambda a: torch.as_tensor(a, dtype=torch.int32, device=dev)                                                # noqa: E731
        batch = self.backend.batch(to(starts), to(self.done), self.table, n_tokens=int(starts[-1]), max_q_len=max(q), max_kv_len=max(self.done))
        tokens = torch.as_tensor([t for i in range(n) for t in new.get(i, ())], dtype=torch.long, device=dev)
        rows = [i for i in range(n) if q[i]]
        last = torch.as_tensor([int(starts[i + 1]) - 1 for i in rows], device=dev)
        return rows, self.model.step(self.backend, self.caches, batch, tokens, last)

    def _next(self, rows, logits):
        """The next token of each row under a repetition penalty."""
        torch, dev = self.torch, self.model.device
        text = [list(self.prompts[i]) + self.answers[i] for i in rows]
        to = lambda a, t: torch.as_tensor(a, dtype=t, device=dev)                                                        # noqa: E731
        shaping = self.backend.shaping(history=to([t for s in text for t in s], torch.int32),
                                       history_start=to(np.concatenate([[0], np.cumsum([len(s) for s in text])]), torch.int32),
                                       prompt_len=to([len(self.prompts[i]) for i in rows], torch.int32),
                                       repetition=to([1.1] * len(rows), torch.float32), frequency=to([0.05] * len(rows), torch.float32))
        _, token = self.backend.shape_logits(logits, shaping)
        for i, t in zip(rows, token.tolist()):
            self.answers[i].append(t)

    def answer(self, n_new):
        """Prompts in chunks, then steps of one token until sequence i has n_new[i]; returns the last logits of each sequence."""
        logits_of = {}
        while any(self.done[i] < len(p) for i, p in enumerate(self.prompts)):
            new = {i: p[self.done[i] : self.done[i] + self.chunk] for i, p in enumerate(self.prompts) if self.done[i] < len(p)}
            rows, logits = self._run(new)
            ready = [k for k, i in enumerate(rows) if self.done[i] == len(self.prompts[i])]
            if ready:
                logits_of.update({rows[k]: logits[k] for k in ready})
                self._next([rows[k] for k in ready], logits[ready])
        while True:
            rows = [i for i, a in enumerate(self.answers) if len(a) < n_new[i]]
            if not rows:
                break
            rows, logits = self._run({i: self.answers[i][-1:] for i in rows})
            logits_of.update({i: logits[k] for k, i in enumerate(rows)})
            self._next(rows, logits)
        self.backend.sync()
        return logits_of

    def verdicts(self, logits, choices):
        """A judge's verdict per row: the best of a few tokens, under a mask that leaves no other."""
        torch, dev = self.torch, self.model.device
        words = np.zeros((1, -(-self.model.vocab // 32)), np.uint32)
        for t in choices:
            words[0, t // 32] |= np.uint32(1 << (t % 32))
        shaping = self.backend.shaping(mask=torch.from_numpy(words.view(np.int32)).to(dev), mask_index=torch.zeros(len(logits), dtype=torch.int32, device=dev))
        _, token = self.backend.shape_logits(logits, shaping)
        self.backend.sync()
        return [choices.index(t) for t in token.tolist()]


def dispatched(n_requests, seed=0):
    """Token counts (prompt, answer) of the requests that the simulator sends to its busiest provider, and how many duels it judged."""
    from paper_2603_20661_b200 import synth
    from paper_2603_20661_b200.binding import Network
    wl = synth.make_workload("tiers64", n_replicas=1, n_requests=4000, n_peers=64, seed=seed)
    net = Network(wl.settings, wl.peers, wl.batch)
    net.bind_requests(wl.requests)
    for s in range(min(wl.n_steps, 4)):
        net.step(s * wl.batch, wl.batch, wl.step_now_ms(s), s % wl.gossip_every == 0)
    res, n = net.results(), min(wl.n_steps, 4) * wl.batch
    who = res["exec_a"][0, :n]
    peer = int(np.bincount(who[who >= 0], minlength=64).argmax())
    mine = np.flatnonzero(who == peer)[:n_requests]
    duels = int(np.isin(res["judges"][0, :n], peer).any(-1).sum())
    net.close()
    return peer, [(int(wl.requests["len_in"][0, i]), int(wl.requests["len_out"][0, i])) for i in mine], duels


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--cache", choices=("16", "int8", "e4m3"), default="int8")
    ap.add_argument("--requests", type=int, default=24)
    ap.add_argument("--most-new", type=int, default=64, help="answers are cut at this many tokens")
    a = ap.parse_args(argv)
    import torch
    model = Decoder()
    peer, lengths, duels = dispatched(a.requests)
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, model.vocab, n_in).tolist() for n_in, _ in lengths]
    n_new = [min(n_out, a.most_new) for _, n_out in lengths]
    serving = Serving(model, prompts, a.most_new, cache=a.cache)
    torch.cuda.synchronize()
    t = time.perf_counter()
    logits = serving.answer(n_new)
    torch.cuda.synchronize()
    seconds = time.perf_counter() - t
    total = sum(len(p) for p in prompts) + sum(n_new)
    verdicts = serving.verdicts(torch.stack([logits[i] for i in sorted(logits)])[: max(1, min(duels, len(logits)))], [11, 12, 13])
    print(f"provider {peer}: {len(prompts)} requests, {total} tokens in {seconds:.2f} s = {total / seconds:.0f} tokens/s (what cap_true_tok_s stands for); "
          f"verdicts {[('first', 'second', 'draw')[v] for v in verdicts[:4]]}")
    return serving


if __name__ == "__main__":
    main()
