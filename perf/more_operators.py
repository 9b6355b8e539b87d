"""Cases of the serving-backend operators for drafts and beams: what is measured, their plain form, and their values in 64 bits.

A case is one call (or the calls of one step) as a peer of the network makes it while it answers requests with several drafted tokens or
several hypotheses each:
  rotate   queries and keys of new tokens normed per head and turned by their positions, in one pass
  append   the same with the keys and values written to the paged cache in that pass
  tree     attention of a tree of drafted tokens over the paged cache
  fork     sequences continued, dropped and given room: their page tables, and the copies of pages that two would write, in every layer
  compact  accepted tokens of a tree moved together, in every layer
  beams    the best continuations over a request's beams and the vocabulary
Lengths follow the request streams of `synth` (lognormal, sigma 0.8, clipped at 8,192 tokens) where a case is ragged.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
TOP = {"int8": 127.0, "e4m3": 448.0}        # largest code of a quantised cache
TINY = 2.0 ** -100                           # rows whose largest magnitude is below this are held as zeros
EPS = 1e-6


def listed():
    rotate = {"mix": 1, "axes": 1, "turned": 128, "interleaved": False, "normed": True, "theta": 1000000.0, "far": 0}
    tree = {"op": "tree", "mix": 1, "window": 0, "sinks": 0}
    pages = {"mix": 1, "ended": 0.0}
    beams = {"op": "beams", "mix": 1, "first": False}
    return [
        # the smallest call: the next token of one request
        dict(rotate, op="append", name="append_one", seqs=1, q=1, kv=301, ragged=False, heads=16, kv_heads=4, dim=64, turned=64, page=16, dtype="f16", cache="16", normed=False, theta=10000.0),
        # newly dispatched prompts of mixed lengths, to a cache of 8 bits
        dict(rotate, op="append", name="append_prompts", seqs=24, q=0, kv=900, ragged=True, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16", cache="int8"),
        # patches of a few pictures and clips, whose positions have a time, a row and a column
        dict(rotate, op="rotate", name="rotate_axes", seqs=6, q=4097, kv=4097, ragged=False, heads=28, kv_heads=4, dim=128, turned=96, dtype="f16", axes=3, interleaved=True),
        # a few drafted tokens of one request
        dict(tree, name="tree_one", seqs=1, q=8, kv=509, ragged=False, heads=16, kv_heads=4, dim=64, page=16, dtype="f16", cache="16"),
        # an ordinary step of a busy peer that drafts
        dict(tree, name="tree_batch", seqs=24, q=21, kv=3001, ragged=True, heads=32, kv_heads=8, dim=128, page=32, dtype="bf16", cache="e4m3"),
        # wide trees behind long contexts
        dict(tree, name="tree_wide", seqs=12, q=61, kv=16001, ragged=False, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16", cache="16"),
        # one request with a few beams
        dict(pages, op="fork", name="fork_one", seqs=1, beams=4, kv=333, ragged=False, kv_heads=4, dim=64, page=16, layers=2, dtype="f16", cache="16"),
        # a step of many requests with beams, some of them answered
        dict(pages, op="fork", name="fork_batch", seqs=48, beams=5, kv=1200, ragged=True, kv_heads=8, dim=128, page=32, layers=6, dtype="bf16", cache="16", ended=0.1),
        # accepted drafts of a batch moved to their places
        dict(pages, op="compact", name="compact_batch", seqs=96, q=61, kv=700, ragged=True, kv_heads=8, dim=128, page=32, layers=8, dtype="bf16", cache="e4m3"),
        # the first token of one request's beams: all but one of them are still empty
        dict(beams, name="beams_first", seqs=1, beams=4, keep=8, vocab=32003, dtype="f32", first=True),
        # many beams of a few requests
        dict(beams, name="beams_many", seqs=8, beams=32, keep=64, vocab=50021, dtype="f16"),
        # a step of a large batch
        dict(beams, name="beams_batch", seqs=64, beams=4, keep=8, vocab=131072, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "append", "tree", "tree", "fork", "compact", "beams", "beams"])
    case = {"op": op, "mix": rng.randrange(1, 1 << 20)}
    if op == "beams":
        beams, vocab = rng.choice([1, 2, 3, 4, 5, 8, 16, 32]), _log(rng, 500, 131072)
        seqs = max(1, min(_log(rng, 1, 64), 256 // beams))
        return dict(case, seqs=seqs, beams=beams, keep=rng.choice([beams, 2 * beams, 2 * beams + 1]), vocab=vocab, dtype=rng.choice(["f32", "bf16", "f16"]) if seqs * beams * vocab < 16000000 else "bf16",
                    first=rng.random() < 0.3)
    kv_heads = rng.choice([1, 2, 4, 8])
    case.update(ragged=rng.random() < 0.6, heads=kv_heads * rng.choice([1, 2, 4, 5, 7, 8]), kv_heads=kv_heads, dim=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]),
                dtype=rng.choice(["bf16", "f16"]))
    if op in ("rotate", "append"):
        cache = rng.choice(["16", "16", "int8", "e4m3"])
        new = _log(rng, 1, 4096)
        seqs = max(1, min(_log(rng, 1, 128), 16000 // (new * (2 if case["ragged"] else 1))))
        # sequences whose whole length is new, or some tokens behind what a 16-bit cache holds
        case.update(seqs=seqs, cache=cache, normed=rng.random() < 0.6, theta=rng.choice([10000.0, 500000.0, 1000000.0]), turned=rng.choice([16, 32, 48, 64, 96, 128][: 4 if case["dim"] == 64 else 6]),
                    interleaved=rng.random() < 0.4, axes=rng.choice([1, 1, 2, 3]), far=0)
        behind = op == "append" and cache == "16" and rng.random() < 0.7
        case.update(q=new if behind else 0, kv=new + _log(rng, 1, 4000) if behind else new)
        if rng.random() < 0.3:
            case["far"] = _log(rng, 1000, 1 << 24)               # positions start far out
        return case
    case["cache"] = rng.choice(["16", "int8", "e4m3"]) if op == "tree" else rng.choice(["16", "e4m3"])
    if op == "tree":
        q, kv = rng.randrange(2, 65), _log(rng, 80, 16384)
        windowed = rng.random() < 0.3
        case.update(seqs=max(1, min(_log(rng, 1, 48), 100000 // kv)), q=q, kv=max(q, kv), window=_log(rng, 70, 4096) if windowed else 0, sinks=rng.choice([0, 1, 4, 16]) if windowed else 0)
    elif op == "fork":
        beams, layers = rng.choice([1, 2, 3, 4, 5, 8]), _log(rng, 1, 8)
        case.update(beams=beams, layers=layers, kv=_log(rng, 20, 4000), ended=rng.choice([0.0, 0.1, 0.3]))
        case["seqs"] = max(1, min(_log(rng, 1, 64), 800000 // (case["kv"] * beams * layers)))
    else:
        layers, kv = _log(rng, 1, 8), _log(rng, 80, 4000)
        case.update(seqs=max(1, min(_log(rng, 1, 96), 800000 // (kv * layers))), q=rng.randrange(2, 65), kv=kv, layers=layers, ended=0.0)
    return case


def _lengths(case):
    """Per sequence (new tokens, tokens in the cache after them); the case alone decides. q = 0: the whole sequence is new."""
    rng = random.Random(case["mix"])
    got = []
    for _ in range(case["seqs"]):
        kv = case["kv"]
        if case["ragged"]:
            kv = max(1, min(8192, 2 * case["kv"], int(kv * math.exp(rng.gauss(0.0, 0.8)))))
        q = kv if case["q"] == 0 else min(case["q"], kv)
        got.append((q, kv))
    return got


def _trees(case):
    """Per sequence, per drafted token: the whole number whose bit j says that the token sees drafted token j (its ancestors and itself)."""
    rng = random.Random(case["mix"] + 1)
    got = []
    for q, _ in _lengths(case):
        bits = []
        for t in range(q):
            # drafts grow in depth more often than in breadth
            parent = -1 if t == 0 or rng.random() < 0.05 else t - 1 if rng.random() < 0.4 else rng.randrange(t)
            bits.append((bits[parent] if parent >= 0 else 0) | 1 << t)
        got.append(bits)
    return got


def _paths(case):
    """Per sequence: places of the accepted drafted tokens among the drafted ones, ascending; none of them lies where another one goes."""
    rng = random.Random(case["mix"] + 2)
    got = []
    for q, _ in _lengths(case):
        n = min(rng.choice([1, 2, 3, 4, 4, 5, 6, 8]), q // 2)
        got.append([0] * (n > 0) + sorted(rng.sample(range(n, q), n - 1) if n > 1 else []))
    return got


def _beams(case):
    """Sequences with beams before the step: per request (length, pages all beams share, pages held by each), and what each new beam continues."""
    rng = random.Random(case["mix"])
    requests, source = [], []
    for r in range(case["seqs"]):
        kv = case["kv"]
        if case["ragged"]:
            kv = max(1, min(8192, 2 * case["kv"], int(kv * math.exp(rng.gauss(0.0, 0.8)))))
        shared = int(kv * rng.uniform(0.3, 0.9)) // case["page"]
        requests.append((kv, shared, -(-kv // case["page"])))
        ended = rng.random() < case["ended"]
        for _ in range(case["beams"]):
            # the better beams are continued more often
            source.append(-1 if ended else r * case["beams"] + min(rng.randrange(case["beams"]), rng.randrange(case["beams"])))
    return requests, source


def _quantise(x, kind):
    """Codes and scales of rows of `x` (f32, [..., dim]): one scale per row."""
    amax = x.abs().amax(-1, keepdim=True)
    scale = torch.where(amax < TINY, torch.zeros_like(amax), amax * torch.tensor(1.0 / TOP[kind], device=x.device))
    inv = torch.where(scale > 0, torch.ones_like(scale) / scale, torch.zeros_like(scale))
    y = (x * inv).clamp(-TOP[kind], TOP[kind])
    code = torch.round(y).to(torch.int8) if kind == "int8" else y.to(torch.float8_e4m3fn)
    return code, scale.squeeze(-1)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _ends(v):
    return [sum(v[:i]) for i in range(len(v) + 1)]


def _frequencies(case):
    return [case["theta"] ** (-2.0 * i / case["turned"]) for i in range(case["turned"] // 2)]


def _axis_of(case):
    """The axis that pair i turns by: the axes share the pairs out in order, the first ones taking what does not divide."""
    n = case["turned"] // 2
    return [i * case["axes"] // n for i in range(n)]


def _pool(case, n_pages, g, names=("k", "v")):
    """Pages and scales of one layer, as written by served sequences: rows of different magnitudes."""
    s = {}
    for name in names:
        x = torch.randn(n_pages, case["kv_heads"], case["page"], case["dim"], generator=g, device="cuda").to(DTYPES[case["dtype"]])
        if case["cache"] == "16":
            s[name + "_pages"], s[name + "_scale"] = x, None
        else:
            s[name + "_pages"], s[name + "_scale"] = _quantise(x.float() * torch.exp(0.3 * torch.randn(n_pages, case["kv_heads"], case["page"], 1, generator=g, device="cuda")), case["cache"])
    return s


def _prepare_beams(case, g):
    rows = case["seqs"] * case["beams"]
    s = {"case": case, "logits": (torch.randn(rows, case["vocab"], generator=g, device="cuda") * 3.0).to(DTYPES[case["dtype"]])}
    totals = -4.0 * torch.rand(rows, generator=g, device="cuda")
    if case["first"]:
        totals.view(case["seqs"], case["beams"])[:, 1:] = -math.inf
        totals.view(case["seqs"], case["beams"])[:, 0] = 0.0
    s["totals"] = totals
    if own:
        from paper_2603_20661_b200.backend import Backend
        s["backend"] = Backend(max_rows=rows, device="cuda")
    return s


def _prepare_fork(case, g):
    requests, source = _beams(case)
    beams, page = case["beams"], case["page"]
    most = max(held for _, _, held in requests) + 1
    table = np.zeros((len(source), most), np.int64)
    held = np.repeat([h for _, _, h in requests], beams)
    at = 0
    for r, (_, shared, h) in enumerate(requests):
        rows = slice(r * beams, (r + 1) * beams)
        table[rows, :shared] = np.arange(at, at + shared)
        at += shared
        table[rows, shared:h] = np.arange(at, at + beams * (h - shared)).reshape(beams, -1)
        at += beams * (h - shared)
    n_pages = at + 2 * len(source) + 5
    order = torch.randperm(n_pages, generator=g, device="cuda")
    mine = torch.arange(most, device="cuda") < torch.tensor(held, device="cuda")[:, None]
    table = torch.where(mine, order[torch.tensor(table, device="cuda")], torch.zeros((), dtype=torch.int64, device="cuda"))
    refs = torch.bincount(table[mine], minlength=n_pages)
    length = np.repeat([kv for kv, _, _ in requests], beams)
    keep = [int(length[j]) if j >= 0 else 0 for j in source]
    s = {"case": case, "n_pages": n_pages, "most": most, "refs": refs.to(torch.int32), "table": table.to(torch.int32), "held": _i32(held.tolist()), "source": _i32(source), "keep": _i32(keep),
         "room": _i32([k + 1 if j >= 0 else 0 for k, j in zip(keep, source)]), "layers": [_pool(case, n_pages, g) for _ in range(case["layers"])]}
    if own:
        from paper_2603_20661_b200.backend import Backend
        s["backend"] = b = Backend(n_heads=case["kv_heads"], n_kv_heads=case["kv_heads"], head_dim=case["dim"], page_tokens=page, n_pages=n_pages, max_seqs=len(source), max_tokens=len(source),
                                   max_pages=most, dtype=DTYPES[case["dtype"]], cache=case["cache"], device="cuda")
        s["caches"] = b.caches([b.bind_cache(x["k_pages"], x["v_pages"], x["k_scale"], x["v_scale"]) for x in s["layers"]])
    return s


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    if case["op"] == "beams":
        return _prepare_beams(case, g)
    if case["op"] == "fork":
        return _prepare_fork(case, g)
    dtype = DTYPES[case["dtype"]]
    lens = _lengths(case)
    kv_heads, dim = case["kv_heads"], case["dim"]
    heads = case.get("heads", kv_heads)
    tokens, max_q, max_kv = sum(q for q, _ in lens), max(q for q, _ in lens), max(kv for _, kv in lens)
    s = {"case": case, "tokens": tokens, "max_q": max_q, "max_kv": max_kv, "q_start": _i32(_ends([q for q, _ in lens])), "kv_len": _i32([kv for _, kv in lens])}
    if case["op"] != "compact":
        # queries, keys and values come as slices of one projection's output
        qkv = torch.randn(tokens, (heads + 2 * kv_heads) * dim, generator=g, device="cuda").to(dtype)
        s["q"] = qkv[:, : heads * dim].view(tokens, heads, dim)
        s["k"] = qkv[:, heads * dim : (heads + kv_heads) * dim].view(tokens, kv_heads, dim)
        s["v"] = qkv[:, (heads + kv_heads) * dim :].view(tokens, kv_heads, dim)
    if case["op"] in ("rotate", "append"):
        if case["normed"]:
            s["q_weight"], s["k_weight"] = (1.0 + 0.2 * torch.randn(dim, generator=g, device="cuda") for _ in range(2))
        else:
            s["q_weight"] = s["k_weight"] = None
        if case["op"] == "rotate" or case["axes"] > 1 or case["far"]:
            # time moves on from sequence to sequence, rows and columns of patches within one
            place = torch.cat([torch.arange(kv - q, kv, device="cuda") for q, kv in lens])
            side = max(1, int(math.isqrt(max_q)))
            s["positions"] = torch.stack([place if case["axes"] == 1 else place // (side * side) if a == 0 else place // side % side if a == 1 else place % side
                                          for a in range(case["axes"])], -1).add_(case["far"]).to(torch.int32)
        else:
            s["positions"] = None                                # the tokens' places in their sequences
    if case["op"] != "rotate":
        page = case["page"]
        # (a sequence that only gains tokens needs no page of what it held before)
        first = [(kv - q) // page if case["op"] == "append" else 0 for q, kv in lens]
        last = [-(-kv // page) for _, kv in lens]
        n_pages = sum(last) - sum(first) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        s["page_table"] = torch.zeros(len(lens), max(last), dtype=torch.int32, device="cuda")
        at = 0
        for i, (lo, hi) in enumerate(zip(first, last)):
            s["page_table"][i, lo:hi] = order[at : at + hi - lo]
            at += hi - lo
    if case["op"] == "compact":
        s["layers"] = [_pool(case, n_pages, g) for _ in range(case["layers"])]
        paths = _paths(case)
        most = max(1, max(len(p) for p in paths))
        s["path"], s["path_len"] = _i32([p + [0] * (most - len(p)) for p in paths]), _i32([len(p) for p in paths])
    elif case["op"] != "rotate":
        s.update(_pool(case, n_pages, g))
    if case["op"] == "tree":
        words = (max_q + 31) // 32
        s["tree"] = torch.tensor(np.array([[b >> 32 * w & 0xFFFFFFFF for w in range(words)] for seq in _trees(case) for b in seq], np.uint32).view(np.int32), device="cuda")
    if case["op"] == "append":
        s["kv_start"], s["total_kv"] = _i32(_ends([kv for _, kv in lens])), sum(kv for _, kv in lens)
    if own:
        from paper_2603_20661_b200.backend import Backend
        paged = case["op"] != "rotate"
        s["backend"] = b = Backend(n_heads=heads, n_kv_heads=kv_heads, head_dim=dim, page_tokens=case["page"] if paged else 16, n_pages=n_pages if paged else 1, max_seqs=len(lens), max_tokens=tokens,
                                   max_pages=s["page_table"].shape[1] if paged else 1, dtype=dtype, cache=case["cache"] if paged else "16", device="cuda")
        if paged:
            s["batch"] = b.batch(s["q_start"], s["kv_len"], s["page_table"], n_tokens=tokens, max_q_len=max_q, max_kv_len=max_kv)
            if case["op"] == "compact":
                s["caches"] = b.caches([b.bind_cache(x["k_pages"], x["v_pages"], x["k_scale"], x["v_scale"]) for x in s["layers"]])
            else:
                s["cache"] = b.bind_cache(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"])
        if case["op"] in ("rotate", "append"):
            s["rotation"] = b.rotation(case["turned"], frequencies=_frequencies(case), axes=_axis_of(case), interleaved=case["interleaved"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS)
    return s


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"rotate": _plain_rotate, "append": _plain_append, "tree": _plain_tree, "fork": _plain_fork, "compact": _plain_compact, "beams": _plain_beams}[op](s)
    b = s["backend"]
    if op == "rotate":
        return b.rotate(s["q"], s["k"], s["positions"], s["rotation"])
    if op == "append":
        q = b.rotate_append(s["cache"], s["batch"], s["q"], s["k"], s["v"], s["rotation"], positions=s["positions"])
        if s["case"]["cache"] == "16":
            return q, s["k_pages"], s["v_pages"]
        return (q, *b.read(s["cache"], s["batch"], s["kv_start"], s["total_kv"]))
    if op == "tree":
        return b.attend(s["cache"], s["batch"], s["q"], window=s["case"]["window"], sinks=s["case"]["sinks"], tree=s["tree"])
    if op == "fork":
        refs, table, held, moves = b.fork(s["refs"], s["table"], s["held"], s["source"], s["keep"], s["room"])
        b.copy_pages(s["caches"], moves)
        return [refs, table, held, moves] + _layers(s)
    if op == "compact":
        b.compact(s["caches"], s["batch"], s["path"], s["path_len"])
        return _layers(s)
    return b.select_beams(s["logits"], s["totals"], beams=s["case"]["beams"], keep=s["case"]["keep"])


def _layers(s):
    return [x[name] for x in s["layers"] for name in ("k_pages", "v_pages", "k_scale", "v_scale") if x[name] is not None]


def _token_of(s):
    """Of each new token: its sequence, its place among the sequence's new tokens, its position in the sequence."""
    start, kv = s["q_start"].long(), s["kv_len"].long()
    t = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(start, t, right=True) - 1
    place = t - start[seq]
    return seq, place, kv[seq] - (start[seq + 1] - start[seq]) + place


def _plain_turned(s):
    """Queries and keys after norm and rotation, in 32 bits (angles in 64)."""
    case = s["case"]
    pos = s["positions"].double() if s["positions"] is not None else _token_of(s)[2].double()[:, None]
    turn = pos[:, _axis_of(case) if s["positions"] is not None else [0] * (case["turned"] // 2)] * torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    cos, sin = turn.cos().float()[:, None], turn.sin().float()[:, None]
    got = []
    for name in ("q", "k"):
        x, n = s[name].float(), case["turned"]
        if s[name + "_weight"] is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * s[name + "_weight"]
        y = x.clone()
        first, second = (slice(0, n, 2), slice(1, n, 2)) if case["interleaved"] else (slice(0, n // 2), slice(n // 2, n))
        y[..., first] = x[..., first] * cos - x[..., second] * sin
        y[..., second] = x[..., second] * cos + x[..., first] * sin
        got.append(y)
    return got


def _plain_rotate(s):
    return [x.to(s["q"].dtype) for x in _plain_turned(s)]


def _plain_append(s):
    case, dtype = s["case"], s["q"].dtype
    q, k = _plain_turned(s)
    seq, _, pos = _token_of(s)
    page, slot = s["page_table"].long()[seq, pos // case["page"]], pos % case["page"]
    if case["cache"] == "16":
        s["k_pages"][page, :, slot], s["v_pages"][page, :, slot] = k.to(dtype), s["v"]
        return q.to(dtype), s["k_pages"], s["v_pages"]
    got = []
    for name, x in (("k", k), ("v", s["v"].float())):
        code, scale = _quantise(x, case["cache"])
        s[name + "_pages"].view(torch.int8)[page, :, slot] = code.view(torch.int8)
        s[name + "_scale"][page, :, slot] = scale
        code = s[name + "_pages"].view(torch.int8)[page, :, slot].view(s[name + "_pages"].dtype)       # (here every token of the sequences is new)
        got.append((code.float() * s[name + "_scale"][page, :, slot].unsqueeze(-1)).to(dtype))
    return (q.to(dtype), *got)


def _plain_rows(s, name):
    """The cached rows of every sequence, padded: f32 [seqs, kv_heads, max_kv, dim]."""
    table = s["page_table"].long()
    x = s[name + "_pages"][table].float()
    if s[name + "_scale"] is not None:
        x = x * s[name + "_scale"][table].unsqueeze(-1)
    n, pages, h, p, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(n, h, pages * p, d)[:, :, : s["max_kv"]]


def _plain_tree(s):
    case, q = s["case"], s["q"]
    n, heads, kv_heads, dim, max_q, max_kv = len(s["kv_len"]), case["heads"], case["kv_heads"], case["dim"], s["max_q"], s["max_kv"]
    group = heads // kv_heads
    seq, place, _ = _token_of(s)
    qp = torch.zeros(n, max_q, heads, dim, device="cuda")
    qp[seq, place] = q.float()
    qp = qp.view(n, max_q, kv_heads, group, dim).permute(0, 2, 1, 3, 4).reshape(n, kv_heads, max_q * group, dim)
    x = (qp @ _plain_rows(s, "k").transpose(-1, -2)).mul_(dim ** -0.5)
    at = torch.arange(max_q, device="cuda")
    bits = ((s["tree"].long()[:, at // 32] >> (at % 32)) & 1).bool()                   # [tokens, drafted tokens]
    drafted = torch.zeros(n, max_q, max_q, dtype=torch.bool, device="cuda")
    drafted[seq, place] = bits & (at <= place[:, None])
    context = (s["kv_len"] - (s["q_start"][1:] - s["q_start"][:-1])).long()
    j = torch.arange(max_kv, device="cuda")
    rel = j - context[:, None]                                                          # place among the drafted tokens
    among = (rel >= 0) & (rel < max_q)
    seen = torch.gather(drafted, 2, rel.clamp(0, max_q - 1)[:, None, :].expand(n, max_q, max_kv)) & among[:, None]
    held = (rel < 0)[:, None].expand(n, max_q, max_kv)
    if case["window"]:
        pos = context[:, None] + drafted.sum(-1) - 1                                    # where the token would stand in its sequence
        held = held & ((j > pos[..., None] - case["window"]) | (j < case["sinks"]))
    x.view(n, kv_heads, max_q, group, max_kv).masked_fill_(~(seen | held)[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x @ _plain_rows(s, "v")) / torch.where(total == 0, torch.ones_like(total), total)
    o = o.view(n, kv_heads, max_q, group, dim).permute(0, 2, 1, 3, 4).reshape(n, max_q, heads, dim)
    return o[seq, place].to(q.dtype)


def _plain_fork(s):
    case, n_pages, most, page = s["case"], s["n_pages"], s["most"], s["case"]["page"]
    table, source, keep = s["table"].long(), s["source"].long(), s["keep"].long()
    n, k = len(source), torch.arange(most, device="cuda")
    refs = s["refs"].long()
    refs.index_add_(0, table.reshape(-1), -(k < s["held"][:, None]).long().reshape(-1))
    rows, full = table[source.clamp(min=0)], torch.where(source >= 0, keep // page, 0)
    whole = k < full[:, None]
    refs.index_add_(0, rows.reshape(-1), whole.long().reshape(-1))
    # the page that `keep` ends inside stays with its first claimant, unless somebody holds it whole
    cut = (source >= 0) & (keep % page > 0)
    end = rows.gather(1, full.clamp(max=most - 1)[:, None])[:, 0]
    i = torch.arange(n, device="cuda")
    first = torch.full((n_pages,), n, device="cuda").scatter_reduce_(0, end, torch.where(cut, i, n), "amin")
    stays = cut & (refs[end] == 0) & (first[end] == i)
    refs.index_add_(0, end, stays.long())
    held = torch.where(source >= 0, (torch.maximum(s["room"].long(), keep) + page - 1) // page, (s["room"].long() + page - 1) // page)
    fresh = (k >= full[:, None]) & (k < held[:, None]) & ~(stays[:, None] & (k == full[:, None]))
    free = torch.nonzero(refs == 0)[:, 0]
    rank = (fresh.reshape(-1).long().cumsum(0) - 1).view(n, most)
    new = torch.where(whole | (stays[:, None] & (k == full[:, None])), rows, 0)
    new = torch.where(fresh, free[rank.clamp(0, len(free) - 1)], new)
    refs.index_add_(0, new.reshape(-1), fresh.long().reshape(-1))
    copied = cut & ~stays
    to = new.gather(1, full.clamp(max=most - 1)[:, None])[:, 0]
    moves = torch.stack([torch.where(copied, end, -1), torch.where(copied, to, -1), torch.where(copied, keep % page, 0)], -1)
    src, dst, count = moves[copied].unbind(-1)
    some = (torch.arange(page, device="cuda") < count[:, None])[:, None, :, None]
    for layer in s["layers"]:
        for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
            if layer[name] is not None:
                x = layer[name].view(torch.int8) if layer[name].dtype == torch.float8_e4m3fn else layer[name]
                x[dst] = torch.where(some if x.dim() == 4 else some[..., 0], x[src], x[dst])
    return [refs.to(torch.int32), new.to(torch.int32), held.to(torch.int32), moves.to(torch.int32)] + _layers(s)


def _plain_compact(s):
    page, path = s["case"]["page"], s["path"].long()
    m = torch.arange(path.shape[1], device="cuda")
    seq, at = torch.nonzero(m < s["path_len"][:, None], as_tuple=True)
    context = (s["kv_len"] - (s["q_start"][1:] - s["q_start"][:-1])).long()[seq]
    src, dst = context + path[seq, at], context + at
    table = s["page_table"].long()
    for layer in s["layers"]:
        for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
            if layer[name] is not None:
                x = layer[name].view(torch.int8) if layer[name].dtype == torch.float8_e4m3fn else layer[name]
                x[table[seq, dst // page], :, dst % page] = x[table[seq, src // page], :, src % page]
    return _layers(s)


def _plain_beams(s):
    case = s["case"]
    seqs, beams, vocab, keep = case["seqs"], case["beams"], case["vocab"], case["keep"]
    x = s["logits"].float()
    top = x.amax(-1, keepdim=True)
    # candidates next to one another are told apart in 64 bits
    lse = top.double() + (x - top).exp().sum(-1, keepdim=True, dtype=torch.float64).log()
    score = s["totals"].double()[:, None] + (s["logits"].double() - lse)
    score = score.view(seqs, beams * vocab)
    best, at = score.topk(min(keep, beams * vocab), dim=-1)
    # ties to the lowest index: everything at or above the last one, by score and then by place
    row, col = torch.nonzero(score >= best[:, -1:].clamp(min=torch.finfo(torch.float64).min), as_tuple=True)
    value = score[row, col]
    order = torch.sort(value, descending=True, stable=True)[1]
    order = order[torch.sort(row[order], stable=True)[1]]
    row, col, value = row[order], col[order], value[order]
    rank = torch.arange(len(row), device="cuda") - torch.searchsorted(row, row)
    row, col, value, rank = (v[rank < keep] for v in (row, col, value, rank))
    scores = torch.full((seqs, keep), -math.inf, device="cuda")
    parent, token = (torch.full((seqs, keep), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    scores[row, rank] = value.float()
    parent[row, rank] = (row * beams + col // vocab).to(torch.int32)
    token[row, rank] = (col % vocab).to(torch.int32)
    return scores, parent, token


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "beams":
        rows = case["seqs"] * case["beams"]
        return {"bytes": rows * (case["vocab"] * size + 4) + 12 * case["seqs"] * case["keep"], "flops": 3 * rows * case["vocab"]}
    row = case["kv_heads"] * (case["dim"] * 2 if case.get("cache", "16") == "16" else case["dim"] + 4) * 2      # cached bytes of one token, K and V
    if case["op"] == "fork":
        requests, source = _beams(case)
        kept = {}
        copied = fresh = entries = 0
        for j in source:
            if j < 0:
                continue
            kv = requests[j // case["beams"]][0]
            entries += kv // case["page"] + 1
            if kv % case["page"]:
                copied += (kv % case["page"]) if j in kept else 0
                kept[j] = True
        held = sum(h for _, _, h in requests) * case["beams"]
        pool = sum(sh + case["beams"] * (h - sh) for _, sh, h in requests) + 2 * len(source) + 5
        return {"bytes": 2 * copied * row * case["layers"] + 4 * (held + entries + 2 * pool) + 32 * len(source), "flops": pool}
    lens = _lengths(case)
    new = sum(q for q, _ in lens)
    if case["op"] == "compact":
        moved = sum(sum(1 for m, p in enumerate(path) if m != p) for path in _paths(case))
        return {"bytes": 2 * moved * row * case["layers"] + 4 * sum(len(p) for p in _paths(case)), "flops": moved}
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] in ("rotate", "append"):
        given = (heads + kv_heads * (2 if case["op"] == "append" else 1)) * dim * 2
        written = heads * dim * 2 + (kv_heads * dim * 2 if case["op"] == "rotate" else row)
        back = row + kv_heads * dim * 4 if case["op"] == "append" and case["cache"] != "16" else 0        # read back from the 8-bit cache
        return {"bytes": new * (given + written + back + 4 * case["axes"]), "flops": new * (heads + kv_heads) * dim * 8}
    keys = pairs = 0
    for (q, kv), bits in zip(lens, _trees(case)):
        c, w = kv - q, case["window"]
        lo = max(0, c - w + 1) if w else 0
        keys += kv - lo + min(case["sinks"], lo)
        for b in bits:
            n = bin(b).count("1")
            lo = min(c, max(0, c + n - 1 - w + 1)) if w else 0
            pairs += n + c - lo + min(case["sinks"], lo)
    return {"bytes": keys * row + 4 * heads * dim * new + new * ((max(q for q, _ in lens) + 31) // 32) * 4, "flops": 4 * dim * heads * pairs}


def exact(case, seed):
    """What run() returns, in 64 bits, sequence by sequence from the definitions. None for what moves pages: nothing is computed there."""
    global own
    if case["op"] in ("fork", "compact"):
        return None
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f64 = torch.float64
    if case["op"] == "beams":
        out = torch.full((case["seqs"], case["keep"]), -math.inf, dtype=f64, device="cuda")
        for r in range(case["seqs"]):
            rows = range(r * case["beams"], (r + 1) * case["beams"])
            each = torch.cat([torch.sort(torch.log_softmax(s["logits"][i].to(f64), -1) + s["totals"][i].to(f64), descending=True)[0][: case["keep"]] for i in rows])
            each = torch.sort(each, descending=True)[0][: case["keep"]]
            out[r, : len(each)] = each
        return out, None, None
    lens, dim, kv_heads = _lengths(case), case["dim"], case["kv_heads"]
    if case["op"] in ("rotate", "append"):
        n = case["turned"]
        place = torch.tensor([p for q, kv in lens for p in range(kv - q, kv)], device="cuda")

        def turned(x, weight):
            x = x.to(f64)
            if weight is not None:
                x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.to(f64)
            out = x.clone()
            for i, (f, axis) in enumerate(zip(_frequencies(case), _axis_of(case))):
                a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + n // 2)
                z = torch.polar(torch.ones_like(place, dtype=f64), (s["positions"][:, axis] if s["positions"] is not None else place).to(f64) * f)
                z = torch.complex(x[..., a], x[..., b]) * z[:, None]
                out[..., a], out[..., b] = z.real, z.imag
            return out

        q, k = turned(s["q"], s["q_weight"]), turned(s["k"], s["k_weight"])
        if case["op"] == "rotate":
            return [q, k]
        if case["cache"] == "16":
            pages = [s["k_pages"].to(f64), s["v_pages"].to(f64)]
            at = 0
            for i, (n_new, kv) in enumerate(lens):
                for p in range(kv - n_new, kv):
                    page, slot = s["page_table"][i, p // case["page"]], p % case["page"]
                    pages[0][page, :, slot], pages[1][page, :, slot] = k[at], s["v"][at].to(f64)
                    at += 1
                if at > 6000:
                    return None
            return (q, *pages)
        held = []
        for x in (k, s["v"].to(f64)):
            amax = x.abs().amax(-1, keepdim=True)
            scale = torch.where(amax < TINY, torch.zeros_like(amax), amax / TOP[case["cache"]])
            y = x / torch.where(scale > 0, scale, torch.ones_like(scale))
            if case["cache"] == "int8":
                y = torch.round(y)
            else:  # e4m3: a sign, 4 bits of exponent (smallest normal 2^-6), 3 of fraction
                step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                y = torch.round(y / step) * step
            held.append(y * scale)
        return (q, *held)
    out = torch.zeros(s["tokens"], case["heads"], dim, dtype=f64, device="cuda")
    at, group = 0, case["heads"] // kv_heads
    for i, ((q, kv), bits) in enumerate(zip(lens, _trees(case))):
        table, c = s["page_table"][i, : -(-kv // case["page"])].long(), kv - q

        def rows_of(name):
            x = s[name + "_pages"][table].to(f64)
            if s[name + "_scale"] is not None:
                x = x * s[name + "_scale"][table].to(f64)[..., None]
            return x.transpose(0, 1).reshape(kv_heads, -1, dim)[:, :kv]

        k, v = rows_of("k"), rows_of("v")
        seen = torch.zeros(q, kv, dtype=torch.bool)
        for t, b in enumerate(bits):
            seen[t, :c] = True
            if case["window"]:
                seen[t, : max(0, min(c, c + bin(b).count("1") - case["window"]))] = False
                seen[t, : min(case["sinks"], c)] = True
            for j in range(q):
                seen[t, c + j] = bool(b >> j & 1)
        seen = seen.cuda()
        for h in range(case["heads"]):
            x = s["q"][at : at + q, h].to(f64) @ k[h // group].T * dim ** -0.5
            out[at : at + q, h] = torch.softmax(x.masked_fill(~seen, -math.inf), -1) @ v[h // group]
        at += q
    return out
