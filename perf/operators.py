"""Cases of the serving-backend operators: what is measured, their plain form, and their values in 64 bits.

A case is one call (or one write and read back) as a peer of the network makes it while it answers requests:
  attend   attention of new tokens over the paged cache, from one token per sequence to whole prompts
  cache    new tokens' keys and values written to the paged cache (as they are, as int8 or as e4m3), the sequences read back
  logits   penalties, biases and a grammar mask on a batch's logits, and the token that a temperature of zero picks
Lengths follow the request streams of `synth` (lognormal, sigma 0.8, clipped at 8,192 tokens) where a case is ragged.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
TOP = {"int8": 127.0, "e4m3": 448.0}        # largest code of a quantised cache
TINY = 2.0 ** -100                           # rows whose largest magnitude is below this are held as zeros


def listed():
    attend = {"op": "attend", "window": 0, "sinks": 0, "mix": 1}
    cache = {"op": "cache", "mix": 1}
    logits = {"op": "logits", "mix": 1}
    return [
        # the smallest call: one short request being answered, where latency is what counts
        dict(attend, name="decode_one", seqs=1, q=1, kv=300, ragged=False, heads=16, kv_heads=4, dim=64, page=16, dtype="bf16", cache="16"),
        # an ordinary decode step of a busy peer: one token for each of 96 requests of mixed lengths
        dict(attend, name="decode_batch", seqs=96, q=1, kv=1500, ragged=True, heads=32, kv_heads=8, dim=128, page=16, dtype="bf16", cache="16"),
        # a few very long contexts in an 8-bit cache: every byte of the cache is read once
        dict(attend, name="decode_long_int8", seqs=6, q=1, kv=65537, ragged=False, heads=32, kv_heads=4, dim=128, page=64, dtype="bf16", cache="int8"),
        # long conversations under a sliding window whose first tokens stay visible
        dict(attend, name="decode_window_e4m3", seqs=64, q=1, kv=12001, ragged=False, heads=32, kv_heads=8, dim=128, page=32, dtype="bf16", cache="e4m3", window=4000, sinks=4),
        # several drafted tokens per request checked in one call
        dict(attend, name="draft_check", seqs=24, q=5, kv=3001, ragged=True, heads=24, kv_heads=4, dim=128, page=32, dtype="f16", cache="e4m3"),
        # a chunk of a prompt behind what is already cached
        dict(attend, name="chunk", seqs=1, q=512, kv=6001, ragged=False, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16", cache="16"),
        # newly dispatched prompts of mixed lengths in one call, windowed, 8-bit cache
        dict(attend, name="prompts_int8", seqs=24, q=0, kv=900, ragged=True, heads=28, kv_heads=4, dim=64, page=16, dtype="f16", cache="int8", window=1000, sinks=8),
        # the longest prompts a request may have, two at once: bound by arithmetic
        dict(attend, name="prompts_long", seqs=2, q=0, kv=8192, ragged=False, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16", cache="16"),
        # a short prompt written and read back
        dict(cache, name="cache_short", seqs=1, q=33, kv=33, ragged=False, heads=16, kv_heads=4, dim=64, page=16, dtype="f16", cache="int8"),
        # newly dispatched prompts written behind shared prefixes, then handed to another peer
        dict(cache, name="cache_prompts", seqs=24, q=0, kv=1700, ragged=True, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16", cache="e4m3"),
        # a judge's verdict: one row whose mask leaves a few tokens
        dict(logits, name="verdict", rows=1, vocab=32003, history=300, bias=2, masked=1.0, left=3, dtype="f32"),
        # sampling inputs of a large batch: histories of mixed lengths, some rows under a grammar
        dict(logits, name="logits_batch", rows=256, vocab=131072, history=1500, bias=40, masked=0.5, left=20000, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "draft", "prompt", "prompt", "cache", "cache", "logits", "logits"])
    mix = rng.randrange(1, 1 << 20)
    if kind == "logits":
        rows, vocab = _log(rng, 1, 256), _log(rng, 1000, 131072)
        return {"op": "logits", "mix": mix, "rows": rows, "vocab": vocab, "history": _log(rng, 10, 2000), "bias": rng.choice([0, 1, 30, 300]),
                "masked": rng.choice([0.0, 0.5, 1.0]), "left": _log(rng, 1, vocab), "dtype": rng.choice(["f32", "bf16", "f16"])}
    kv_heads = rng.choice([1, 2, 4, 8])
    case = {"op": "cache" if kind == "cache" else "attend", "mix": mix, "ragged": rng.random() < 0.6, "heads": kv_heads * rng.choice([1, 2, 4, 5, 7, 8]),
            "kv_heads": kv_heads, "dim": rng.choice([64, 128]), "page": rng.choice([16, 32, 64, 128]), "dtype": rng.choice(["bf16", "f16"]),
            "cache": rng.choice(["16", "int8", "e4m3"])}
    if kind == "decode":
        kv = _log(rng, 16, 65536)
        case.update(seqs=max(1, min(_log(rng, 1, 256), 130000 // kv)), q=1, kv=kv)
    elif kind == "draft":
        kv = _log(rng, 64, 16384)
        case.update(seqs=max(1, min(_log(rng, 1, 64), 130000 // kv)), q=rng.randrange(2, 17), kv=kv)
    else:
        q = _log(rng, 17, 6000)
        kv = q + rng.choice([0, _log(rng, 16, 4000)])
        most = 60000000 if kind == "cache" or not case["ragged"] else 10000000
        case.update(seqs=max(1, min(_log(rng, 1, 32), most // (kv * kv))), q=0 if kv == q else q, kv=kv)
    if case["op"] == "attend":
        windowed = rng.random() < 0.4
        case.update(window=_log(rng, 16, 4096) if windowed else 0, sinks=rng.choice([0, 1, 4, 16]) if windowed else 0)
    return case


def _lengths(case):
    """Per sequence (new tokens, tokens in the cache after them); the case alone decides. q = 0: the whole sequence is new."""
    rng = random.Random(case["mix"])
    got = []
    for _ in range(case["seqs"]):
        kv = case["kv"]
        if case["ragged"]:
            kv = max(1, min(8192, 4 * case["kv"], int(kv * math.exp(rng.gauss(0.0, 0.8)))))
        q = kv if case["q"] == 0 else min(case["q"], kv)
        got.append((q, kv))
    return got


def _histories(case):
    """Per row (prompt tokens, output tokens, bias entries, has a mask)."""
    rng = random.Random(case["mix"])
    got = []
    for _ in range(case["rows"]):
        n = max(1, min(8192, int(case["history"] * math.exp(rng.gauss(0.0, 0.8)))))
        got.append((n * 2 // 3, n - n * 2 // 3, min(case["bias"], case["vocab"]), rng.random() < case["masked"]))
    return got


def _quantise(x, kind):
    """Codes and scales of rows of `x` (f32, [..., dim]): one scale per row."""
    amax = x.abs().amax(-1, keepdim=True)
    scale = torch.where(amax < TINY, torch.zeros_like(amax), amax * torch.tensor(1.0 / TOP[kind], device=x.device))
    inv = torch.where(scale > 0, torch.ones_like(scale) / scale, torch.zeros_like(scale))
    y = (x * inv).clamp(-TOP[kind], TOP[kind])
    code = torch.round(y).to(torch.int8) if kind == "int8" else y.to(torch.float8_e4m3fn)
    return code, scale.squeeze(-1)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    ends = lambda v: [sum(v[:i]) for i in range(len(v) + 1)]  # noqa: E731
    dtype = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "logits":
        rows, vocab = case["rows"], case["vocab"]
        h = _histories(case)
        s["logits"] = (torch.randn(rows, vocab, generator=g, device="cuda") * 3.0).to(dtype)
        n = sum(p + o for p, o, _, _ in h)
        # text repeats itself: token ids crowd at the low end
        s["history"] = (torch.rand(n, generator=g, device="cuda") ** 3 * vocab).to(torch.int32).clamp_(max=vocab - 1)
        s["history_start"] = i32(ends([p + o for p, o, _, _ in h]))
        s["prompt_len"] = i32([p for p, _, _, _ in h])
        s["n_history"] = n
        s["repetition"] = 1.0 + 0.3 * torch.rand(rows, generator=g, device="cuda")
        s["presence"] = torch.rand(rows, generator=g, device="cuda") - 0.2
        s["frequency"] = 0.5 * torch.rand(rows, generator=g, device="cuda")
        nb = sum(b for _, _, b, _ in h)
        s["bias_start"] = i32(ends([b for _, _, b, _ in h]))
        stride = max(1, vocab // max(1, case["bias"]))       # distinct ids within a row
        s["bias_id"] = i32([j * stride for _, _, b, _ in h for j in range(b)])
        s["bias_value"] = 4.0 * torch.randn(nb, generator=g, device="cuda")
        # a few grammar states shared by the rows: words of 32 tokens, a set bit allows its token
        words = (vocab + 31) // 32
        allowed = torch.zeros(4, words * 32, dtype=torch.bool, device="cuda")
        at = torch.randint(0, vocab, (4, case["left"]), generator=g, device="cuda")
        allowed.scatter_(1, at, True)
        bits = allowed.view(4, words, 32).long() << torch.arange(32, device="cuda")
        s["mask"] = bits.sum(-1).to(torch.int32)
        s["mask_index"] = i32([i % 4 if m else -1 for i, (_, _, _, m) in enumerate(h)])
        if own:
            from paper_2603_20661_b200.backend import Backend
            s["backend"] = Backend(max_rows=rows, device="cuda")
            s["shaping"] = s["backend"].shaping(**{k: s[k] for k in ("history", "history_start", "prompt_len", "repetition", "presence", "frequency",
                                                                      "bias_id", "bias_value", "bias_start", "mask", "mask_index")})
        return s
    lens = _lengths(case)
    heads, kv_heads, dim, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    tokens, max_kv = sum(q for q, _ in lens), max(kv for _, kv in lens)
    # queries, keys and values come as slices of one projection's output
    qkv = torch.randn(tokens, (heads + 2 * kv_heads) * dim, generator=g, device="cuda").to(dtype)
    s["q"] = qkv[:, : heads * dim].view(tokens, heads, dim)
    s["k"] = qkv[:, heads * dim : (heads + kv_heads) * dim].view(tokens, kv_heads, dim)
    s["v"] = qkv[:, (heads + kv_heads) * dim :].view(tokens, kv_heads, dim)
    pages = [-(-kv // page) for _, kv in lens]
    n_pages = sum(pages) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(len(lens), max(pages), dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = order[at : at + n]
        at += n
    s.update(q_start=i32(ends([q for q, _ in lens])), kv_len=i32([kv for _, kv in lens]), page_table=table, tokens=tokens, max_q=max(q for q, _ in lens), max_kv=max_kv,
             kv_start=i32(ends([kv for _, kv in lens])), total_kv=sum(kv for _, kv in lens))
    for name in ("k", "v"):
        x = torch.randn(n_pages, kv_heads, page, dim, generator=g, device="cuda").to(dtype)
        if case["cache"] == "16":
            s[name + "_pages"], s[name + "_scale"] = x, None
        else:
            # the written values of a served sequence: rows of different magnitudes
            x = x.float() * torch.exp(0.3 * torch.randn(n_pages, kv_heads, page, 1, generator=g, device="cuda"))
            s[name + "_pages"], s[name + "_scale"] = _quantise(x, case["cache"])
    if own:
        from paper_2603_20661_b200.backend import Backend
        s["backend"] = Backend(n_heads=heads, n_kv_heads=kv_heads, head_dim=dim, page_tokens=page, n_pages=n_pages, max_seqs=len(lens), max_tokens=tokens,
                               max_pages=table.shape[1], dtype=dtype, cache=case["cache"], device="cuda")
        s["cache"] = s["backend"].bind_cache(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"])
        s["batch"] = s["backend"].batch(s["q_start"], s["kv_len"], s["page_table"], n_tokens=tokens, max_q_len=s["max_q"], max_kv_len=max_kv)
    return s


def run(state):
    case = state["case"]
    if own:
        b = state["backend"]
        if case["op"] == "attend":
            return b.attend(state["cache"], state["batch"], state["q"], window=case["window"], sinks=case["sinks"])
        if case["op"] == "cache":
            b.append(state["cache"], state["batch"], state["k"], state["v"])
            return b.read(state["cache"], state["batch"], state["kv_start"], state["total_kv"])
        return b.shape_logits(state["logits"], state["shaping"])
    return {"attend": _plain_attend, "cache": _plain_cache, "logits": _plain_logits}[case["op"]](state)


def _token_of(s):
    """Of each new token: its sequence, its place among the sequence's new tokens, its position in the sequence."""
    start, kv = s["q_start"].long(), s["kv_len"].long()
    t = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(start, t, right=True) - 1
    place = t - start[seq]
    return seq, place, kv[seq] - (start[seq + 1] - start[seq]) + place


def _plain_rows(s, name):
    """The cached rows of every sequence, padded: f32 [seqs, kv_heads, max_kv, dim]."""
    table = s["page_table"].long()
    x = s[name + "_pages"][table].float()
    if s[name + "_scale"] is not None:
        x = x * s[name + "_scale"][table].unsqueeze(-1)
    n, pages, h, p, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(n, h, pages * p, d)[:, :, : s["max_kv"]]


def _plain_attend(s):
    case, q = s["case"], s["q"]
    n, heads, kv_heads, dim = len(s["kv_len"]), case["heads"], case["kv_heads"], case["dim"]
    group = heads // kv_heads
    seq, place, _ = _token_of(s)
    qp = torch.zeros(n, s["max_q"], heads, dim, device="cuda")
    qp[seq, place] = q.float()
    qp = qp.view(n, s["max_q"], kv_heads, group, dim).permute(0, 2, 1, 3, 4).reshape(n, kv_heads, s["max_q"] * group, dim)
    x = (qp @ _plain_rows(s, "k").transpose(-1, -2)).mul_(dim ** -0.5)
    q_len = (s["q_start"][1:] - s["q_start"][:-1]).long()
    pos = (s["kv_len"].long() - q_len)[:, None] + torch.arange(s["max_q"], device="cuda")
    j = torch.arange(s["max_kv"], device="cuda")
    hidden = j > pos[..., None]
    if case["window"]:
        hidden |= (j <= pos[..., None] - case["window"]) & (j >= case["sinks"])
    x.view(n, kv_heads, s["max_q"], group, s["max_kv"]).masked_fill_(hidden[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x @ _plain_rows(s, "v")) / torch.where(total == 0, torch.ones_like(total), total)
    o = o.view(n, kv_heads, s["max_q"], group, dim).permute(0, 2, 1, 3, 4).reshape(n, s["max_q"], heads, dim)
    return o[seq, place].to(q.dtype)


def _plain_cache(s):
    case = s["case"]
    seq, _, pos = _token_of(s)
    page, slot = s["page_table"].long()[seq, pos // case["page"]], pos % case["page"]
    for name in ("k", "v"):
        if case["cache"] == "16":
            s[name + "_pages"][page, :, slot] = s[name]
        else:
            code, scale = _quantise(s[name].float(), case["cache"])
            s[name + "_pages"].view(torch.int8)[page, :, slot] = code.view(torch.int8)
            s[name + "_scale"][page, :, slot] = scale
    start = s["kv_start"].long()
    row = torch.arange(s["total_kv"], device="cuda")
    seq = torch.searchsorted(start, row, right=True) - 1
    pos = row - start[seq]
    page, slot = s["page_table"].long()[seq, pos // case["page"]], pos % case["page"]
    got = []
    for name in ("k", "v"):
        x = s[name + "_pages"].view(torch.int8)[page, :, slot].view(s[name + "_pages"].dtype) if case["cache"] == "e4m3" else s[name + "_pages"][page, :, slot]
        x = x.float()
        got.append((x if s[name + "_scale"] is None else x * s[name + "_scale"][page, :, slot].unsqueeze(-1)).to(s["k"].dtype))
    return got


def _plain_logits(s):
    rows, vocab = s["logits"].shape
    x = s["logits"].float()
    start = s["history_start"].long()
    at = torch.arange(s["n_history"], device="cuda")
    row = torch.searchsorted(start, at, right=True) - 1
    output = (at - start[row] >= s["prompt_len"].long()[row]).float()
    ids = s["history"].long()
    count = torch.zeros(rows, vocab, device="cuda").index_put_((row, ids), output, accumulate=True)
    seen = torch.zeros(rows, vocab, dtype=torch.bool, device="cuda").index_put_((row, ids), torch.ones((), dtype=torch.bool, device="cuda"))
    rep = s["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - s["frequency"][:, None] * count
    x = x - s["presence"][:, None] * (count > 0).float()
    bias_row = torch.searchsorted(s["bias_start"].long(), torch.arange(len(s["bias_id"]), device="cuda"), right=True) - 1
    x = x + torch.zeros(rows, vocab, device="cuda").index_put_((bias_row, s["bias_id"].long()), s["bias_value"])
    v = torch.arange(vocab, device="cuda")
    index = s["mask_index"].long()
    allowed = ((s["mask"][index.clamp(min=0)][:, v // 32] >> (v % 32)) & 1).bool() | (index < 0)[:, None]
    x = torch.where(allowed, x, torch.full_like(x, -math.inf)).to(s["logits"].dtype)
    top = x.amax(-1, keepdim=True)
    first = torch.where(x == top, v, vocab).amin(-1)
    return x, torch.where(top.squeeze(-1) == -math.inf, -1, first).to(torch.int32)


def work(case):
    if case["op"] == "logits":
        h = _histories(case)
        size = 4 if case["dtype"] == "f32" else 2
        n = case["rows"] * case["vocab"]
        masks = min(4, sum(m for _, _, _, m in h)) * ((case["vocab"] + 31) // 32) * 4
        return {"bytes": 2 * n * size + 4 * sum(p + o for p, o, _, _ in h) + 8 * sum(b for _, _, b, _ in h) + masks + 28 * case["rows"], "flops": n}
    lens = _lengths(case)
    row = case["kv_heads"] * (case["dim"] * 2 if case["cache"] == "16" else case["dim"] + 4) * 2     # cached bytes of one token, K and V
    given = case["kv_heads"] * case["dim"] * 2 * 2                                                   # the same as given or returned
    if case["op"] == "cache":
        new, total = sum(q for q, _ in lens), sum(kv for _, kv in lens)
        return {"bytes": new * (given + row) + total * (row + given), "flops": 4 * case["kv_heads"] * case["dim"] * (new + total)}
    keys = pairs = 0
    for q, kv in lens:
        w, p0 = case["window"], kv - q
        lo = max(0, p0 - w + 1) if w else 0
        keys += kv - lo + min(case["sinks"], lo)
        for p in range(p0, kv):
            lo = max(0, p - w + 1) if w else 0
            pairs += p - lo + 1 + min(case["sinks"], lo)
    return {"bytes": keys * row + 4 * case["heads"] * case["dim"] * sum(q for q, _ in lens), "flops": 4 * case["dim"] * case["heads"] * pairs}


def exact(case, seed):
    """What run() returns, in 64 bits, sequence by sequence from the definitions."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f64 = torch.float64
    if case["op"] == "logits":
        rows, vocab = s["logits"].shape
        out = s["logits"].to(f64)
        start, bstart = s["history_start"].tolist(), s["bias_start"].tolist()
        for r, (n_prompt, _, _, masked) in enumerate(_histories(case)):
            ids = s["history"][start[r] : start[r + 1]].long()
            count = torch.bincount(ids[n_prompt:], minlength=vocab).to(f64)
            seen = torch.bincount(ids, minlength=vocab) > 0
            rep = s["repetition"][r].to(f64)
            x = out[r]
            x = torch.where(seen & (x > 0), x / rep, torch.where(seen, x * rep, x))
            x = x - s["frequency"][r].to(f64) * count - s["presence"][r].to(f64) * (count > 0)
            x[s["bias_id"][bstart[r] : bstart[r + 1]].long()] += s["bias_value"][bstart[r] : bstart[r + 1]].to(f64)
            if masked:
                word = s["mask"][r % 4].long() & 0xFFFFFFFF
                bit = (word[:, None] >> torch.arange(32, device="cuda")) & 1
                x = x.masked_fill(bit.reshape(-1)[:vocab] == 0, -math.inf)
            out[r] = x
        return out, None
    page, dim, kv_heads = case["page"], case["dim"], case["kv_heads"]
    group = case["heads"] // kv_heads
    lens = _lengths(case)

    def rows_of(name, i, kv):
        """Cached rows of sequence i: [kv_heads, kv, dim]."""
        table = s["page_table"][i, : -(-kv // page)].long()
        x = s[name + "_pages"][table].to(f64)
        if s[name + "_scale"] is not None:
            x = x * s[name + "_scale"][table].to(f64)[..., None]
        return x.transpose(0, 1).reshape(kv_heads, -1, dim)[:, :kv].clone()

    at = 0
    if case["op"] == "cache":
        got = {"k": [], "v": []}
        for i, (q, kv) in enumerate(lens):
            for name in got:
                x, new = rows_of(name, i, kv), s[name][at : at + q].to(f64)
                if case["cache"] != "16":
                    amax = new.abs().amax(-1, keepdim=True)
                    scale = torch.where(amax < TINY, torch.zeros_like(amax), amax / TOP[case["cache"]])
                    y = new / torch.where(scale > 0, scale, torch.ones_like(scale))
                    if case["cache"] == "int8":
                        y = torch.round(y)
                    else:  # e4m3: a sign, 4 bits of exponent (smallest normal 2^-6), 3 of fraction
                        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                        y = torch.round(y / step) * step
                    new = y * scale
                x[:, kv - q :] = new.transpose(0, 1)
                got[name].append(x.transpose(0, 1))
            at += q
        return [torch.cat(got["k"]), torch.cat(got["v"])]
    out = torch.zeros(s["tokens"], case["heads"], dim, dtype=f64, device="cuda")
    for i, (q, kv) in enumerate(lens):
        k, v = rows_of("k", i, kv), rows_of("v", i, kv)
        for first in range(0, q, 1024):
            n = min(1024, q - first)
            p = torch.arange(kv - q + first, kv - q + first + n, device="cuda")[:, None]
            j = torch.arange(kv, device="cuda")
            seen = j <= p
            if case["window"]:
                seen &= (j > p - case["window"]) | (j < case["sinks"])
            for h in range(case["heads"]):
                x = s["q"][at + first : at + first + n, h].to(f64) @ k[h // group].T * dim ** -0.5
                x = torch.softmax(x.masked_fill(~seen, -math.inf), -1)
                out[at + first : at + first + n, h] = x @ v[h // group]
        at += q
    return out
