"""Sequences over a paged cache for the backend tests, and the operators' definitions in 64 bits."""
import math

import torch

TOP = {"int8": 127.0, "e4m3": 448.0}


def quantise(x, kind):
    """Codes and scales of rows (last axis) of `x`, in fp32 as the header words it; rows with NaN or infinity: scale NaN, codes 0."""
    x = x.float()
    amax = x.abs().amax(-1, keepdim=True)
    finite = torch.isfinite(x).all(-1, keepdim=True)
    scale = torch.where(amax < 2.0 ** -100, torch.zeros_like(amax), amax * torch.tensor(1.0 / TOP[kind], device=x.device))
    inv = torch.where(finite & (scale > 0), torch.ones_like(scale) / scale, torch.zeros_like(scale))
    y = torch.where(finite, (x * inv).clamp(-TOP[kind], TOP[kind]), torch.zeros_like(x))
    code = torch.round(y).to(torch.int8) if kind == "int8" else y.to(torch.float8_e4m3fn)
    return code, torch.where(finite, scale, torch.full_like(scale, math.nan)).squeeze(-1)


class Case:
    """Sequences (new tokens, cached tokens) with random pages in random order.  Cells that no row may look at hold NaN (16-bit values,
    scales) and page-table entries past a sequence's end, or wholly before its window, name no page.  On the CPU
    (device="cpu") it holds the inputs alone."""

    def __init__(self, lens, kv_heads, group, dim, page, dtype, cache, seed, window=0, sinks=0, loud=1.0, stream=None, extra_pages=0, max_rows=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.lens, self.kv_heads, self.group, self.heads, self.dim, self.page, self.dtype, self.kind = lens, kv_heads, group, kv_heads * group, dim, page, dtype, cache
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")                        # noqa: E731
        self.tokens = sum(q for q, _ in lens)
        pages = [-(-kv // page) for _, kv in lens]
        used = sum(pages)
        self.n_pages = used + 2 + extra_pages
        self.max_pages = max(1, max(pages))
        order = (torch.randperm(used + 2, generator=g, device="cuda") + extra_pages).to(torch.int32)
        self.table = torch.full((len(lens), self.max_pages), -1, dtype=torch.int32, device="cuda")
        shape = (self.n_pages, kv_heads, page)
        shown = torch.zeros(shape, dtype=torch.bool, device="cuda")
        at = 0
        for i, (q, kv) in enumerate(lens):
            self.table[i, : pages[i]] = order[at : at + pages[i]]
            at += pages[i]
            j = torch.arange(kv, device="cuda")
            lo = max(0, kv - q - window + 1) if window else 0
            for p in range(pages[i]):
                n = min(page, kv - p * page)
                shown[self.table[i, p].item(), :, :n] = ((j >= lo) | (j < sinks))[p * page : p * page + n]
                if window and not shown[self.table[i, p].item()].any():
                    self.table[i, p] = -1
        self.q = torch.randn(self.tokens, self.heads, dim, generator=g, device="cuda").mul_(loud).to(dtype)
        self.scales = {}
        for name in ("k", "v"):
            x = torch.empty(shape + (dim,), dtype=dtype, device="cuda").normal_(generator=g).mul_(loud if name == "k" else 1.0)
            if cache == "16":
                x[~shown] = math.nan
                setattr(self, name, x)
                setattr(self, name + "_scale", None)
            else:
                x = x.float() * torch.exp(0.5 * torch.randn(shape + (1,), generator=g, device="cuda"))
                code, scale = quantise(x, cache)
                scale[~shown] = math.nan
                setattr(self, name, code)
                setattr(self, name + "_scale", scale)
        starts = [0]
        for q, _ in lens:
            starts.append(starts[-1] + q)
        self.q_start, self.kv_len = i32(starts), i32([kv for _, kv in lens])
        from paper_2603_20661_b200.backend import Backend
        self.backend = Backend(n_heads=self.heads, n_kv_heads=kv_heads, head_dim=dim, page_tokens=page, n_pages=self.n_pages, max_seqs=len(lens),
                               max_tokens=max(1, self.tokens), max_pages=self.max_pages, max_rows=max_rows, dtype=dtype, cache=cache, device="cuda:0", stream=stream)
        self.cache = self.backend.bind_cache(self.k, self.v, self.k_scale, self.v_scale)
        self.batch = self.backend.batch(self.q_start, self.kv_len, self.table, n_tokens=self.tokens, max_q_len=max(q for q, _ in lens),
                                        max_kv_len=max(kv for _, kv in lens))

    def attend(self, window=0, sinks=0, scale=None, stride_pad=0):
        if not stride_pad:
            return self.backend.attend(self.cache, self.batch, self.q, scale=scale, window=window, sinks=sinks)
        wide = lambda: torch.full((self.tokens, self.heads * self.dim + stride_pad), 77.0, dtype=self.dtype, device="cuda")   # noqa: E731
        q, out = wide(), wide()
        q[:, : self.heads * self.dim] = self.q.flatten(1)
        view = lambda t: t[:, : self.heads * self.dim].unflatten(1, (self.heads, self.dim))      # noqa: E731
        self.backend.attend(self.cache, self.batch, view(q), out=view(out), scale=scale, window=window, sinks=sinks)
        assert (out[:, self.heads * self.dim :] == 77.0).all(), "written outside the rows"
        return view(out)

    def rows(self, name, i):
        """Cached rows of sequence i in 64 bits: [kv_heads, kv, dim] (0 where its table names no page)."""
        kv = self.lens[i][1]
        x = torch.zeros(self.kv_heads, kv, self.dim, dtype=torch.float64, device="cuda")
        data, scale = getattr(self, name), getattr(self, name + "_scale")
        for p in range(-(-kv // self.page)):
            n, id = min(self.page, kv - p * self.page), self.table[i, p].item()
            if id < 0:
                continue
            y = data[id, :, :n].double()
            x[:, p * self.page : p * self.page + n] = y if scale is None else y * scale[id, :, :n, None].double()
        return x


def attend_exact(case, window, sinks, scale):
    """The definition in 64 bits: outputs; per output sum_j p_j |v_j|; per row the largest sum of |q k| scale over seen keys."""
    scale = case.dim ** -0.5 if scale is None else scale
    out = torch.zeros(case.tokens, case.heads, case.dim, dtype=torch.float64, device="cuda")
    weight, scores = torch.zeros_like(out), torch.zeros(case.tokens, case.heads, dtype=torch.float64, device="cuda")
    at = 0
    for i, (q_len, kv) in enumerate(case.lens):
        if q_len and kv:
            k, v = case.rows("k", i), case.rows("v", i)
            p = torch.arange(kv - q_len, kv, device="cuda")[:, None]
            j = torch.arange(kv, device="cuda")
            seen = j <= p
            if window:
                seen &= (j > p - window) | (j < sinks)
            for h in range(case.heads):
                q = case.q[at : at + q_len, h].double()
                kh, vh = torch.nan_to_num(k[h // case.group]), torch.nan_to_num(v[h // case.group])
                x = (q @ kh.T * scale).masked_fill(~seen, -math.inf)
                top = x.amax(-1, keepdim=True)
                e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
                e = torch.nan_to_num(e / e.sum(-1, keepdim=True))
                out[at : at + q_len, h] = e @ vh
                weight[at : at + q_len, h] = e @ vh.abs()
                scores[at : at + q_len, h] = ((q.abs() @ kh.abs().T) * abs(scale)).masked_fill(~seen, 0.0).amax(-1)
        at += q_len
    return out, weight, scores


def attend_bound(case, want, weight, scores):
    """How far a result may be off, from the formats alone.  u: the unit roundoff of the activation type, half the spacing of the
    numbers just above 1: 2^-8 for bf16 (8 significant bits), 2^-11 for f16 (11).
      output rounded once                     u |o|                (and half the smallest subnormal)
      weights rounded for the second product  u W,  W = sum p |v|  (their sum is fp32 of the unrounded or of the rounded weights: at most u W more)
      scores in fp32                          a relative error d of each weight, which the normalisation at most doubles:
                                              products and additions of dim terms, the scale(s) and the shift by the maximum each
                                              2^-24 of at most s = max sum |q k| scale, s (dim + 8) 2^-24, and 2^-21 for the exponential
      sums over kv keys in fp32               (2 kv + 64) 2^-24 W: kv additions in numerator and denominator, in any order, and the joining of parts
      fp32 weights below 2^-126 are zero        2^-126 sum |v| <= 2^-126 kv max|v|
      f16 weights below 2^-14 lose bits       at most 2^-25 per key relative to a largest weight of 1 (the lift of quantised weights makes up for
                                              scales down to 2^-6 and less): 2^-25 sum |v| <= 2^-25 kv max|v|"""
    u = 2.0 ** -8 if case.dtype == torch.bfloat16 else 2.0 ** -11
    kv = max(kv for _, kv in case.lens)
    d = scores[..., None] * (case.dim + 8) * 2.0 ** -24 + 2.0 ** -21
    bound = u * want.abs() + (2 * u + 2 * d + (2 * kv + 64) * 2.0 ** -24) * weight + 2.0 ** -126 * kv * 64.0
    if case.dtype == torch.float16:
        bound = bound + 2.0 ** -25 + 2.0 ** -25 * kv * 64.0
    return bound * (1 + 2.0 ** -7)
