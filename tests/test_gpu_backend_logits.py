"""Logits shaping against the definition: in fp32, operation by operation, the outputs are equal bit for bit; in 64 bits they are
within the roundings that fp32 and the type allow; the token is the lowest index of the largest rounded value."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def backend(rows):
    from paper_2603_20661_b200.backend import Backend
    return Backend(max_rows=rows, device="cuda:0")


def inputs(rows, vocab, seed, history=40, bias=5, masks=3, dup=False):
    g = torch.Generator().manual_seed(seed)
    lens = [(history * (r + 1)) % (2 * history + 1) for r in range(rows)]
    nb = [(bias * (r + 2)) % (2 * bias + 1) for r in range(rows)]
    ends = lambda v: torch.tensor([sum(v[:i]) for i in range(len(v) + 1)], dtype=torch.int32)    # noqa: E731
    ids = lambda n: (torch.rand(n, generator=g) ** 2 * vocab).to(torch.int32).clamp_(max=vocab - 1)   # noqa: E731
    words = (vocab + 31) // 32
    s = {"history": ids(sum(lens)), "history_start": ends(lens), "prompt_len": torch.tensor([n // 2 for n in lens], dtype=torch.int32),
         "repetition": 0.7 + torch.rand(rows, generator=g), "presence": torch.rand(rows, generator=g) - 0.3, "frequency": torch.rand(rows, generator=g) - 0.2,
         "bias_id": ids(sum(nb)), "bias_value": 5 * torch.randn(sum(nb), generator=g), "bias_start": ends(nb),
         "mask": torch.randint(-2 ** 31, 2 ** 31 - 1, (masks, words), generator=g, dtype=torch.int64).to(torch.int32),
         "mask_index": torch.tensor([r % (masks + 1) - 1 for r in range(rows)], dtype=torch.int32)}
    return s, torch.randn(rows, vocab, generator=g) * 4


def plain(logits, s, dtype):
    """The definition row by row on the CPU in `dtype`; the last entry of a repeated bias id holds."""
    out = logits.to(dtype).clone()
    rows, vocab = out.shape
    for r in range(rows):
        x = out[r]
        if s.get("history") is not None:
            ids = s["history"][s["history_start"][r] : s["history_start"][r + 1]].long()
            count = torch.bincount(ids[(int(s["prompt_len"][r]) if s.get("prompt_len") is not None else 0):], minlength=vocab)
            seen = torch.bincount(ids, minlength=vocab) > 0
            one = torch.ones((), dtype=dtype)
            rep = s["repetition"][r].to(dtype) if s.get("repetition") is not None else one
            freq = s["frequency"][r].to(dtype) if s.get("frequency") is not None else 0 * one
            pres = s["presence"][r].to(dtype) if s.get("presence") is not None else 0 * one
            x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
            x = torch.where(count > 0, x - freq * count.to(dtype), x)
            x = torch.where(count > 0, x - pres, x)
        if s.get("bias_id") is not None:
            last = {}
            for e in range(int(s["bias_start"][r]), int(s["bias_start"][r + 1])):
                last[int(s["bias_id"][e])] = e
            for i, e in last.items():
                x[i] += s["bias_value"][e].to(dtype)
        if s.get("mask") is not None:
            m = int(s["mask_index"][r]) if s.get("mask_index") is not None else r
            if m >= 0:
                bit = (s["mask"][m].long()[:, None] >> torch.arange(32)) & 1
                x = x.masked_fill(bit.reshape(-1)[:vocab] == 0, -math.inf)
        out[r] = x
    return out


def token_of(x):
    x = torch.where(torch.isnan(x.float()), torch.full_like(x.float(), -math.inf), x.float())
    top = x.amax(-1, keepdim=True)
    first = torch.where(x == top, torch.arange(x.shape[1]), x.shape[1]).amin(-1)
    return torch.where(top[:, 0] == -math.inf, -1, first).to(torch.int32)


def run(b, logits, s, **more):
    dev = {k: v.cuda() if v is not None else None for k, v in s.items()}
    out, token = b.shape_logits(logits, b.shaping(**dev), **more)
    b.sync()
    return out.cpu(), token.cpu() if token is not None else None


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 7), (2, 31), (5, 33), (4, 1000), (7, 1025), (2, 8191), (3, 8193), (2, 32003), (40, 20001), (300, 517)])
def test_bit_for_bit(dtype, rows, vocab):
    s, x = inputs(rows, vocab, rows * vocab)
    x = x.to(dtype)
    got, token = run(backend(rows), x.cuda(), s)
    want = plain(x.float(), s, F32).to(dtype)
    assert torch.equal(got.float(), want.float())
    assert torch.equal(token, token_of(want))
    # 64 bits: a handful of fp32 operations on numbers of the size of the largest term, then one rounding
    exact = plain(x.double(), s, torch.float64)
    size = 60.0
    u = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}[dtype]          # unit roundoffs
    fine = torch.isfinite(exact)
    assert torch.equal(fine, torch.isfinite(got))
    assert ((got.double() - exact)[fine].abs() <= u * exact[fine].abs() + 8 * size * 2.0 ** -24).all()


@pytest.mark.parametrize("left_out", ["history", "prompt_len", "repetition", "presence", "frequency", "bias_id", "mask", "mask_index", "all"])
def test_parts_left_out(left_out):
    s, x = inputs(3, 3001, 17)
    if left_out == "all":
        s = {}
    else:
        s[left_out] = None
        if left_out == "bias_id":
            s["bias_value"] = s["bias_start"] = None
        if left_out == "history":
            s["history_start"] = s["prompt_len"] = None
    got, token = run(backend(3), x.cuda(), s)
    want = plain(x, s, F32)
    assert torch.equal(got, want) and torch.equal(token, token_of(want))


def test_strides_alignment_and_in_place():
    for dtype in (F32, BF16):
        s, x = inputs(6, 5003, 23)
        want = plain(x.to(dtype).float(), s, F32).to(dtype)
        b = backend(6)
        wide = torch.full((6, 5120), 9.0, dtype=dtype, device="cuda")
        for shift in (0, 1, 3):
            view = wide[:, shift : shift + 5003]
            view.copy_(x)
            got, token = run(b, view, s)                                  # aligned output, input `shift` elements off
            assert torch.equal(got, want) and torch.equal(token, token_of(want))
            run(b, view, s, out=view)
            assert torch.equal(view.cpu(), want)
            assert (wide[:, shift + 5003:] == 9.0).all()
            wide.fill_(9.0)
        view = wide[:, :5003]
        view.copy_(x)
        got, token = run(b, view, s, tokens=False)
        assert token is None and torch.equal(got, want)


def test_rows_with_nothing_left_ties_and_special_values():
    x = torch.zeros(8, 300)
    x[0] = 1.0                                    # all equal: the first
    x[1, 200] = x[1, 100] = 5.0                   # a tie
    x[2] = -math.inf
    x[3] = math.nan
    x[4, 7] = math.nan
    x[4, 9] = 2.0
    x[5] = -3.4e38                                # the type's lowest values
    x[5, 250] = -3.3e38
    x[6, 11] = math.inf
    x[7] = -0.0
    x[7, 40] = 0.0                                # -0 and +0 tie: the first
    s = {"mask": torch.zeros(2, 10, dtype=torch.int32), "mask_index": torch.tensor([-1, -1, -1, -1, -1, -1, -1, -1], dtype=torch.int32)}
    b = backend(8)
    got, token = run(b, x.cuda(), s)
    assert torch.equal(torch.nan_to_num(got, nan=7.0), torch.nan_to_num(x, nan=7.0))
    assert token.tolist() == [0, 100, -1, -1, 9, 250, 11, 0]
    s["mask_index"] = torch.full((8,), 1, dtype=torch.int32)              # a mask that allows nothing
    got, token = run(b, x.cuda(), s)
    assert (got == -math.inf).all() and (token == -1).all()
    s["mask"][1, 3] = 1 << 4                                              # token 100 alone: NaN elsewhere is gone
    got, token = run(b, x.cuda(), s)
    assert token.tolist() == [100, 100, -1, -1, 100, 100, 100, 100]


def test_repeated_ids_and_long_histories():
    vocab = 50
    history = torch.tensor([7] * 5000 + [9] + [7] * 3, dtype=torch.int32)
    s = {"history": history, "history_start": torch.tensor([0, len(history)], dtype=torch.int32), "prompt_len": torch.tensor([1000], dtype=torch.int32),
         "frequency": torch.tensor([0.001]), "presence": torch.tensor([0.25]), "repetition": torch.tensor([2.0]),
         "bias_id": torch.tensor([3, 4, 3, 3], dtype=torch.int32), "bias_value": torch.tensor([1.0, 2.0, 10.0, -4.0]), "bias_start": torch.tensor([0, 4], dtype=torch.int32)}
    x = torch.ones(1, vocab)
    got, _ = run(backend(1), x.cuda(), s)
    assert torch.equal(got, plain(x, s, F32))
    assert got[0, 3] == -3.0 and abs(got[0, 7].item() - (0.5 - 4.003 - 0.25)) < 1e-5


def test_bad_ids_are_skipped_and_reported():
    from paper_2603_20661_b200.binding import WwwsError
    s, x = inputs(3, 100, 3)
    b = backend(3)
    for name, value, status in (("history", 100, 8), ("history", -1, 8), ("bias_id", 1 << 20, 8), ("mask_index", 3, 8), ("history_start", -4, 1)):
        t = {k: v.clone() for k, v in s.items()}
        t[name][1] = value
        dev = {k: v.cuda() for k, v in t.items()}
        b.shape_logits(x.cuda(), b.shaping(**dev))
        with pytest.raises(WwwsError) as e:
            b.sync()
        assert e.value.status == status, name
    got, token = run(b, x.cuda(), s)                                      # and the next call is whole again
    want = plain(x, s, F32)
    assert torch.equal(got, want) and torch.equal(token, token_of(want))


def test_refusals():
    from paper_2603_20661_b200.binding import WwwsError
    b = backend(4)
    s, x = inputs(3, 100, 3)
    dev = {k: v.cuda() for k, v in s.items()}
    with pytest.raises(ValueError):
        b.shape_logits(x.double().cuda(), b.shaping())
    with pytest.raises(ValueError):
        b.shape_logits(x[:2].cuda(), b.shaping(**dev))
    with pytest.raises(ValueError):
        b.shaping(**{**dev, "history": dev["history"].long()})
    with pytest.raises(ValueError):
        b.shaping(**{**dev, "presence": dev["presence"][:2]})
    with pytest.raises(WwwsError) as e:
        b.shape_logits(torch.zeros(5, 10, device="cuda"), b.shaping())
    assert e.value.status == 1 and "max_rows" in str(e.value)
    with pytest.raises(WwwsError):
        b.shape_logits(x.cuda(), b.shaping(mask=dev["mask"][:, :2].contiguous(), mask_index=dev["mask_index"]))
    with pytest.raises(WwwsError):
        b.shape_logits(torch.zeros(1, 8, device="cuda").expand(3, 8), b.shaping())
