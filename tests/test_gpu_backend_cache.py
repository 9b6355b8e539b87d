"""Writing to and reading from the paged cache: codes and scales bit for bit against the definition in fp32, values within half a code
step of the given ones in 64 bits, nothing written outside the new tokens' cells."""
import math

import pytest
import torch

from tests.backend_cases import Case, quantise

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
LENS = [(1, 1), (1, 17), (5, 5), (0, 30), (33, 64), (16, 16), (0, 0), (40, 12), (130, 300), (1, 128)]


def raw(t):
    return t.contiguous().view(torch.uint8)


def appended(case, k, v):
    """What the pool has to hold after the append, computed cell by cell."""
    want = {n: getattr(case, n).clone() if getattr(case, n) is not None else None for n in ("k", "v", "k_scale", "v_scale")}
    at = 0
    for i, (q, kv) in enumerate(case.lens):
        for t in range(q):
            pos = kv - q + t
            if pos >= 0:
                page, slot = case.table[i, pos // case.page].item(), pos % case.page
                for n, x in (("k", k), ("v", v)):
                    if case.kind == "16":
                        want[n][page, :, slot] = x[at + t]
                    else:
                        code, scale = quantise(x[at + t], case.kind)
                        want[n].view(torch.uint8)[page, :, slot] = code.view(torch.uint8)
                        want[n + "_scale"][page, :, slot] = scale
        at += q
    return want


def new_rows(case, seed, pad=0):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(case.tokens, 2 * case.kv_heads * case.dim + pad, generator=g, device="cuda").to(case.dtype)
    n = case.kv_heads * case.dim
    shape = (case.kv_heads, case.dim)
    return x[:, :n].unflatten(1, shape), x[:, n : 2 * n].unflatten(1, shape)      # strided: slices of one projection


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("dim,page,kv_heads,pad", [(64, 16, 1, 0), (128, 32, 3, 8), (64, 128, 8, 40), (128, 64, 2, 0)])
def test_append_and_read_bit_for_bit(cache, dtype, dim, page, kv_heads, pad):
    case = Case(LENS, kv_heads=kv_heads, group=1, dim=dim, page=page, dtype=dtype, cache=cache, seed=1)
    k, v = new_rows(case, 2, pad)
    want = appended(case, k, v)
    case.backend.append(case.cache, case.batch, k, v)
    case.backend.sync()
    for n in ("k", "v", "k_scale", "v_scale"):
        if want[n] is not None:
            assert torch.equal(raw(getattr(case, n)), raw(want[n])), n
    total = sum(kv for _, kv in LENS)
    start = torch.tensor([sum(kv for _, kv in LENS[:i]) for i in range(len(LENS) + 1)], dtype=torch.int32, device="cuda")
    got = case.backend.read(case.cache, case.batch, start, total)
    case.backend.sync()
    for n, x in zip(("k", "v"), got):
        rows = torch.cat([case.rows(n, i).transpose(0, 1) for i in range(len(LENS))])
        # code * scale is one fp32 rounding, then one to the activation type
        data, scale = getattr(case, n), getattr(case, n + "_scale")
        if scale is None:
            assert torch.equal(x, rows.to(dtype))
        else:
            cell = (data.float() * scale[..., None]).to(dtype)
            assert torch.equal(x, torch.cat([cell[case.table[i, : -(-kv // page)].long()].transpose(0, 1).reshape(kv_heads, -1, dim)[:, :kv].transpose(0, 1)
                                             for i, (_, kv) in enumerate(LENS) if kv]))


@pytest.mark.parametrize("cache", ["int8", "e4m3"])
def test_values_within_half_a_code_step(cache):
    """In 64 bits: int8 within half a step (amax / 127) of the given value; e4m3 within 2^-4 of its magnitude or half the subnormal
    step 2^-10 of the scale; 2^-20 relative for the fp32 scale and its inverse."""
    case = Case([(200, 200)], kv_heads=4, group=1, dim=128, page=64, dtype=BF16, cache=cache, seed=3)
    k, v = new_rows(case, 4)
    case.backend.append(case.cache, case.batch, k, v)
    for n, x in (("k", k), ("v", v)):
        x = x.double().transpose(0, 1)
        scale = x.abs().amax(-1, keepdim=True) / (127.0 if cache == "int8" else 448.0)
        step = scale * 0.5 if cache == "int8" else torch.maximum(x.abs() * 2.0 ** -4, scale * 2.0 ** -10)
        assert ((case.rows(n, 0) - x).abs() <= step * (1 + 2.0 ** -10) + x.abs() * 2.0 ** -20).all()


@pytest.mark.parametrize("cache", ["int8", "e4m3"])
def test_rows_at_the_ends_of_the_range(cache):
    case = Case([(8, 8)], kv_heads=1, group=1, dim=64, page=16, dtype=BF16, cache=cache, seed=5)
    k = torch.randn(8, 1, 64, device="cuda").to(BF16)
    k[0] = 0.0
    k[1] *= 2.0 ** -110                      # below 2^-100: held as zeros
    k[2, 0, 5] = math.nan
    k[3, 0, 63] = math.inf
    k[4, 0, 0] = -math.inf
    k[5] = 0.0
    k[5, 0, 7] = -3.0e38                      # near the type's lowest value
    k[6] *= 2.0 ** -80
    case.backend.append(case.cache, case.batch, k, k)
    got, _ = case.backend.read(case.cache, case.batch, torch.tensor([0, 8], dtype=torch.int32, device="cuda"), 8)
    case.backend.sync()
    assert (got[0] == 0).all() and (got[1] == 0).all()
    assert torch.isnan(got[2]).all() and torch.isnan(got[3]).all() and torch.isnan(got[4]).all()
    assert torch.isfinite(got[5]).all() and abs(got[5, 0, 7].item() + 3.0e38) < 3.0e38 * 2.0 ** -7
    tolerance = 2.0 ** -3 if cache == "e4m3" else 2.0 ** -6          # half a code step relative to the row's largest value, generously
    assert ((got[6].double() - k[6].double()).abs() <= k[6].double().abs().max() * tolerance).all()
    want = quantise(k, cache)
    cells = case.k[case.table[0, 0].item(), 0, :8]
    assert torch.equal(cells.view(torch.uint8), want[0][:, 0].view(torch.uint8))


def test_part_of_a_sequence_and_empty_ones():
    case = Case([(0, 50), (0, 0), (0, 33)], kv_heads=2, group=1, dim=64, page=16, dtype=F16, cache="16", seed=6)
    start = torch.tensor([0, 20, 20, 53], dtype=torch.int32, device="cuda")
    k, v = case.backend.read(case.cache, case.batch, start, 53)
    case.backend.sync()
    for x, n in ((k, "k"), (v, "v")):
        want = torch.cat([case.rows(n, 0)[:, :20].transpose(0, 1), case.rows(n, 2).transpose(0, 1)])
        assert torch.equal(x, want.to(F16))


def test_bad_ids_are_skipped_and_reported():
    from paper_2603_20661_b200.binding import WwwsError
    case = Case([(20, 20), (3, 40)], kv_heads=1, group=1, dim=64, page=16, dtype=BF16, cache="16", seed=7)
    k, v = new_rows(case, 8)
    page = case.table[0, 1].item()
    case.table[0, 1] = case.n_pages + 5
    before = case.k[page].clone()
    case.backend.append(case.cache, case.batch, k, v)
    with pytest.raises(WwwsError) as e:
        case.backend.sync()
    assert e.value.status == 8
    assert torch.equal(raw(case.k[page]), raw(before))
    assert torch.equal(case.k[case.table[1, 2].item(), 0, 5:8], k[20:23, 0])       # the other sequence is written
    case.kv_len[0] = 1000
    case.backend.append(case.cache, case.batch, k, v)
    with pytest.raises(WwwsError) as e:
        case.backend.sync()
    assert e.value.status == 1
    with pytest.raises(WwwsError):                                                 # more rows asked for than the sequence has
        case.kv_len[0] = 20
        case.backend.read(case.cache, case.batch, torch.tensor([0, 0, 41], dtype=torch.int32, device="cuda"), 41)
        case.backend.sync()


def test_refusals():
    from paper_2603_20661_b200.binding import WwwsError
    case = Case([(2, 20)], kv_heads=2, group=1, dim=64, page=16, dtype=BF16, cache="int8", seed=9)
    k, v = new_rows(case, 10)
    with pytest.raises(ValueError):
        case.backend.append(case.cache, case.batch, k[:1], v)
    with pytest.raises(ValueError):
        case.backend.append(case.cache, case.batch, k.half(), v)
    with pytest.raises(ValueError):
        case.backend.bind_cache(case.k, case.v)                                    # scales missing
    wide = torch.zeros(2, 2 * 64 + 4, dtype=BF16, device="cuda")[:, : 2 * 64].unflatten(1, (2, 64))
    with pytest.raises(WwwsError) as e:
        case.backend.append(case.cache, case.batch, wide, v)
    assert e.value.status == 1
