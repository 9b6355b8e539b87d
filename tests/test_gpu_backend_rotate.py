"""Norms and rotation of queries and keys, with and without the write to the paged cache, against the formulas in 64 bits."""
import math

import pytest
import torch

from tests.backend_cases import TOP, Case

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")        # noqa: E731


def exact(x, weight, eps, positions, frequencies, axes, interleaved):
    """(the result, its pairs' lengths) of x [tokens, heads, dim] in 64 bits."""
    x, n = x.double(), 2 * len(frequencies)
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    out, size = x.clone(), x.abs()
    for i, f in enumerate(frequencies):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n // 2)
        # positions up to 2^31 times f in 64 bits would be off by up to 2^-22: the whole turns are taken out in whole numbers
        turn = round(f / (2 * math.pi) * 2 ** 64)
        t = torch.tensor([((p * turn) % 2 ** 64) / 2 ** 64 * 2 * math.pi for p in positions[:, axes[i]].tolist()], dtype=torch.float64, device=x.device)[:, None]
        out[..., a], out[..., b] = x[..., a] * t.cos() - x[..., b] * t.sin(), x[..., b] * t.cos() + x[..., a] * t.sin()
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, size


def bound(want, size, u):
    """A rounding to the output's type (u: half a step), and in fp32: the norm's sum of at most 128 squares in chains of 16 and 3 steps between lanes, halved by
    the root, the root itself (2 ulp), three products: 24 2^-24 of the element; the angle: 2^-24 half turns and cos and sin to 2 ulp: pi 2^-24 + 2^-22, with
    their two products and sum: 16 2^-24 of the pair.  Numbers below fp32's and f16's normal range: their smallest step."""
    return u * want.abs() + 48 * 2.0 ** -24 * size + 2.0 ** -24


def u_of(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("dim,turned", [(64, 64), (64, 16), (64, 48), (128, 128), (128, 32), (128, 96)])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("heads,kv_heads,tokens,normed,n_axes", [(4, 4, 1, True, 1), (7, 1, 5, False, 1), (32, 8, 33, True, 3), (3, 3, 3001, True, 2), (40, 8, 300, False, 1)])
def test_rotate(dtype, dim, turned, interleaved, heads, kv_heads, tokens, normed, n_axes):
    from paper_2603_20661_b200.backend import Backend
    g = torch.Generator("cuda").manual_seed(3)
    b = Backend(n_heads=heads, n_kv_heads=kv_heads, head_dim=dim, page_tokens=16, n_pages=1, max_seqs=1, max_tokens=1, max_pages=1, dtype=dtype, device="cuda")
    wide = torch.randn(tokens, (heads + 2 * kv_heads) * dim + 8, generator=g, device="cuda").to(dtype)
    q, k = wide[:, : heads * dim].unflatten(1, (heads, dim)), wide[:, heads * dim : (heads + kv_heads) * dim].unflatten(1, (kv_heads, dim))
    wq, wk = (1.0 + 0.3 * torch.randn(dim, generator=g, device="cuda") for _ in range(2)) if normed else (None, None)
    frequencies = [10000.0 ** (-2.0 * i / turned) for i in range(turned // 2)]
    axes = [i % n_axes for i in range(turned // 2)]
    positions = torch.randint(-5, 1 << 30, (tokens, n_axes), generator=g, device="cuda").to(torch.int32)
    positions[0] = 0
    rotation = b.rotation(turned, frequencies=frequencies, axes=axes, interleaved=interleaved, q_weight=wq, k_weight=wk, eps=1e-5)
    got = b.rotate(q, k, positions, rotation)
    b.sync()
    for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
        want, size = exact(x, w, 1e-5, positions, frequencies, axes, interleaved)
        assert y.shape == x.shape and y.dtype == dtype
        assert ((y.double() - want).abs() <= bound(want, size, u_of(dtype))).all()
        if not normed:
            assert torch.equal(y[..., turned:], x[..., turned:])
    # over the inputs themselves: the same, and nothing beside them is touched
    rest = wide[:, (heads + kv_heads) * dim :].clone()
    again = b.rotate(q, k, positions, rotation, q_out=q, k_out=k)
    b.sync()
    assert torch.equal(again[0], got[0]) and torch.equal(q, got[0]) and torch.equal(k, got[1]) and torch.equal(wide[:, (heads + kv_heads) * dim :], rest)


def test_position_zero_changes_nothing_and_lengths_stay():
    from paper_2603_20661_b200.backend import Backend
    b = Backend(n_heads=4, n_kv_heads=2, head_dim=128, page_tokens=16, n_pages=1, max_seqs=1, max_tokens=1, max_pages=1, dtype=BF16, device="cuda")
    q, k = torch.randn(9, 4, 128, device="cuda").to(BF16), torch.randn(9, 2, 128, device="cuda").to(BF16)
    r = b.rotation(128)
    got = b.rotate(q, k, torch.zeros(9, dtype=torch.int32, device="cuda"), r)
    assert torch.equal(got[0], q) and torch.equal(got[1], k)
    none = b.rotate(q[:0], k[:0], torch.zeros(0, dtype=torch.int32, device="cuda"), r)
    assert none[0].shape == (0, 4, 128)
    b.sync()


def test_an_element_that_is_not_a_number_stays_in_its_pair():
    from paper_2603_20661_b200.backend import Backend
    b = Backend(n_heads=2, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=1, max_seqs=1, max_tokens=1, max_pages=1, dtype=F16, device="cuda")
    q, k = torch.randn(3, 2, 64, device="cuda").to(F16), torch.randn(3, 2, 64, device="cuda").to(F16)
    q[1, 0, 3], q[1, 1, 60], k[2, 1, 33] = math.nan, math.inf, math.inf
    y, z = b.rotate(q, k, i32([5, 6, 7]), b.rotation(32))
    hurt = torch.zeros_like(q, dtype=torch.bool)
    hurt[1, 0, 3] = hurt[1, 0, 19] = hurt[1, 1, 60] = True
    assert torch.equal(~torch.isfinite(y), hurt) and y[1, 1, 60] == math.inf
    assert (~torch.isfinite(z)).nonzero().tolist() == [[2, 1, 33]]
    # a norm carries it through its head, and no further
    y, _ = b.rotate(q, k, i32([5, 6, 7]), b.rotation(32, q_weight=torch.ones(64, device="cuda")))
    assert torch.isnan(y[1, 0]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2]).all()


LENS = [(1, 1), (1, 17), (16, 16), (5, 40), (0, 9), (33, 65), (70, 70), (2, 1), (0, 0), (130, 300)]


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("dim,turned,interleaved,page,kv_heads,group", [(64, 64, False, 16, 2, 2), (128, 96, True, 32, 1, 7), (128, 128, False, 64, 8, 4), (64, 32, True, 128, 3, 1)])
@pytest.mark.parametrize("placed", [True, False], ids=["places", "positions"])
def test_rotate_append(cache, dtype, dim, turned, interleaved, page, kv_heads, group, placed):
    case = Case(LENS, kv_heads=kv_heads, group=group, dim=dim, page=page, dtype=dtype, cache=cache, seed=5)
    b, heads = case.backend, kv_heads * group
    g = torch.Generator("cuda").manual_seed(6)
    wide = torch.randn(case.tokens, (heads + 2 * kv_heads) * dim + 16, generator=g, device="cuda").to(dtype)
    q, k, v = (t.unflatten(1, (-1, dim)) for t in (wide[:, : heads * dim], wide[:, heads * dim : (heads + kv_heads) * dim], wide[:, (heads + kv_heads) * dim : -16]))
    wq, wk = (1.0 + 0.3 * torch.randn(dim, generator=g, device="cuda") for _ in range(2))
    frequencies = [500000.0 ** (-2.0 * i / turned) for i in range(turned // 2)]
    rotation = b.rotation(turned, frequencies=frequencies, interleaved=interleaved, q_weight=wq, k_weight=wk)
    places = torch.tensor([[p] for n, kv in LENS for p in range(kv - n, kv)], device="cuda")
    positions = places if placed else torch.randint(0, 1 << 20, (case.tokens, 1), generator=g, device="cuda")
    before = {n: getattr(case, n).clone() for n in ("k", "v", "k_scale", "v_scale") if getattr(case, n) is not None}
    got = b.rotate_append(case.cache, case.batch, q, k, v, rotation, positions=None if placed else positions.to(torch.int32))
    b.sync()
    want, size = exact(q, wq, 1e-6, positions, frequencies, [0] * (turned // 2), interleaved)
    assert ((got.double() - want).abs() <= bound(want, size, u_of(dtype))).all()
    keys, size = exact(k, wk, 1e-6, positions, frequencies, [0] * (turned // 2), interleaved)
    at, touched = 0, torch.zeros(before["k"].shape[:3], dtype=torch.bool, device="cuda")
    for i, (n, kv) in enumerate(LENS):
        for p in range(kv - n, kv):
            if p >= 0:
                cell = (case.table[i, p // page].item(), slice(None), p % page)
                touched[cell] = True
                for name, x, e in (("k", keys[at], bound(keys[at], size[at], 0.0)), ("v", v[at].double(), torch.zeros_like(keys[at]))):
                    y = getattr(case, name)[cell].double()
                    if cache == "16":
                        assert ((y - x).abs() <= e + u_of(dtype) * x.abs() * (name == "k")).all()
                        continue
                    scale = getattr(case, name + "_scale")[cell].double()[:, None]
                    amax = (x.abs() + e).amax(-1, keepdim=True)
                    assert ((scale - x.abs().amax(-1, keepdim=True) / TOP[cache]).abs() <= e.amax(-1, keepdim=True) / TOP[cache] + 2.0 ** -22 * scale).all()
                    # a code is off by half a step: 1/2 of int8, 2^-4 of the value in e4m3 (or half its smallest step, 2^-10); and what moved the value before that
                    step = 0.5 * scale if cache == "int8" else torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * scale)
                    assert ((y * scale - x).abs() <= step * (1 + 2.0 ** -4) + 2 * e + 2.0 ** -21 * amax).all()
            at += 1
    for name, x in before.items():           # nothing else was written
        now = getattr(case, name)
        assert torch.equal(now[~touched].view(torch.uint8), x[~touched].view(torch.uint8)), name


def test_without_norm_or_turn_it_is_append():
    """At position 0 and without weights the keys come through unchanged: the same bytes as `append`."""
    for cache in ("16", "int8", "e4m3"):
        a, b = (Case(LENS, kv_heads=2, group=2, dim=64, page=16, dtype=BF16, cache=cache, seed=7) for _ in range(2))
        k, v = (torch.randn(a.tokens, 2, 64, device="cuda").to(BF16) for _ in range(2))
        v[3, 1, 5], k[4, 0, 63] = math.nan, math.inf
        a.backend.append(a.cache, a.batch, k, v)
        q = b.backend.rotate_append(b.cache, b.batch, b.q, k, v, b.backend.rotation(16), positions=torch.zeros(a.tokens, dtype=torch.int32, device="cuda"))
        a.backend.sync(), b.backend.sync()
        assert torch.equal(q, b.q)
        for name in ("k", "v", "k_scale", "v_scale"):
            if getattr(a, name) is not None:
                assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8)), (cache, name)


def test_bad_pages_sequences_and_axes_are_reported():
    from paper_2603_20661_b200.binding import WwwsError
    case = Case([(20, 20), (3, 40)], kv_heads=2, group=2, dim=64, page=16, dtype=BF16, cache="16", seed=8)
    b, r = case.backend, case.backend.rotation(64)
    k, v = (torch.randn(23, 2, 64, device="cuda").to(BF16) for _ in range(2))
    good = b.rotate_append(case.cache, case.batch, case.q, k, v, r).clone()
    b.sync()
    keys = case.k.clone()
    case.table[0, 1] = case.n_pages
    again = b.rotate_append(case.cache, case.batch, case.q, k, v, r)
    with pytest.raises(WwwsError) as e:
        b.sync()
    assert e.value.status == 8 and torch.equal(again, good)          # queries do not need the page
    assert torch.equal(case.k.view(torch.int16), keys.view(torch.int16))
    case.kv_len[1] = 100
    again = b.rotate_append(case.cache, case.batch, case.q, k, v, r, q_out=torch.zeros_like(case.q))
    with pytest.raises(WwwsError):
        b.sync()
    assert torch.equal(again[:20], good[:20]) and (again[20:] == 0).all()


def test_far_pool_and_strides():
    """A pool of more than 2^32 bytes each for keys and values, the sequence's pages at its far end."""
    case = Case([(200, 300)], kv_heads=8, group=1, dim=128, page=128, dtype=BF16, cache="16", seed=12, extra_pages=17000)
    k, v = (torch.randn(200, 8, 128, device="cuda").to(BF16) for _ in range(2))
    case.backend.rotate_append(case.cache, case.batch, case.q, k, v, case.backend.rotation(128), positions=torch.zeros(200, dtype=torch.int32, device="cuda"))
    case.backend.sync()
    assert torch.equal(torch.cat([case.k[case.table[0, p].item()].transpose(0, 1) for p in range(3)])[100:300], k)
    assert torch.equal(torch.cat([case.v[case.table[0, p].item()].transpose(0, 1) for p in range(3)])[100:300], v)


def test_captured_and_replayed():
    case = Case([(4, 40), (1, 9)], kv_heads=2, group=2, dim=64, page=16, dtype=BF16, cache="int8", seed=9)
    k, v = (torch.randn(5, 2, 64, device="cuda").to(BF16) for _ in range(2))
    side = torch.cuda.Stream()
    from paper_2603_20661_b200.backend import Backend
    b = Backend(n_heads=4, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=case.n_pages, max_seqs=2, max_tokens=5, max_pages=case.max_pages, dtype=BF16, cache="int8", device="cuda", stream=side)
    r = b.rotation(64, q_weight=torch.ones(64, device="cuda"))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = b.rotate_append(case.cache, case.batch, case.q, k, v, r)
    for seed in (1, 2):
        case.q.copy_(torch.randn(case.q.shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(BF16))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, case.backend.rotate_append(case.cache, case.batch, case.q, k, v, case.backend.rotation(64, q_weight=torch.ones(64, device="cuda"))))
    case.backend.sync()


def test_refusals():
    from paper_2603_20661_b200.binding import WwwsError
    case = Case([(3, 20)], kv_heads=2, group=2, dim=64, page=16, dtype=BF16, cache="16", seed=10)
    other = Case([(3, 20)], kv_heads=2, group=2, dim=128, page=16, dtype=BF16, cache="16", seed=10)
    b, k = case.backend, torch.zeros(3, 2, 64, dtype=BF16, device="cuda")
    r, pos = b.rotation(64), i32([0, 1, 2])
    for more in (dict(dim=24), dict(dim=80), dict(dim=0), dict(dim=64, frequencies=[1.0]), dict(dim=64, axes=[0]), dict(dim=16, axes=[8] * 8), dict(dim=16, axes=[-1] * 8),
                 dict(dim=64, q_weight=torch.ones(32, device="cuda")), dict(dim=64, k_weight=torch.ones(64))):
        with pytest.raises(ValueError):
            b.rotation(**more)
    for q, kk, p, rr in ((case.q[:2], k, pos, r), (case.q, k[:, :1], pos, r), (case.q.float(), k, pos, r), (case.q, k, pos[:2], r), (case.q, k, pos.long(), r), (case.q, k, pos[:, None].expand(3, 2), r),
                         (case.q, k, pos, other.backend.rotation(64)), (case.q, k, pos, case.batch)):
        with pytest.raises(ValueError):
            b.rotate(q, kk, p, rr)
        with pytest.raises(ValueError):
            b.rotate_append(case.cache, case.batch, q, kk, k, rr, positions=p)
    with pytest.raises(ValueError):
        b.rotate_append(other.cache, case.batch, case.q, k, k, r)
    with pytest.raises(ValueError):
        b.rotate(case.q, k, pos, r, q_out=case.q[:2])
    with pytest.raises(WwwsError) as e:
        b.rotate(case.q, k, pos, b.rotation(64, eps=-1.0))
    assert e.value.status == 1 and "eps" in str(e.value)
    odd = torch.zeros(3 * 4 * 64 + 8, dtype=BF16, device="cuda")[1 : 3 * 4 * 64 + 1].view(3, 4, 64)
    with pytest.raises(WwwsError):
        b.rotate(odd, k, pos, r)
    b.sync()
