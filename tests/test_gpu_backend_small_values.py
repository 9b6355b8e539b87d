"""The softmax weights keep their precision whatever the size of the values: f16 has no room below 2^-24, so weights that are multiplied by a
row's scale have to be kept relative to the largest scale, and small ones away from the subnormals."""
import pytest
import torch

from tests.backend_cases import Case, attend_exact

pytestmark = pytest.mark.gpu


def bound(case, want, weight, scores, floor):
    """As `attend_bound` for f16, but every absolute term goes with the values: u = 2^-11; outputs are rounded once (u |o|, half a subnormal step
    2^-25); weights rounded to f16 and the sum of them (2 u W); scores and exponentials in fp32 (2 d W) and sums of kv terms ((2 kv + 64) 2^-24 W); and
    weights in f16's subnormals lose at most half a step, 2^-25 over the factor that the kernel multiplies them with: `floor` relative to the
    row's largest weight and the largest value, per key."""
    kv = max(kv for _, kv in case.lens)
    u, d = 2.0 ** -11, scores[..., None] * (case.dim + 8) * 2.0 ** -24 + 2.0 ** -21
    top = max(torch.nan_to_num(case.rows("v", i)).abs().max().item() for i in range(len(case.lens)))
    return (u * want.abs() + 2.0 ** -25 + (2 * u + 2 * d + (2 * kv + 64) * 2.0 ** -24) * weight + floor * kv * top) * (1 + 2.0 ** -7)


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -8, 2.0 ** -12])
@pytest.mark.parametrize("lens", [[(1, 4000)], [(3, 1000)], [(70, 4000)], [(300, 1500), (40, 500)]], ids=str)
def test_one_key_far_ahead_of_many(cache, dim, size, lens):
    """One key 8 nats ahead of the rest, whose sum weighs about as much as it does."""
    case = Case(lens, kv_heads=2, group=4, dim=dim, page=32, dtype=torch.float16, cache=cache, seed=21)
    g = torch.Generator("cuda").manual_seed(22)
    way = torch.randn(dim, generator=g, device="cuda")
    way /= way.norm()
    # scores of the others: +-1 about 0 along `way`; the key ahead: 8
    case.q.copy_((way * dim ** 0.5).expand_as(case.q) + 0.05 * torch.randn(case.q.shape, generator=g, device="cuda"))
    for i, (q_len, kv) in enumerate(lens):
        at = (kv - q_len) // 2
        page, slot = case.table[i, at // 32].item(), at % 32
        from tests.backend_cases import quantise
        row = (way * 8.0).expand(2, dim)
        if cache == "16":
            case.k[page, :, slot] = row.to(case.dtype)
        else:
            code, scale = quantise(row, cache)
            case.k.view(torch.uint8)[page, :, slot] = code.view(torch.uint8)
            case.k_scale[page, :, slot] = scale
    if cache == "16":
        case.v.mul_(size)
    else:
        case.v_scale.mul_(size)
    got = case.attend(0, 0)
    case.backend.sync()
    want, weight, scores = attend_exact(case, 0, 0, None)
    # the smallest factor of a kernel: 2^7, of the tile kernel over 16-bit values
    off = (got.double() - want).abs() - bound(case, want, weight, scores, 2.0 ** -32)
    assert (off <= 0).all(), f"{off.max().item():.3g} too far, outputs up to {want.abs().max().item():.3g}"


@pytest.mark.parametrize("cache", ["int8", "e4m3"])
@pytest.mark.parametrize("rising", [True, False])
@pytest.mark.parametrize("lens", [[(1, 2000)], [(100, 2000)], [(300, 700)]], ids=str)
def test_value_scales_that_change_along_the_sequence(cache, rising, lens):
    """Scales that grow or shrink by 2^24 from a sequence's first key to its last: what was summed before is not lost when a larger one comes, and small ones
    behind it stay exact relative to the outputs that they make."""
    case = Case(lens, kv_heads=2, group=4, dim=64, page=64, dtype=torch.float16, cache=cache, seed=23)
    for i, (_, kv) in enumerate(lens):
        for p in range(-(-kv // 64)):
            f = 2.0 ** (-24.0 * p * 64 / kv)
            id = case.table[i, (-(-kv // 64) - 1 - p) if rising else p].item()
            case.v_scale[id] *= f
    got = case.attend(0, 0)
    case.backend.sync()
    assert torch.isfinite(got).all()
    want, weight, scores = attend_exact(case, 0, 0, None)
    off = (got.double() - want).abs() - bound(case, want, weight, scores, 2.0 ** -32)
    assert (off <= 0).all(), f"{off.max().item():.3g} too far"


@pytest.mark.parametrize("cache", ["int8", "e4m3"])
@pytest.mark.parametrize("lens", [[(1, 70)], [(70, 200)]], ids=str)
def test_largest_and_absent_values(cache, lens):
    """Value scales at f16's upper end, and none at all (scale 0)."""
    case = Case(lens, kv_heads=1, group=4, dim=64, page=16, dtype=torch.float16, cache=cache, seed=24)
    scale = case.v_scale.clone()
    case.v_scale.copy_(scale * (30000.0 / torch.nan_to_num(case.rows("v", 0)).abs().max().item()))
    got = case.attend(0, 0)
    want, weight, scores = attend_exact(case, 0, 0, None)
    assert ((got.double() - want).abs() <= bound(case, want, weight, scores, 2.0 ** -32)).all()
    case.v_scale.copy_(scale * 0.0)
    got = case.attend(0, 0)
    case.backend.sync()
    assert (got == 0).all()


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("lens", [[(1, 4000)], [(20, 4000)], [(70, 4000)]], ids=str)
def test_many_keys_that_are_faint_alone(cache, lens):
    """One key 17.5 nats ahead whose value is 0, 4,000 others with a value of 1: what is left is their sum, 1e-4, though each weighs 2^-25.2, less than half
    of f16's smallest number."""
    case = Case(lens, kv_heads=1, group=4, dim=64, page=32, dtype=torch.float16, cache=cache, seed=25)
    way = torch.ones(64, device="cuda") / 8.0
    case.q.copy_((way * 8.0).expand_as(case.q))
    page, slot = case.table[0, 1].item(), 3                          # key 35
    if cache == "16":
        case.k.copy_(torch.where(torch.isnan(case.k), case.k, 0.0))
        case.v.copy_(torch.where(torch.isnan(case.v), case.v, 1.0))
        case.k[page, :, slot], case.v[page, :, slot] = (way * 17.5).half(), 0.0
    else:
        one = 1 if cache == "int8" else 0x38                         # code 1
        case.k.view(torch.uint8).zero_()
        case.v.view(torch.uint8).fill_(one)
        for scale in (case.k_scale, case.v_scale):
            scale.copy_(torch.where(torch.isnan(scale), scale, 1.0))
        case.k.view(torch.uint8)[page, :, slot], case.k_scale[page, :, slot] = one, 17.5 / 8.0
        case.v.view(torch.uint8)[page, :, slot] = 0
    got = case.attend(0, 0)
    case.backend.sync()
    want, weight, scores = attend_exact(case, 0, 0, None)
    assert 0.8e-4 < want.min().item() and want.max().item() < 1.2e-4
    off = (got.double() - want).abs() - bound(case, want, weight, scores, 2.0 ** -32)
    assert (off <= 0).all(), f"{off.max().item():.3g} too far"
