"""Scores that are equal although the logits are not: beside a total of 2^60 the 64-bit scores of a row are a few values, and ties go to the lowest row and token."""
import pytest
import torch

from tests.test_gpu_backend_beams import check

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [700, 5000, 70001])
@pytest.mark.parametrize("total", [2.0 ** 60, -2.0 ** 60])
def test_totals_that_leave_no_room_for_logits(dtype, vocab, total):
    g = torch.Generator("cuda").manual_seed(vocab)
    logits = torch.randn(6, vocab, generator=g, device="cuda").to(dtype)
    totals = torch.full((6,), total, device="cuda")
    _, parent, token = check(logits, totals, 3, 100)
    assert (parent == torch.tensor([[0], [3]], device="cuda")).all() and (token == torch.arange(100, device="cuda")).all()
    # some tokens are ahead by more than a step of such scores (128 and 256).  (The others' scores lie about 3,000 lower on either side of a border between two steps, 23.5 x 128,
    # so that their order follows from the exact scores, which `check` holds them against, and not from their tokens alone.)
    ahead = torch.arange(vocab // 3, vocab, 29, device="cuda")[:20]
    logits[:, ahead] += 3000.0
    _, parent, token = check(logits, totals, 1, 33)
    assert (token[:, : len(ahead)] == ahead).all()
