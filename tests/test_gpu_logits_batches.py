"""Logits shaping of batches large enough for the kernel that sorts histories (more than 2,048 blocks of 2,048 tokens): every way it takes."""
import pytest
import torch

from tests.test_gpu_backend_logits import BF16, F16, F32, backend, plain, run, token_of

pytestmark = pytest.mark.gpu


def inputs(rows, vocab, history, bias, seed, spread):
    """The first three rows have `history` tokens and `bias` entries, the others a few."""
    g = torch.Generator().manual_seed(seed)
    ends = lambda v: torch.tensor([sum(v[:i]) for i in range(len(v) + 1)], dtype=torch.int32)                    # noqa: E731
    lens, nb = [history if r < 3 else 20 * (r % 3) for r in range(rows)], [bias if r < 3 else r % 2 for r in range(rows)]
    ids = lambda n: (torch.rand(n, generator=g) ** 3 * min(vocab, spread)).to(torch.int32)                       # noqa: E731
    words = (vocab + 31) // 32
    s = {"history": ids(sum(lens)), "history_start": ends(lens), "prompt_len": torch.tensor([n // 3 for n in lens], dtype=torch.int32),
         "repetition": 0.7 + torch.rand(rows, generator=g), "presence": torch.rand(rows, generator=g) - 0.3, "frequency": 0.05 * torch.rand(rows, generator=g),
         "bias_id": ids(sum(nb)), "bias_value": 5 * torch.randn(sum(nb), generator=g), "bias_start": ends(nb),
         "mask": torch.randint(-2 ** 31, 2 ** 31 - 1, (2, words), generator=g, dtype=torch.int64).to(torch.int32),
         "mask_index": torch.tensor([r % 3 - 1 for r in range(rows)], dtype=torch.int32)}
    return s, torch.randn(rows, vocab, generator=g) * 4


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,history,bias,spread", [
    (2100, 33, 40, 3, 33), (2100, 517, 60, 3, 517), (700, 5003, 100, 5, 5003), (60, 80011, 3000, 40, 80011),
    (700, 5003, 900, 4, 1000),              # more than 128 touched tokens in a slice
    (700, 5003, 900, 700, 3000),            # more than 512 bias entries
    (60, 80011, 20000, 2047, 50000)])       # more than 8,192 entries of history in a part
@pytest.mark.parametrize("shift", [0, 3])
def test_bit_for_bit(dtype, rows, vocab, history, bias, spread, shift):
    s, x = inputs(rows, vocab, history, bias, rows + vocab + shift, spread)
    x = x.to(dtype)
    want = plain(x.float(), s, F32).to(dtype)
    b = backend(rows)
    wide = torch.full((rows, vocab + 21), 9.0, dtype=dtype, device="cuda")
    view = wide[:, shift : shift + vocab]
    view.copy_(x)
    got, token = run(b, view, s)
    assert torch.equal(got.float(), want.float()) and torch.equal(token, token_of(want))
    got, token = run(b, view, s, out=view)
    assert torch.equal(got.float(), want.float()) and torch.equal(token, token_of(want))
    assert (wide[:, :shift] == 9.0).all() and (wide[:, shift + vocab :] == 9.0).all()


def test_special_values():
    """Rows with ties, nothing left, NaN and infinities amid a large batch."""
    x = torch.randn(2100, 300) - 50
    x[0] = 1.0
    x[1, 200] = x[1, 100] = 5.0
    x[2] = -float("inf")
    x[3] = float("nan")
    x[4, 7], x[4, 9] = float("nan"), 2.0
    x[5, 11] = float("inf")
    x[6] = -0.0
    x[6, 40] = 0.0
    got, token = run(backend(2100), x.cuda(), {})
    assert torch.equal(torch.nan_to_num(got, nan=7.0), torch.nan_to_num(x, nan=7.0)) and torch.equal(token, token_of(x))
    assert token[:7].tolist() == [0, 100, -1, -1, 9, 11, 0]
