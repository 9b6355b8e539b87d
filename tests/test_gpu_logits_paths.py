"""Logits shaping where its kernel takes another way: slices crowded with touched tokens, histories and bias lists past what a block keeps."""

import pytest
import torch

from tests.test_gpu_backend_logits import BF16, F16, F32, backend, plain, run, token_of

pytestmark = pytest.mark.gpu


def inputs(rows, vocab, history, bias, seed, spread):
    g = torch.Generator().manual_seed(seed)
    ends = lambda v: torch.tensor([sum(v[:i]) for i in range(len(v) + 1)], dtype=torch.int32)                    # noqa: E731
    lens, nb = [max(0, history - 3 * r) for r in range(rows)], [max(0, bias - r) for r in range(rows)]
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
    (3, 5003, 600, 0, 1000),            # more than 128 touched tokens in a slice
    (2, 3000, 900, 700, 3000),          # more than 512 bias entries
    (3, 20011, 14000, 5, 20011),        # more than 8,192 entries of history in a part
    (2, 4099, 9000, 2047, 1500),        # all of it
    (300, 2100, 700, 3, 900),           # the same with a block per row
    (200, 1030, 8700, 600, 1030)])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_bit_for_bit(dtype, rows, vocab, history, bias, spread, shift):
    """Fresh outputs and in place, and inputs that start off a 16-byte boundary."""
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


def test_most_history_that_a_row_may_have():
    vocab, n = 3000, (1 << 20) - 1
    g = torch.Generator().manual_seed(5)
    history = (torch.rand(n, generator=g) ** 2 * vocab).to(torch.int32)
    s = {"history": history, "history_start": torch.tensor([0, n], dtype=torch.int32), "prompt_len": torch.tensor([1000], dtype=torch.int32),
         "frequency": torch.tensor([2.0 ** -10]), "presence": torch.tensor([0.25]), "repetition": torch.tensor([1.5])}
    x = torch.randn(1, vocab, generator=g)
    got, token = run(backend(1), x.cuda(), s)
    want = plain(x, s, F32)
    assert torch.equal(got, want) and torch.equal(token, token_of(want))
    s["history"] = torch.full((n,), 7, dtype=torch.int32)              # one token, as often as can be
    s["prompt_len"] = torch.tensor([0], dtype=torch.int32)
    got, _ = run(backend(1), x.cuda(), s)
    assert torch.equal(got, plain(x, s, F32))


@pytest.mark.parametrize("prompt", [2 ** 31 - 1, 2 ** 31 - 40, 50, -2 ** 31])
def test_prompts_longer_than_their_history(prompt):
    """A prompt length past the end of a row's history says that all of it is prompt, wherever the row's history starts; one below zero, none."""
    s, x = inputs(3, 500, 40, 0, 9, 500)
    s["prompt_len"][:] = prompt
    got, token = run(backend(3), x.cuda(), s)
    s["prompt_len"] = torch.full((3,), 40 if prompt > 0 else 0, dtype=torch.int32)
    want = plain(x, s, F32)
    assert torch.equal(got, want) and torch.equal(token, token_of(want))


def test_an_empty_set_of_masks():
    """No masks in this step: rows that ask for one are reported, rows that do not are left alone."""
    from paper_2603_20661_b200.binding import WwwsError
    x = torch.randn(2, 100)
    none = {"mask": torch.zeros(0, 4, dtype=torch.int32), "mask_index": torch.tensor([-1, -1], dtype=torch.int32)}
    b = backend(2)
    got, token = run(b, x.cuda(), none)
    assert torch.equal(got, x) and torch.equal(token, token_of(x))
    none["mask_index"][1] = 0
    with pytest.raises(WwwsError) as e:
        run(b, x.cuda(), none)
    assert e.value.status == 8 and "mask" in str(e.value)
    with pytest.raises(WwwsError) as e:
        run(b, x.cuda(), {"mask": none["mask"]})                       # a mask per row is asked for
    assert e.value.status == 1
