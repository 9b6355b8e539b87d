"""The operators together, as the example uses them: prompts in chunks and answers token by token over the paged cache give what the whole
text at once gives, and masked verdicts are among their choices."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("answer_requests", os.path.join(ROOT, "examples", "answer_requests.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("cache", ["16", "int8", "e4m3"])
def test_steps_over_the_cache_equal_the_whole_text(example, cache):
    """A cached key or value is the same code whether its token came in a chunk, alone or with the whole text, as long as the layers'
    inputs agree.  In a model of one layer they do (embeddings); what is left is the order of sums and the weights' rounding: each of
    512 outputs of the layer is off by a few bf16 roundings of its terms, and a logit adds 512 of them in fp32, so 2^-5 of the logits'
    own size is an ample bound, far below what a wrong position, mask or page would do."""
    model = example.Decoder(vocab=512, layers=1, seed=3)
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(0, 512, (n,), generator=g).tolist() for n in (1, 17, 40, 129, 70)]
    stepwise = example.Serving(model, prompts, 12, page=16, cache=cache, chunk=32)
    logits = stepwise.answer([6] * len(prompts))
    whole = example.Serving(model, [p + a[:5] for p, a in zip(prompts, stepwise.answers)], 12, page=64, cache=cache, chunk=1000)
    want = whole.answer([1] * len(prompts))
    for i in range(len(prompts)):
        assert len(stepwise.answers[i]) == 6
        a, b = logits[i].float(), want[i].float()
        assert (a - b).abs().max() <= b.abs().max() * 2.0 ** -5, i


def test_verdicts_are_among_their_choices(example):
    model = example.Decoder(vocab=300, layers=1, seed=5)
    s = example.Serving(model, [[1, 2, 3], [4]], 4)
    logits = torch.stack([v for _, v in sorted(s.answer([1, 1]).items())])
    got = s.verdicts(logits, [7, 255, 299])
    assert got == [int(x) for x in logits[:, [7, 255, 299]].float().argmax(-1)]


def test_the_example_runs(example, capsys):
    s = example.main(["--cache", "e4m3", "--requests", "6", "--most-new", "5"])
    assert "tokens/s" in capsys.readouterr().out and all(1 <= len(a) <= 5 for a in s.answers)
