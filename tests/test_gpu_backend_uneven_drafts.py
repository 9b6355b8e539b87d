"""The example's requests with drafts, where one request's drafts are always right and another's never."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["16", "int8"])
@pytest.mark.parametrize("most_new", [1, 48, 120])
def test_a_request_that_is_answered_early_grows_no_further(cache, most_new):
    from examples.answer_with_drafts import Answers, TurningDecoder

    class Steady(TurningDecoder):
        """Runs the whole step, and then says: tokens below 10 are followed by themselves, others by the next number."""

        def step(self, backend, rotation, caches, batch, tokens, positions=None, tree=None):
            logits = super().step(backend, rotation, caches, batch, tokens, positions=positions, tree=tree)
            assert torch.isfinite(logits).all()
            after = torch.where(tokens < 10, tokens, tokens + 1)
            return torch.zeros_like(logits).scatter_(1, after[:, None], 1.0)

    prompts = [[20 + i for i in range(7)], [3] * 40, [40, 7], [200 + i for i in range(90)]]
    answers, steps = Answers(Steady(vocab=512), prompts, most_new, cache=cache).with_drafts()
    assert answers == [[27 + i for i in range(most_new)], [3] * most_new, [7] * most_new, [290 + i for i in range(most_new)]]
    assert steps == most_new                                 # a request whose drafts are never right gains a token a step
