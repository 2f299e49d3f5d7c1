"""moe_decoder.MoeDecoder refuses a step that it has no answer for (runs without a GPU)."""
import pytest
import torch

from paper_2501_04052_amd import moe_decoder


class NoPool:
    def step(self, fresh):
        raise AssertionError("the pool is changed before the step is refused")


@pytest.mark.parametrize("fresh", [(0, 1), (1, 0, 2), (3, 0), (0,)])
def test_a_request_without_new_tokens_is_refused(fresh):
    """The row ahead of its (empty) place in the step is another request's, or the last one's: no logits of its own."""
    model = moe_decoder.MoeDecoder(torch.zeros(10, 32, dtype=torch.bfloat16), [], torch.ones(32), None)
    with pytest.raises(ValueError):
        model.step(NoPool(), [torch.zeros(n, dtype=torch.int64) for n in fresh])
