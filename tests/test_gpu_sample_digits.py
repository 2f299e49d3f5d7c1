"""razer_sample where the order is resolved digit by digit of the logits (more than 2^18 tokens, or too many alike): sums and
logarithms as exact as the header says, to the longest vocabulary."""
import math

import numpy as np
import pytest
import torch

import paper_2501_04052_amd as razer
import step_oracle as so
from test_gpu_sample import up
from test_gpu_sample_borders import near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [(1 << 18) + 64, 1 << 22, 1 << 24])
def test_a_tail_that_weighs_in_sum_alone(vocab, dtype):
    """One logit at 0, all others far below it, so that together they have some 2^-15 of the weight: a random number beyond the
    first one's share draws among them, and the logarithms are theirs."""
    low = torch.tensor(-15 * math.log(2) - math.log(vocab), dtype=dtype).item()
    x = torch.full((1, vocab), low, device="cuda", dtype=dtype)
    x[0, vocab // 3] = 0.0
    w = math.exp(low)
    total = 1.0 + (vocab - 1) * w
    for tail in (0.0, 0.1, 0.5, 0.9):
        u = np.float32((1.0 + tail * (vocab - 1) * w) / total) if tail else np.float32(0.9999)
        tok, lp = (t.item() for t in razer.razer_sample(x, up(np.array([u]))))
        if not tail:
            assert tok == vocab // 3 and abs(lp + math.log(total)) <= 2.0 ** -26 + 2 * so.U32 * math.log(total)
            continue
        place = (float(u) * total - 1.0) / w                               # of the others, in their order
        at = tok if tok < vocab // 3 else tok - 1
        assert tok != vocab // 3 and abs(at - place) <= 2.0 ** -26 * total / w + 1, (tok, place)
        want = low - math.log(total)
        assert abs(lp - want) <= 2 * so.U32 * abs(want) + 2.0 ** -26


@pytest.mark.parametrize("vocab", [300007, 1 << 21])
def test_light_tokens_beyond_the_bins(vocab):
    """A long vocabulary whose tokens weigh between 2^-8 and 2^-57 of the largest; draws all along the order, also of what
    weighs least, with the logarithms of their own weights."""
    rng = np.random.default_rng(vocab)
    l = (-rng.uniform(8 * math.log(2), 57 * math.log(2), vocab)).astype(np.float32)
    l[5] = 0.0
    order = np.argsort(-l, kind="stable")
    run = np.cumsum(np.exp(l[order].astype(np.float64)))
    us = np.unique((run[[0, 1, 10, 1000, vocab // 100, vocab // 10, vocab // 4, vocab // 2]] / run[-1]).astype(np.float32))
    tok, lp = razer.razer_sample(up(np.tile(l, (len(us), 1))), up(us))
    near(l, us, vocab, tok.cpu().numpy(), lp.double().cpu().numpy())
    # top_p and min_p that end among them
    p, m = np.float32(0.9), np.float32(1e-6)
    tok, lp = (t.item() for t in razer.razer_sample(up(l[None]), up(np.array([0.75])), top_p=up(np.array([p])), min_p=up(np.array([m]))))
    n = min(1 + int((run < float(p) * run[-1]).sum()), int((np.exp(l[order].astype(np.float64)) >= float(m)).sum()))
    near(l, np.array([0.75], np.float32), n, np.array([tok]), np.array([lp]))


def test_the_last_of_a_long_row_is_drawn_at_the_end():
    """uniform 1 gives the last token that stays, also where it weighs 2^-50 of the first and less than the sum's own rounding."""
    vocab = (1 << 18) + 1000
    x = torch.full((1, vocab), -20.0, device="cuda")
    x[0, :1000] = 0.0
    x[0, 4321] = -35.0
    tok, lp = razer.razer_sample(x, up(np.ones(1)))
    total = 1000 + (vocab - 1001) * math.exp(-20.0)
    assert tok.item() == 4321 and abs(lp.item() + 35.0 + math.log(total)) <= 1e-5
    k = torch.full((1,), vocab - 1, dtype=torch.int32, device="cuda")
    assert razer.razer_sample(x, up(np.ones(1)), top_k=k)[0].item() == vocab - 1
