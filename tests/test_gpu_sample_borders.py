"""razer_sample where a border of min_p or top_p lies at the end of what can be listed."""
import math

import numpy as np
import pytest
import torch

from test_gpu_sample import check, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [5200, 60000])
@pytest.mark.parametrize("listed", [4095, 4096, 4097])
def test_a_cut_behind_the_last_listed_token(listed, vocab, dtype):
    """So many equal logits stay, and what does not has weight of its own: 1/e each."""
    rng = np.random.default_rng(listed)
    x = torch.full((5, vocab), -1.0, device="cuda")
    for r in range(5):
        x[r, up(rng.permutation(vocab)[:listed], torch.int64)] = 0.0
    x, u = x.to(dtype), np.array([0.0, 0.3, 0.6, 0.9, 0.9999])
    check(x, u, min_p=np.full(5, 0.99))
    check(x, u, top_p=np.full(5, (listed - 0.5) / (listed + (vocab - listed) * math.exp(-1.0))))
    check(x, u, top_k=np.full(5, listed), min_p=np.full(5, 0.99))
