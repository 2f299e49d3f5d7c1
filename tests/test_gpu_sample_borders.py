"""razer_sample where a border of min_p or top_p lies at the end of what can be listed, or between two bins."""
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


# temperature, a logit below 0, min_p: exp(logit / temperature) is min_p (1 + 6e-10 .. 1.4e-9), and both lie within 2^-22 of a
# 64th of an octave, the logit so that it counts to the bin behind
CLOSE = [(1.2040646076202393, -8.619791030883789, 0.0007779014413245022), (1.0963901281356812, -0.2493617832660675, 0.7965710759162903),
         (0.501380205154419, -0.4615636467933655, 0.39828553795814514), (0.924815833568573, -0.8513725996017456, 0.39828553795814514),
         (1.6412262916564941, -10.611781120300293, 0.0015558028826490045), (0.5895054936408997, -0.13407649099826813, 0.7965710759162903)]


@pytest.mark.parametrize("vocab", [70, 60000])
def test_min_p_at_a_bin_s_border(vocab):
    n = len(CLOSE)
    x = torch.full((n, vocab), -50.0, device="cuda")
    x[:, 7] = 0.0
    for r, (t, l, m) in enumerate(CLOSE):
        assert math.exp(np.float64(np.float32(l)) / np.float64(np.float32(t))) >= (1 + 1e-10) * float(np.float32(m))
        x[r, 60] = l
    t, m = np.array([c[0] for c in CLOSE]), np.array([c[2] for c in CLOSE])
    assert check(x, np.full(n, 0.9999), t, min_p=m, sure=False).tolist() == [60] * n
    assert check(x, np.full(n, 0.0001), t, min_p=m, sure=False).tolist() == [7] * n
