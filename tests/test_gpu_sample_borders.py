"""razer_sample where a border (of min_p, of top_p, of the draw) lies at the end of what can be listed, between two bins, or
so close to a token that the sums' own bounds decide."""
import math

import numpy as np
import pytest
import torch

import paper_2501_04052_amd as razer
import step_oracle as so
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


def near(row, uniform, top_k, tokens, logprobs, share=2.0 ** -26):
    """Each token is one whose part of the running sum lies within `share` of uniform times the sum (sums are right to 2^-27 of
    themselves, the one on either side), its logarithm within fp32 of that."""
    l = row.astype(np.float64)
    order = np.argsort(-l, kind="stable")
    place = np.empty(len(l), np.int64)
    place[order] = np.arange(len(l))
    w = np.exp(l[order] - l.max())[:top_k]
    run = np.cumsum(w)
    want = uniform.astype(np.float64) * run[-1]
    low, high = (np.minimum(np.searchsorted(run, want * (1 + s), side="right"), len(w) - 1) for s in (-share, share))
    at = place[tokens]
    bad = (at < low) | (at > high)
    assert not bad.any(), (uniform[bad][:4], tokens[bad][:4], at[bad][:4], low[bad][:4], high[bad][:4])
    logp = np.log(w[at] / run[-1])
    assert (np.abs(logprobs - logp) <= 2 * so.U32 * np.abs(logp) + share).all()


@pytest.mark.parametrize("first,second", [(3000, 2028), (1500, 1000), (2000, 100)])
@pytest.mark.parametrize("vocab", [0, 60000])
def test_draws_at_the_border_of_a_bin(first, second, vocab):
    """One logit at 0, many alike whose bin's sum errs in one direction, many half an octave and more below, and top_k among
    some far below: random numbers around the border between the two groups draw one of its neighbours."""
    rng = np.random.default_rng(first)
    for value in (-1.8167176246643066, -1.3, -0.7771, -2.90123, -0.1 - 2 * rng.random()):
        l = np.full(max(vocab, 1 + first + second + 100), -60.0, np.float32)
        value = np.float32(value)
        l[:1 + first + second + 100] = np.concatenate([[0.0], np.full(first, value), np.full(second, value - np.float32(0.5)), np.full(100, value - np.float32(20.0))])
        k = 1 + first + second + 50
        w = np.exp(np.sort(l.astype(np.float64))[::-1][:k])
        u = np.float32((1 + first * math.exp(float(value))) / w.sum())
        us = np.array([np.float32(u) + np.float32(i * 2.0 ** -24) for i in range(-12, 13)], np.float32)
        rows = up(np.tile(l, (len(us), 1)))
        tok, lp = razer.razer_sample(rows, up(us), top_k=torch.full((len(us),), k, dtype=torch.int32, device="cuda"))
        near(l, us, k, tok.cpu().numpy(), lp.double().cpu().numpy())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(4000, 200), (600, 2500), (8, 45000)])
def test_uniform_of_one_gives_the_last_that_stays(rows, vocab, dtype):
    """Or one behind the last that weighs 2^-57 of the first: a running sum that reaches the whole by rounding does not end it."""
    rng = np.random.default_rng(rows)
    x = up(rng.standard_normal((rows, vocab)) * rng.choice([3.0, 10.0, 30.0], (rows, 1))).to(dtype)
    l = x.double().cpu().numpy()
    for top_k in (None, rng.integers(1, vocab + 1, rows)):
        tok, _ = razer.razer_sample(x, up(rng.choice([1.0, 1.5], rows)), top_k=None if top_k is None else up(top_k, torch.int32))
        tok = tok.cpu().numpy()
        for r in range(rows):
            order = np.argsort(-l[r], kind="stable")[:None if top_k is None else top_k[r]]
            at = np.flatnonzero(order == tok[r])
            last = np.flatnonzero(np.exp(l[r, order] - l[r, order[0]]) >= 2.0 ** -57)[-1]
            assert len(at) == 1 and at[0] >= last, (r, at, last, len(order))
