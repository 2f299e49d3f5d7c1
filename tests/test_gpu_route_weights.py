"""razer_moe_route / razer_moe_select: where a NaN stands, weights that are far below others, the largest calls."""
import numpy as np
import pytest
import torch

import paper_2501_04052_amd as razer
import step_oracle as so

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def order_of(logits, score, bias):
    """Experts of each row by score + bias, equal ones by the lower index, NaN behind everything."""
    l = np.minimum(logits.astype(np.float64), np.finfo(np.float32).max)
    with np.errstate(over="ignore", invalid="ignore"):
        key = (1.0 / (1.0 + np.exp(-l)) if score == "sigmoid" else l) + (0 if bias is None else bias.astype(np.float64))
    return np.array([sorted(range(len(k)), key=lambda e: (np.isnan(k[e]), 0.0 if np.isnan(k[e]) else -k[e], e)) for k in key])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_a_nan_stands_behind_everything(score):
    rng = np.random.default_rng(3)
    l = rng.standard_normal((40, 70)).astype(np.float32)
    l[:4, :4] = np.array([[0.0, -3.0, NAN, NAN], [NAN, -INF, 1.0, -INF], [NAN, NAN, NAN, -INF], [-INF, NAN, -800.0, -INF]])
    for row in range(4, 40):
        l[row, rng.integers(0, 70, row)] = NAN
    l[39] = NAN
    for bias in (None, np.linspace(0, 0.9, 70), np.linspace(0.9, 0, 70) * 1e3, np.where(np.arange(70) % 3 == 0, NAN, 0.5), np.where(np.arange(70) % 5 == 0, -INF, 0.25)):
        b = None if bias is None else bias.astype(np.float32)
        for dtype in (torch.float32, torch.bfloat16):
            d = torch.from_numpy(l).to(dtype)
            for n, k in ((4, 4), (4, 2), (70, 32), (65, 7)):
                want = order_of(d[:, :n].float().numpy(), score, None if b is None else b[:n])[:, :k]
                ids, w = razer.razer_moe_select(d.cuda()[:, :n], k, score=score, bias=None if b is None else torch.from_numpy(b[:n].copy()).cuda())
                assert np.array_equal(ids.cpu().numpy(), want), (score, n, k)
                w = w.cpu().numpy()
                assert np.isfinite(w).all() and (w[np.isnan(np.take_along_axis(d.float().numpy(), want, 1))] == 0).all()


def test_a_nan_among_the_products():
    """Not the router's rows of finite numbers, but the one with a NaN in it, goes last, whatever its bias."""
    x = torch.ones(3, 64, device="cuda", dtype=torch.bfloat16)
    r = torch.zeros(6, 64, device="cuda", dtype=torch.bfloat16)
    r[2, 5] = NAN
    bias = torch.tensor([0.0, 0.1, 9.0, 0.2, 0.3, 0.4], device="cuda")
    for score in ("softmax", "sigmoid"):
        assert razer.razer_moe_route(x, r, 6, score=score, bias=bias)[0].tolist() == [[5, 4, 3, 1, 0, 2]] * 3


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_renormalized_weights_of_experts_far_below_the_others(score):
    """A bias (or a row far below 0) leads to experts whose weights are nothing beside the others': among themselves they still
    add up to the scale."""
    l = np.array([[0.0, -1000.0, -1001.0, -1000.5], [-900.0, -902.0, -901.0, -5000.0], [3e38, -3e38, 1.0, 2.0], [-INF, -750.0, -750.25, 0.0]], np.float32)
    bias = np.array([0.0, 0.0, 0.0, 0.0], np.float32) if score == "sigmoid" else np.array([0.0, 5000.0, 5000.0, 0.0], np.float32)
    top_k = 2
    if score == "sigmoid":
        bias[1:3] = 5.0
    ids, w = razer.razer_moe_select(torch.from_numpy(l).cuda(), top_k, score=score, bias=torch.from_numpy(bias).cuda(), scale=2.5)
    ids, w = ids.cpu().numpy(), w.double().cpu().numpy()
    assert np.array_equal(ids, order_of(l, score, bias)[:, :top_k])
    c = np.take_along_axis(l.astype(np.float64), ids, 1)
    log_w = c if score == "softmax" else -np.logaddexp(0.0, -c)
    want = np.exp(log_w - np.logaddexp.reduce(log_w, axis=1, keepdims=True)) * 2.5
    assert np.allclose(w, want, rtol=4 * so.U32, atol=1e-37), (w, want)


@pytest.mark.parametrize("tokens,experts", [(1 << 20, 5), ((1 << 19) + 16, 16), (70000, 8), (1040, 16), (1024, 17), (64, 256), (65, 256), (16, 512)])
def test_as_many_tokens_as_there_may_be(tokens, experts):
    """The same choices as in calls of a few tokens, at the ends and in the middle: one and two fragments a workgroup alike."""
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    x = torch.randn(tokens, 64, generator=gen, device="cuda").bfloat16()
    r = torch.randn(experts, 64, generator=gen, device="cuda").bfloat16()
    ids, w = razer.razer_moe_route(x, r, 3)
    for a in (0, tokens // 2 - 7, tokens - 13):
        part, pw = razer.razer_moe_route(x[a:a + 13].contiguous(), r, 3)
        assert torch.equal(ids[a:a + 13], part) and torch.allclose(w[a:a + 13], pw, rtol=2 * so.U32, atol=0)
