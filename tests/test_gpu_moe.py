"""razer_moe_route and razer_moe_experts on the GPU against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2501_04052_amd as razer
import step_oracle as so
from gpu_util import launched_kernels

pytestmark = pytest.mark.gpu


# ---- routing --------------------------------------------------------------------------------------------------

def check_route(got, want, keys, delta):
    """keys [tokens][experts]: what the order goes by; delta [tokens]: how far a product (and so a key) may be off."""
    (ids, w), (wi, ww, gap) = got, want
    ids, w = ids.cpu().numpy(), w.double().cpu().numpy()
    # every row: an order that keys off by delta can give
    chosen = np.take_along_axis(keys, ids, 1)
    rest = keys.copy()
    np.put_along_axis(rest, ids, -np.inf, 1)
    assert all(len(set(row)) == len(row) for row in ids.tolist())
    assert (np.diff(chosen, axis=1) <= 2 * delta[:, None]).all() and (rest.max(1) <= chosen[:, -1] + 2 * delta).all()
    same = (ids == wi).all(1)
    assert same[gap > 2 * delta].all()
    assert (np.abs(w - ww) <= np.abs(ww) * (4 * delta[:, None] + 4 * so.U32) + 1e-37)[same].all()


@pytest.mark.parametrize("tokens,hidden,experts,top_k", [(1, 32, 1, 1), (1, 4096, 64, 8), (3, 96, 5, 5), (16, 256, 16, 2), (17, 544, 33, 6), (65, 1024, 200, 8), (300, 160, 512, 32), (2, 8192, 256, 3)])
def test_route(tokens, hidden, experts, top_k):
    rng = np.random.default_rng(tokens + hidden + experts)
    x, r = so.bf16(rng.standard_normal((tokens, hidden))), so.bf16(rng.standard_normal((experts, hidden)) * hidden ** -0.5)
    bias = (0.3 * rng.standard_normal(experts)).astype(np.float32)
    logits = x.astype(np.float64) @ r.astype(np.float64).T
    delta = 32 * so.U32 * (np.abs(x).astype(np.float64) @ np.abs(r).astype(np.float64).T).max(1)
    xd = torch.from_numpy(x).cuda().bfloat16()
    wide = torch.zeros(tokens, hidden + 8, device="cuda", dtype=torch.bfloat16)
    wide[:, :hidden] = xd
    rd, bd = torch.from_numpy(r).cuda().bfloat16(), torch.from_numpy(bias).cuda()
    for score in ("softmax", "sigmoid"):
        for use_bias, renorm, scale in ((False, True, 1.0), (True, False, 2.5), (True, True, 0.5)):
            got = razer.razer_moe_route(wide[:, :hidden] if use_bias else xd, rd, top_k, score=score, bias=bd if use_bias else None, renormalize=renorm, scale=scale)
            keys = (logits if score == "softmax" else 1 / (1 + np.exp(-logits))) + (bias.astype(np.float64) if use_bias else 0)
            check_route(got, so.route(logits, top_k, score, bias if use_bias else None, renorm, scale), keys, delta)


def test_equal_scores_go_to_the_lower_index():
    x = torch.ones(5, 64, device="cuda", dtype=torch.bfloat16)
    r = torch.zeros(130, 64, device="cuda", dtype=torch.bfloat16)
    r[[7, 70, 129, 64]] = 0.25
    for score in ("softmax", "sigmoid"):
        ids, w = razer.razer_moe_route(x, r, 6, score=score)
        assert ids.tolist() == [[7, 64, 70, 129, 0, 1]] * 5 and torch.allclose(w.sum(1), torch.ones(5, device="cuda"), atol=2e-7)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,experts,top_k", [(1, 2, 1), (5, 8, 2), (130, 65, 4), (9, 512, 7)])
def test_select(dtype, tokens, experts, top_k):
    rng = np.random.default_rng(tokens * experts)
    wide = torch.from_numpy(rng.standard_normal((tokens, experts + 3)) * 3).to(dtype).cuda()
    l = wide[:, :experts]
    for score in ("softmax", "sigmoid"):
        ids, w, _ = so.route(l.double().cpu().numpy(), top_k, score)
        got = razer.razer_moe_select(l, top_k, score=score)
        assert np.array_equal(got[0].cpu().numpy(), ids) and np.allclose(got[1].double().cpu().numpy(), w, rtol=4 * so.U32, atol=1e-37)


def test_select_with_infinities_and_nan():
    inf, nan = float("inf"), float("nan")
    l = torch.tensor([[0.0, -inf, nan, 1.0], [-inf] * 4, [nan] * 4, [inf, 1.0, inf, 0.0], [3e38, -3e38, 0.0, -inf]], device="cuda")
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            ids, w, _ = so.route(l.double().cpu().numpy(), 3, score, renormalize=renorm)
            gi, gw = razer.razer_moe_select(l, 3, score=score, renormalize=renorm)
            assert np.array_equal(gi.cpu().numpy(), ids) and np.allclose(gw.double().cpu().numpy(), w, rtol=1e-6, atol=1e-37), (score, renorm, gi, gw, ids, w)


# ---- experts --------------------------------------------------------------------------------------------------

def stack(rng, experts, rows, cols, block=16, sv=(5.0, 8.0)):
    """(RazerExperts, their exact values)"""
    w = [razer.razer_quantize(torch.from_numpy((rng.standard_normal((rows, cols)) * cols ** -0.5).astype(np.float32)).cuda(), razer.WEIGHT, sv, block=block) for _ in range(experts)]
    s = razer.RazerExperts.stack(w)
    return s, [razer.razer_dequant(t).double().cpu().numpy() for t in w]


def check_experts(got, want, bound):
    got = got.double().cpu().numpy()
    bad = np.abs(got - want) > bound
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], bound[bad][:4])


SIZES = [  # tokens, hidden, inter, experts, top_k, out
    (1, 64, 32, 1, 1, 64), (1, 2048, 1024, 16, 8, 2048), (1, 96, 160, 4, 2, 96), (2, 1056, 224, 3, 3, 64), (4, 256, 512, 9, 1, 256), (5, 512, 96, 2, 2, 512), (8, 288, 320, 40, 4, 288),
    (9, 256, 128, 3, 2, 256), (17, 160, 2528, 5, 3, 160), (40, 320, 64, 2, 1, 352), (64, 128, 256, 64, 8, 128), (70, 256, 160, 2, 2, 256), (200, 96, 96, 3, 1, 96), (33, 1184, 1120, 4, 4, 1184)]


@pytest.mark.parametrize("tokens,hidden,inter,experts,top_k,out", SIZES)
@pytest.mark.parametrize("block", [16, 32])
def test_experts(tokens, hidden, inter, experts, top_k, out, block):
    rng = np.random.default_rng(tokens * 7 + hidden + inter + block)
    act = ("silu", "gelu", "relu")[(tokens + block // 16) % 3]
    gate, g64 = stack(rng, experts, inter, hidden, block)
    up, u64 = stack(rng, experts, inter, hidden, block) if (tokens + hidden // 32) % 4 else (None, None)
    down, d64 = stack(rng, experts, out, inter, 16 if block == 32 else 32, (4.5, 9.0))
    x = so.bf16(rng.standard_normal((tokens, hidden)))
    ids = np.stack([rng.permutation(max(experts, top_k))[:top_k] % experts for _ in range(tokens)]).astype(np.int32)
    w = rng.random((tokens, top_k)).astype(np.float32)
    wide = torch.full((tokens, hidden + 8), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide[:, :hidden] = torch.from_numpy(x).cuda().bfloat16()
    y = razer.razer_moe_experts(wide[:, :hidden], torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda(), gate, up, down, act=act)
    check_experts(y, *so.experts(x, ids, w, g64, u64, d64, act))


@pytest.mark.parametrize("tokens,hidden,inter,experts,top_k", [(1, 256, 96, 4, 2), (1, 128, 544, 8, 8), (5, 256, 320, 3, 2), (8, 64, 512, 2, 2), (9, 128, 96, 4, 2), (32, 96, 288, 16, 4)])
@pytest.mark.parametrize("block", [16, 128])
def test_two_parts_between_the_products(tokens, hidden, inter, experts, top_k, block):
    """With few tokens what stands between the products is held to a bf16 and a bf16 of its rest: off by the square of one rounding."""
    rng = np.random.default_rng(tokens + inter)
    hidden, inter = (hidden, inter) if block == 16 else (-(-hidden // 128) * 128, -(-inter // 128) * 128)
    (gate, g), (up, u), (down, d) = stack(rng, experts, inter, hidden, block), stack(rng, experts, inter, hidden, block), stack(rng, experts, 64, inter, block)
    x, w = so.bf16(rng.standard_normal((tokens, hidden))), rng.random((tokens, top_k)).astype(np.float32)
    ids = rng.integers(0, experts, (tokens, top_k)).astype(np.int32)
    y = razer.razer_moe_experts(torch.from_numpy(x).cuda().bfloat16(), torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda(), gate, up, down)
    check_experts(y, *so.experts(x, ids, w, g, u, d, between=so.U16 ** 2))


@pytest.mark.parametrize("tokens", [1, 3, 12])
def test_infinite_between_the_products(tokens):
    """An intermediate value that leaves the range gives infinities and NaN as one rounding would, and no others."""
    rng, (gate, _), (up, _), (down, d) = small(11, experts=2, hidden=64, inter=64)
    x = torch.full((tokens, 64), 1e30, device="cuda", dtype=torch.bfloat16)
    ids, w = torch.zeros(tokens, 1, dtype=torch.int32, device="cuda"), torch.ones(tokens, 1, device="cuda")
    y = razer.razer_moe_experts(x, ids, w, gate, up, down)
    a = razer.razer_linear(gate.expert(0), x[:1]).double()
    b = razer.razer_linear(up.expert(0), x[:1]).double()
    a = (torch.where(a > 0, a * b, 0.0)).float().cpu().double().numpy()[0]
    assert np.isinf(a).any()
    with np.errstate(invalid="ignore"):
        want = np.array([np.sum(row[row != 0] * a[row != 0]) + (np.nan if (np.isinf(a) & (row == 0)).any() else 0.0) for row in d[0]])
    got = y.float().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.broadcast_to(np.isnan(want), got.shape)) and np.array_equal(np.isinf(got), np.broadcast_to(np.isinf(want), got.shape))


@pytest.mark.parametrize("block", [64, 128])
def test_experts_in_long_blocks(block):
    rng = np.random.default_rng(block)
    gate, g64 = stack(rng, 3, 384, 256, block)
    down, d64 = stack(rng, 3, 256, 384, block)
    x, ids, w = so.bf16(rng.standard_normal((6, 256))), rng.integers(0, 3, (6, 2)).astype(np.int32), rng.random((6, 2)).astype(np.float32)
    y = razer.razer_moe_experts(torch.from_numpy(x).cuda().bfloat16(), torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda(), gate, None, down)
    check_experts(y, *so.experts(x, ids, w, g64, None, d64))


def small(seed=0, experts=6, hidden=128, inter=96):
    rng = np.random.default_rng(seed)
    return rng, stack(rng, experts, inter, hidden), stack(rng, experts, inter, hidden), stack(rng, experts, hidden, inter)


def test_ids_out_of_range_repeated_and_all_the_same():
    rng, (gate, g), (up, u), (down, d) = small()
    for tokens in (1, 3, 21, 100):
        x = so.bf16(rng.standard_normal((tokens, 128)))
        xd = torch.from_numpy(x).cuda().bfloat16()
        w = rng.standard_normal((tokens, 3)).astype(np.float32)
        for ids in (np.full((tokens, 3), -1), np.full((tokens, 3), 4), rng.integers(-3, 9, (tokens, 3)), np.where(np.arange(tokens)[:, None] % 2, -1, rng.integers(0, 6, (tokens, 3))),
                    np.full((tokens, 3), 2 ** 31 - 1), np.full((tokens, 3), -2 ** 31)):
            ids = ids.astype(np.int32)
            out = torch.full((tokens + 2, 128 + 8), 5.0, device="cuda", dtype=torch.bfloat16)
            razer.razer_moe_experts(xd, torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda(), gate, up, down, out=out[1:-1, :128])
            check_experts(out[1:-1, :128], *so.experts(x, ids, w, g, u, d))
            assert (out[0] == 5).all() and (out[-1] == 5).all() and (out[:, 128:] == 5).all()


def test_other_tokens_do_not_matter():
    """A token's output is the same to the bit whatever stands beside it, as long as the sizes are the same."""
    rng, (gate, _), (up, _), (down, _) = small(3)
    x = torch.from_numpy(rng.standard_normal((30, 128))).cuda().bfloat16()
    ids, w = torch.from_numpy(rng.integers(0, 6, (30, 2)).astype(np.int32)).cuda(), torch.rand(30, 2, device="cuda")
    y = razer.razer_moe_experts(x, ids, w, gate, up, down)
    for _ in range(5):
        assert torch.equal(razer.razer_moe_experts(x, ids, w, gate, up, down), y)
    p = torch.randperm(30, device="cuda")
    assert torch.equal(razer.razer_moe_experts(x[p], ids[p], w[p], gate, up, down), y[p])
    x2, ids2 = x.clone(), ids.clone()
    x2[5:] = float("nan")
    ids2[5:] = 3
    assert torch.equal(razer.razer_moe_experts(x2, ids2, w, gate, up, down)[:5], y[:5])


def test_one_expert_is_the_linear_layers():
    rng, (gate, _), (up, _), (down, _) = small(4, experts=1, hidden=256, inter=512)
    x = torch.from_numpy(rng.standard_normal((3, 256))).cuda().bfloat16()
    one = torch.ones(3, 1, device="cuda")
    y = razer.razer_moe_experts(x, torch.zeros(3, 1, dtype=torch.int32, device="cuda"), one, gate, up, down)
    g, u = (razer.razer_linear(s.expert(0), x).float() for s in (gate, up))
    want = razer.razer_linear(down.expert(0), (torch.nn.functional.silu(g) * u).bfloat16())
    assert float((y.float() - want.float()).abs().max()) <= 0.02 * float(want.float().abs().max())


def test_too_small_a_workspace_is_refused_and_a_larger_one_taken():
    rng, (gate, _), (up, _), (down, _) = small(5)
    x = torch.zeros(4, 128, device="cuda", dtype=torch.bfloat16)
    ids, w = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.ones(4, 2, device="cuda")
    from paper_2501_04052_amd import step
    need = step.razer_moe_workspace_bytes(x, ids, w, gate, up, down)
    with pytest.raises(razer.RazerError):
        razer.razer_moe_experts(x, ids, w, gate, up, down, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert not razer.razer_moe_experts(x, ids, w, gate, up, down, workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda")).any()


def test_a_workspace_elsewhere_or_with_gaps_is_refused():
    rng, (gate, _), (up, _), (down, _) = small(5)
    x, ids, w = torch.zeros(4, 128, device="cuda", dtype=torch.bfloat16), torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    router = torch.zeros(8, 128, device="cuda", dtype=torch.bfloat16)
    for bad in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(1 << 21, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(AssertionError):
            razer.razer_moe_experts(x, ids, w, gate, up, down, workspace=bad)
        with pytest.raises(AssertionError):
            razer.razer_moe_route(x, router, 2, workspace=bad)
        with pytest.raises(AssertionError):
            razer.razer_sample(torch.zeros(2, 64, device="cuda"), torch.zeros(2, device="cuda"), workspace=bad)


def test_two_streams_with_workspaces_of_their_own():
    rng, (gate, _), (up, _), (down, _) = small(6)
    xs = [torch.from_numpy(rng.standard_normal((n, 128))).cuda().bfloat16() for n in (12, 31)]
    ids = [torch.from_numpy(rng.integers(0, 6, (n, 2)).astype(np.int32)).cuda() for n in (12, 31)]
    ws = [torch.rand(n, 2, device="cuda") for n in (12, 31)]
    alone = [razer.razer_moe_experts(x, i, w, gate, up, down) for x, i, w in zip(xs, ids, ws)]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(10):
        both = []
        for s, x, i, w in zip(streams, xs, ids, ws):
            with torch.cuda.stream(s):
                both.append(razer.razer_moe_experts(x, i, w, gate, up, down))
        torch.cuda.synchronize()
        assert torch.equal(both[0], alone[0]) and torch.equal(both[1], alone[1])


def test_more_tokens_than_a_grid_dimension_holds():
    """70000 tokens: the same as in parts."""
    rng, (gate, _), (up, _), (down, _) = small(7, experts=5, hidden=64, inter=32)
    n = 70000
    x = torch.randn(n, 64, device="cuda").bfloat16()
    ids, w = razer.razer_moe_route(x, torch.randn(5, 64, device="cuda").bfloat16(), 2)
    y = razer.razer_moe_experts(x, ids, w, gate, up, down)
    for a, b in ((0, 500), (65400, 66000), (69900, n)):
        part = razer.razer_moe_experts(x[a:b].contiguous(), ids[a:b].contiguous(), w[a:b].contiguous(), gate, up, down)
        assert float((part.float() - y[a:b].float()).abs().max()) <= 2 * so.U16 * float(y.float().abs().max())
    assert int(ids.min()) >= 0 and int(ids.max()) < 5 and torch.allclose(w.sum(1), torch.ones(n, device="cuda"), atol=4e-7)


def test_no_tokens():
    rng, (gate, _), (up, _), (down, _) = small(8)
    x = torch.empty(0, 128, device="cuda", dtype=torch.bfloat16)
    ids, w = razer.razer_moe_route(x, torch.zeros(6, 128, device="cuda", dtype=torch.bfloat16), 2)
    assert ids.shape == (0, 2) and razer.razer_moe_experts(x, ids, w, gate, up, down).shape == (0, 128)
