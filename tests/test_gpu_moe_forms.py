"""razer_moe_experts in forms and at sizes that test_gpu_moe.py does not reach, against the same definition."""
import numpy as np
import pytest
import torch

import paper_2501_04052_amd as razer
import step_oracle as so
from gpu_util import launched_kernels
from test_gpu_moe import check_experts, stack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("tokens", [1, 5, 60])
def test_relu_keeps_a_nan(tokens, gated):
    """max(z, 0) of a NaN is a NaN: a token with one in it does not come out as if it were 0, and no other token changes."""
    rng = np.random.default_rng(tokens)
    (gate, g), (up, u), (down, d) = (stack(rng, 2, n, k) for n, k in ((64, 96), (64, 96), (96, 64)))
    x = torch.from_numpy(so.bf16(rng.standard_normal((tokens, 96)))).cuda().bfloat16()
    ids, w = torch.from_numpy(rng.integers(0, 2, (tokens, 1)).astype(np.int32)).cuda(), torch.ones(tokens, 1, device="cuda")
    call = lambda: razer.razer_moe_experts(x, ids, w, gate, up if gated else None, down, act="relu")
    clean = call()
    x[tokens - 1, 3] = float("nan")
    y = call()
    assert y[tokens - 1].isnan().all() and torch.equal(y[:tokens - 1], clean[:tokens - 1])


def test_an_intermediate_longer_than_32_bits_of_bytes():
    """1100 choices of 2^20 intermediate values in two parts: 4.6 GB, whose rows from the 1024th choice on begin beyond 2^32.
    The down products read 64 of the values, the rest of their codes is 0 and adds nothing, not even a rounding."""
    experts, inter, hidden, tokens, top_k = 128, 1 << 20, 32, 275, 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    byte = lambda *s: torch.randint(0, 256, s, generator=gen, device="cuda", dtype=torch.uint8)
    ts = torch.full((experts,), 2.0 ** -9, device="cuda")
    gate = razer.RazerExperts(byte(experts, inter, hidden // 2), byte(experts, inter, hidden // 16), ts)
    codes = torch.zeros(experts, hidden, inter // 2, dtype=torch.uint8, device="cuda")
    pairs = torch.tensor([0, 1, 31, 32, 64 * 100 + 5, inter // 4, inter // 2 - 64, inter // 2 - 1] + list(range(12345, 12345 + 24 * 4099, 4099)), device="cuda")
    codes[:, :, pairs] = byte(experts, hidden, len(pairs))
    down = razer.RazerExperts(codes, byte(experts, hidden, inter // 16), ts)
    at = torch.stack([2 * pairs, 2 * pairs + 1], 1).flatten()
    rng = np.random.default_rng(1)
    x, w = so.bf16(rng.standard_normal((tokens, hidden))), rng.random((tokens, top_k)).astype(np.float32)
    ids = rng.integers(0, experts, (tokens, top_k)).astype(np.int32)
    y = razer.razer_moe_experts(torch.from_numpy(x).cuda().bfloat16(), torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda(), gate, None, down)
    look = [0, 1, 200, 255, 256, 257, 273, 274]
    values = lambda s, pick: {e: pick(razer.razer_dequant(s.expert(e))).double().cpu().numpy() for e in sorted(set(ids[look].flatten().tolist()))}
    g, d = values(gate, lambda t: t[at]), values(down, lambda t: t[:, at])
    every = lambda m: [m.get(e, next(iter(m.values()))) for e in range(experts)]
    check_experts(y[look], *so.experts(x[look], ids[look], w[look], every(g), None, every(d), between=so.U16 ** 2))


@pytest.mark.parametrize("tokens,hidden,inter,experts,top_k", [(9, 64, 512, 1, 1), (30, 128, 544, 3, 2), (64, 96, 288, 2, 2), (64, 160, 1408, 4, 4), (200, 64, 96, 3, 1), (256, 128, 2080, 2, 2)])
@pytest.mark.parametrize("gated", [True, False])
def test_two_parts_between_the_products_with_many_tokens(tokens, hidden, inter, experts, top_k, gated):
    """However many tokens an expert has, what stands between the products is held to a bf16 and a bf16 of its rest."""
    rng = np.random.default_rng(tokens + inter)
    (gate, g), (up, u), (down, d) = stack(rng, experts, inter, hidden), stack(rng, experts, inter, hidden), stack(rng, experts, 64, inter)
    x, w = so.bf16(rng.standard_normal((tokens, hidden))), rng.random((tokens, top_k)).astype(np.float32)
    ids = rng.integers(0, experts, (tokens, top_k)).astype(np.int32)
    y = razer.razer_moe_experts(torch.from_numpy(x).cuda().bfloat16(), torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda(), gate, up if gated else None, down)
    check_experts(y, *so.experts(x, ids, w, g, u if gated else None, d, between=so.U16 ** 2))


@pytest.mark.parametrize("tokens,inter,rows", [(64, 352, 16), (60, 1440, 16), (128, 352, 32), (125, 2080, 32)])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("gated", [True, False])
def test_a_batch_that_four_groups_of_rows_serve(tokens, inter, rows, block, gated):
    """Enough workgroups for four groups of weight rows in each, over tiles of 16 and 32 rows, short and long sums."""
    rng = np.random.default_rng(tokens + inter + block)
    experts, top_k, hidden = 64, 8, 352
    (gate, g), (up, u), (down, d) = stack(rng, experts, inter, hidden, block), stack(rng, experts, inter, hidden, block), stack(rng, experts, hidden, inter, block)
    x, w = so.bf16(rng.standard_normal((tokens, hidden))), rng.random((tokens, top_k)).astype(np.float32)
    ids = np.stack([rng.permutation(experts)[:top_k] for _ in range(tokens)]).astype(np.int32)
    ids[rng.random(ids.shape) < 0.03] = -1
    xd, idd, wd = torch.from_numpy(x).cuda().bfloat16(), torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda()
    call = lambda: razer.razer_moe_experts(xd, idd, wd, gate, up if gated else None, down)
    y = call()
    for mode in (0 if gated else 1, 2):
        name = "expert_kernel<%d, 4, %s, %d>" % (rows // 4, "true" if block > 16 else "false", mode)
        assert any(name in n for n in launched_kernels(call)), name
    look = rng.permutation(tokens)[:16]
    check_experts(y[torch.from_numpy(look).cuda()], *so.experts(x[look], ids[look], w[look], g, u if gated else None, d, between=so.U16 ** 2))


@pytest.mark.parametrize("out", [2048, 2080, 4160])
@pytest.mark.parametrize("block", [16, 64])
@pytest.mark.parametrize("gated", [True, False])
def test_one_token_with_more_outputs_than_one_round_of_workgroups(out, block, gated):
    """Up to 2048 outputs a workgroup has up to 16 waves, beyond that up to 8."""
    rng = np.random.default_rng(out + block)
    (gate, g), (up, u), (down, d) = stack(rng, 5, 576, 320, block), stack(rng, 5, 576, 320, block), stack(rng, 5, out, 576, block)
    x, w = so.bf16(rng.standard_normal((1, 320))), rng.random((1, 7)).astype(np.float32)
    for ids in ([[4, 0, 3, 1, 2, 4, 0]], [[-1, 2, 5, 2, 99, 0, 1]]):
        ids = np.array(ids, np.int32)
        y = razer.razer_moe_experts(torch.from_numpy(x).cuda().bfloat16(), torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda(), gate, up if gated else None, down)
        check_experts(y, *so.experts(x, ids, w, g, u if gated else None, d, between=so.U16 ** 2))


@pytest.mark.parametrize("tokens", [1, 3, 40])
def test_special_values_of_nine_and_a_half(tokens):
    """9.5 times a block scale needs up to 9 bits (19 x 15): the operand is that product rounded to bf16, every other special
    value and element is exact."""
    rng = np.random.default_rng(tokens)
    for sv in ((9.5, 5.0), (8.5, 9.5), (7.5, 9.0)):
        byte = lambda *s: torch.from_numpy(rng.integers(0, 256, s).astype(np.uint8)).cuda()
        ts = torch.full((2,), 2.0 ** -9, device="cuda")
        new = lambda rows, cols: razer.RazerExperts(byte(2, rows, cols // 2), byte(2, rows, cols // 16), ts, sv)
        gate, up, down = new(96, 64), new(96, 64), new(64, 96)
        exact = [[razer.razer_dequant(s.expert(e)).cpu().numpy() for e in range(2)] for s in (gate, up, down)]
        rounded = [[so.bf16(m) for m in s] for s in exact]                 # (the tensor scale is a power of two)
        assert any((a != b).any() for s, r in zip(exact, rounded) for a, b in zip(s, r)) == (9.5 in sv)
        assert all((np.abs(a - b) <= np.abs(a) / 285).all() for s, r in zip(exact, rounded) for a, b in zip(s, r))
        x, w = so.bf16(rng.standard_normal((tokens, 64))), rng.random((tokens, 2)).astype(np.float32)
        ids = rng.integers(0, 2, (tokens, 2)).astype(np.int32)
        y = razer.razer_moe_experts(torch.from_numpy(x).cuda().bfloat16(), torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda(), gate, up, down)
        check_experts(y, *so.experts(x, ids, w, *[[m.astype(np.float64) for m in s] for s in rounded], between=so.U16 ** 2))
