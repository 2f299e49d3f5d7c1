"""razer_moe_experts in forms and at sizes that test_gpu_moe.py does not reach, against the same definition."""
import numpy as np
import pytest
import torch

import paper_2501_04052_amd as razer
import step_oracle as so
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
