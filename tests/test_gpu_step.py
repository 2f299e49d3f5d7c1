"""The operators of a step together: a decoder with experts against the same model without a cache, and a captured step that
is replayed on new inputs."""
import torch
import pytest

import paper_2501_04052_amd as razer
from paper_2501_04052_amd import moe_decoder

pytestmark = pytest.mark.gpu


def test_decoder_command_runs_and_repeats():
    error, texts = moe_decoder.run(prompts=(5, 70, 33), steps=6)
    assert 0 < error < 1 and [len(t) for t in texts] == [11, 76, 39]
    assert moe_decoder.run(prompts=(5, 70, 33), steps=6) == (error, texts)


def plain_step(model, pool, tokens):
    """MoeDecoder.step with norm, routing and experts in 64 bits, rounded to bf16 where the operators' outputs are."""
    plan, known = pool.step([t.numel() for t in tokens])
    h = model.embedding[torch.cat(tokens)].float()
    rms = lambda v, w: (v.double() / torch.sqrt(v.double().square().mean(-1, keepdim=True) + 1e-6) * w.double())
    for layer in model.layers:
        h = h + layer.attention(rms(h, layer.norm_in).bfloat16(), plan, pool.table, **known).float()
        y = rms(h, layer.norm_mid).bfloat16().double()
        p = torch.softmax(y @ layer.router.double().t(), -1)
        w, ids = torch.topk(p, layer.top_k)
        share = torch.zeros_like(p).scatter_(1, ids, w / w.sum(-1, keepdim=True))
        z = torch.zeros_like(y)
        for e in range(layer.gate.experts):
            g, u, d = (razer.razer_dequant(s.expert(e)).double() for s in (layer.gate, layer.up, layer.down))
            z += share[:, e:e + 1] * ((torch.nn.functional.silu(y @ g.t()) * (y @ u.t())) @ d.t())
        h = h + z.bfloat16().float()
    last = (plan.cu[1:] - 1).long()
    return rms(h[last], model.norm_out)


@pytest.mark.parametrize("head_scale", [None, 5.0 / 2688])
def test_decoder_against_plain_operators(head_scale):
    """Every expert is chosen, so that nothing jumps.  What the plain steps do not have, relative to a layer's sum: the bf16
    rounding between the experts' products (2^-8), and a bf16 result of norm, attention or experts that falls to the other
    side (2^-7 each, where it does): 2 (2^-8 + 3 2^-7) < 2^-4 over two layers if all of that fell together."""
    shape = dict(pages=12, page=32, seed=3, experts=3, top_k=3, head_scale=head_scale)
    model, plain = moe_decoder.random_decoder(**shape), moe_decoder.random_decoder(**shape)
    pools = [moe_decoder.PagePool(12, 3, 90, 32) for _ in range(2)]
    gen = torch.Generator(device="cuda").manual_seed(5)
    for fresh in ((5, 70, 33), (1, 1, 1), (2, 1, 4), (1, 1, 1)):
        tokens = [torch.randint(1000, (n,), generator=gen, device="cuda") for n in fresh]
        got, y = model.step(pools[0], tokens), plain_step(plain, pools[1], tokens)
        if head_scale is not None:                     # (the codes of almost the same numbers: as the library encodes them)
            y = razer.razer_dequant(razer.razer_quantize(y.float(), razer.ACT, (5.0,), tensor_scale=plain.head_scale)).double()
        want = y @ razer.razer_dequant(plain.head).double().t()
        error = float((got.double() - want).norm() / want.norm())
        # 4-bit codes: an element near a border of two goes to the other one, by up to a third of itself, for 2^-4 in a step of 2^-2 .. 2^-1
        assert error < (2.0 ** -4 if head_scale is None else 2.0 ** -3), (fresh, error)


def make_step(tokens, hidden=256, inter=160, experts=12, vocab=9000, rows=4):
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
    w = lambda n, k: razer.razer_quantize(normal(n, k) * k ** -0.5, razer.WEIGHT, (5.0, 8.0))
    stack = lambda n, k: razer.RazerExperts.stack([w(n, k) for _ in range(experts)])
    gate, up, down, head = stack(inter, hidden), stack(inter, hidden), stack(hidden, inter), w(vocab, hidden)
    router, norm = normal(experts, hidden).bfloat16(), torch.ones(hidden, device="cuda")
    x, h, u = normal(tokens, hidden).bfloat16(), normal(tokens, hidden), torch.rand(tokens, generator=gen, device="cuda")
    scale = torch.full((1,), 5.0 / 2688, device="cuda")
    t = torch.full((tokens,), 0.7, device="cuda")
    p = torch.full((tokens,), 0.9, device="cuda")

    def step():
        y, total = razer.razer_norm(x, norm, residual=h)
        ids, weights = razer.razer_moe_route(y, router, 3)
        z = razer.razer_moe_experts(y, ids, weights, gate, up, down)
        q, total = razer.razer_norm_quantize(z, norm, scale, residual=total)
        y2, _ = razer.razer_norm(z, norm, residual=total)
        logits = razer.razer_linear(head, y2)
        tok, lp = razer.razer_sample(logits, u, temperature=t, top_p=p)
        return ids, weights, z, q.codes, q.scales, total, logits, tok, lp
    return step, (x, h, u)


@pytest.mark.parametrize("tokens", [1, 3, 40])
def test_captured_step_replayed_on_new_inputs(tokens):
    step, inputs = make_step(tokens)
    want_first = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for k in range(5):
        if k:
            for t in inputs:
                t.copy_(torch.rand_like(t) if t.dim() == 1 else torch.randn_like(t))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(out, want):
            assert torch.equal(g, w)
        if k == 0:
            for a, b in zip(want, want_first):
                assert torch.equal(a, b)


@pytest.mark.parametrize("rows,vocab", [(2, 50000), (3, 131072), (5, 260000)])
def test_captured_sampling_of_rows_in_pieces(rows, vocab):
    """Two graphs that share no workspace, replayed in turn and beside eager calls."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    l = [torch.randn(rows, vocab, generator=gen, device="cuda") * 2 for _ in range(2)]
    u = torch.rand(rows, generator=gen, device="cuda")
    razer.razer_sample(l[0], u)
    graphs, outs = [], []
    for x in l:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(razer.razer_sample(x, u))
        graphs.append(g)
    for _ in range(4):
        for x in l:
            x.copy_(torch.randn(rows, vocab, generator=gen, device="cuda") * 2)
        u.copy_(torch.rand(rows, generator=gen, device="cuda"))
        want = [razer.razer_sample(x, u) for x in l]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
