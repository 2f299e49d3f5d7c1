"""A decoder whose feed-forward half is a mixture of experts, as a serving loop runs it on quantized weights, an 8-bit cache
and random numbers of its own:

    embedding -> per layer: razer_norm -> CachedAttention -> razer_norm (residual) -> razer_moe_route -> razer_moe_experts
              -> razer_norm (residual), or razer_norm_quantize in front of a head with 4-bit activations -> head (razer_linear)
              -> razer_sample

`MoeLayer` holds one layer's weights, `MoeDecoder` the layers, the page pool and one step of all requests.

    python -m paper_2501_04052_amd.moe_decoder     # prompts, then decoding, checked against the same model without a cache
"""
import torch

from . import binding as _b
from .cached_attention import CachedAttention, PagePool, uncached
from .step import RazerExperts, razer_moe_experts, razer_moe_route, razer_norm, razer_norm_quantize, razer_sample


class MoeLayer:
    """One layer: attention (a CachedAttention), the weights of its two norms, the router and the experts' three stacks."""

    def __init__(self, attention, norm_in, norm_mid, router, gate, up, down, top_k):
        self.attention, self.norm_in, self.norm_mid = attention, norm_in, norm_mid
        self.router, self.gate, self.up, self.down, self.top_k = router, gate, up, down, top_k

    def experts(self, y):
        ids, weights = razer_moe_route(y, self.router, self.top_k)
        return razer_moe_experts(y, ids, weights, self.gate, self.up, self.down)

    def __call__(self, x, h, plan, table, **options):
        """x: what the last layer adds to the residual h.  Returns the same two for the next one."""
        y, h = razer_norm(x, self.norm_in, residual=h, sum_out=h)
        y, h = razer_norm(self.attention(y, plan, table, **options), self.norm_mid, residual=h, sum_out=h)
        return self.experts(y), h


class MoeDecoder:
    """embedding [vocab][hidden] (bfloat16), layers, the last norm's weight and the head (a RazerTensor [vocab][hidden]).
    head_scale: a calibrated tensor scale; the head then takes 4-bit activations."""

    def __init__(self, embedding, layers, norm_out, head, head_scale=None):
        self.embedding, self.layers, self.norm_out, self.head, self.head_scale = embedding, layers, norm_out, head, head_scale

    def logits(self, x, h):
        if self.head_scale is None:
            y, _ = razer_norm(x, self.norm_out, residual=h)
        else:
            y, _ = razer_norm_quantize(x, self.norm_out, self.head_scale, residual=h)
        return _b.razer_linear(self.head, y)

    def step(self, pool, tokens):
        """tokens: a list of each request's new tokens (int64 tensors), one at least of each.  The logits behind each request's last one."""
        fresh = [t.numel() for t in tokens]
        if not all(fresh):
            raise ValueError("a request without new tokens has no logits in this step")
        plan, known = pool.step(fresh)
        h = self.embedding[torch.cat(tokens)].float()                # the residual, in 32 bits
        x = torch.zeros(h.shape, dtype=torch.bfloat16, device=h.device)
        for layer in self.layers:
            x, h = layer(x, h, plan, pool.table, **known)
        last = (plan.cu[1:] - 1).long()
        return self.logits(x[last], h[last])

    def without_cache(self, tokens):
        """The logits behind every token of one request, attention and experts computed without cache and kernels for few
        tokens: every expert in 32 bits on all tokens."""
        h = self.embedding[tokens].float()
        rms = lambda v, w: (v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6) * w.float()).bfloat16()
        for layer in self.layers:
            h = h + uncached(layer.attention, rms(h, layer.norm_in)).float()
            y = rms(h, layer.norm_mid)
            p = torch.softmax(y.float() @ layer.router.float().t(), -1)
            w, ids = torch.topk(p, layer.top_k)
            share = torch.zeros_like(p).scatter_(1, ids, w / w.sum(-1, keepdim=True))
            for e in range(layer.gate.experts):
                g, u, d = (_b.razer_dequant(s.expert(e)) for s in (layer.gate, layer.up, layer.down))
                h = h + share[:, e:e + 1] * ((torch.nn.functional.silu(y.float() @ g.t()) * (y.float() @ u.t())) @ d.t())
        return rms(h, self.norm_out).float() @ _b.razer_dequant(self.head).t()


def random_decoder(hidden=512, heads=(4, 2), head_dim=128, inter=256, experts=8, top_k=2, layers=2, vocab=1000, pages=64, page=32, seed=0, head_scale=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
    w = lambda rows, cols: _b.razer_quantize(normal(rows, cols) * cols ** -0.5, _b.WEIGHT, (5.0, 8.0))
    stack = lambda rows, cols: RazerExperts.stack([w(rows, cols) for _ in range(experts)])
    norm = lambda: (1.0 + 0.1 * normal(hidden)).bfloat16()
    q, kv = heads[0] * head_dim, heads[1] * head_dim
    built = [MoeLayer(CachedAttention(w(q, hidden), w(kv, hidden), w(kv, hidden), w(hidden, q), head_dim, pages, page), norm(), norm(),
                      (normal(experts, hidden) * hidden ** -0.5).bfloat16(), stack(inter, hidden), stack(inter, hidden), stack(hidden, inter), top_k) for _ in range(layers)]
    scale = None if head_scale is None else torch.full((1,), head_scale, device="cuda")
    return MoeDecoder(normal(vocab, hidden).bfloat16(), built, norm(), w(vocab, hidden), scale)


def run(prompts=(37, 200, 64), steps=12, page=32, temperature=0.8, top_k=50, top_p=0.95, seed=0, **shape):
    """Prompts in one step, then `steps` sampled tokens of every request.  Relative error of all logits against
    without_cache() on the tokens that came out, and those tokens."""
    pages = sum(-(-(p + steps) // page) for p in prompts)
    model = random_decoder(pages=pages, page=page, seed=seed, **shape)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    n, vocab = len(prompts), model.head.rows
    pool = PagePool(pages, n, max(prompts) + steps, page)
    fresh = [torch.randint(vocab, (p,), generator=gen, device="cuda") for p in prompts]
    texts, got = [t for t in fresh], [[] for _ in prompts]
    f32 = lambda v: torch.full((n,), v, device="cuda")
    settings = dict(temperature=f32(temperature), top_k=torch.full((n,), top_k, dtype=torch.int32, device="cuda"), top_p=f32(top_p))
    for _ in range(steps):
        logits = model.step(pool, fresh)
        tokens, _ = razer_sample(logits, torch.rand(n, generator=gen, device="cuda"), **settings)
        fresh = list(tokens.long().split(1))
        for r in range(n):
            got[r].append(logits[r])
            texts[r] = torch.cat([texts[r], fresh[r]])
    got = torch.cat([torch.stack(g) for g in got]).float()
    want = torch.cat([model.without_cache(t[:-1])[p - 1:] for t, p in zip(texts, prompts)])
    return float((got - want).norm() / want.norm()), [t.tolist() for t in texts]


def main():
    error, texts = run()
    print("logits of %d requests against the model without a cache: relative error %.4f (8-bit keys and values)" % (len(texts), error))


if __name__ == "__main__":
    main()
