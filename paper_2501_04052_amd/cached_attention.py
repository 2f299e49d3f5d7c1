"""The attention half of a decoder layer on quantized weights and an 8-bit cache, as a step of a serving loop runs it:

    {q,k,v} projections (razer_linear_grouped) -> rotary positions -> razer_cache_append -> razer_cache_attention
    -> o projection (razer_linear)

with the step's bookkeeping (razer_cache_plan) once for all layers.  `PagePool` owns the page list and the block tables,
`CachedAttention` one layer's weights and cache.

    python -m paper_2501_04052_amd.cached_attention     # prompts, then decoding, checked against uncached attention
"""
import torch

from . import binding as _b
from .cache import KVCache, razer_cache_append, razer_cache_attention, razer_cache_plan


class PagePool:
    """Block tables of up to `requests` requests over `pages` pages; the lengths live on the GPU and on the host.  Pages are only
    taken: giving back those of finished requests and of drafts that were not kept is left to a server's own pool."""

    def __init__(self, pages, requests, max_len, page=64, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.page, self.max_len = page, max_len
        self.table = torch.full((requests, -(-max_len // page)), -1, **i32)
        self.free = torch.arange(pages, **i32)
        self.lens = torch.zeros(requests, **i32)
        self.host_lens = [0] * requests
        self.taken = 0

    def step(self, fresh):
        """Plans a step with fresh[r] new tokens of request r (a list): (plan, what razer_cache_attention is told)."""
        new = torch.tensor(fresh, dtype=torch.int32, device=self.table.device)
        want = sum(-(-(n + f) // self.page) - -(-n // self.page) for n, f in zip(self.host_lens, fresh))
        if self.taken + want > self.free.numel() or max(n + f for n, f in zip(self.host_lens, fresh)) > self.max_len:
            raise RuntimeError("the pool has no room for this step")
        plan = razer_cache_plan(self.lens, new, self.table, self.free[self.taken:], self.page, sum(fresh))
        self.lens = plan.total
        self.host_lens = [n + f for n, f in zip(self.host_lens, fresh)]
        self.taken += want
        return plan, dict(max_new=max(fresh), max_len=max(self.host_lens))


def rotary(x, positions, base=10000.0):
    """Rotary positions on x [tokens][heads][dim] (halves paired), in fp32."""
    half = x.shape[-1] // 2
    f = base ** (-torch.arange(half, device=x.device, dtype=torch.float32) / half)
    a = positions.to(torch.float32)[:, None, None] * f
    c, s = a.cos(), a.sin()
    lo, hi = x[..., :half].float(), x[..., half:].float()
    return torch.cat([lo * c - hi * s, hi * c + lo * s], dim=-1).to(x.dtype)


class CachedAttention:
    """One layer: q, k, v and o projections in a RaZeR weight format and the layer's key/value cache."""

    def __init__(self, wq, wk, wv, wo, head_dim, pages, page=64):
        self.wq, self.wk, self.wv, self.wo, self.dim = wq, wk, wv, wo, head_dim
        self.q_heads, self.kv_heads = wq.rows // head_dim, wk.rows // head_dim
        self.cache = KVCache.allocate(pages, self.kv_heads, head_dim, page, device=wq.codes.device)

    def __call__(self, x, plan, table, **options):
        """x [tokens][hidden] (bfloat16) of the plan's tokens; options: as razer_cache_attention takes them."""
        n = x.shape[0]
        q, k, v = _b.razer_linear_grouped([self.wq, self.wk, self.wv], x)
        q = rotary(q.view(n, self.q_heads, self.dim), plan.positions)
        k = rotary(k.view(n, self.kv_heads, self.dim), plan.positions)
        razer_cache_append(self.cache, k, v.view(n, self.kv_heads, self.dim), plan.slots)
        y = razer_cache_attention(self.cache, q, plan.cu, plan.total, table, **options)
        return _b.razer_linear(self.wo, y.view(n, -1))


def uncached(layer, x):
    """The same layer over one request's tokens x without a cache: keys and values as projected, softmax in fp32."""
    n, pos = x.shape[0], torch.arange(x.shape[0], device=x.device)
    q, k, v = _b.razer_linear_grouped([layer.wq, layer.wk, layer.wv], x)
    q = rotary(q.view(n, layer.q_heads, layer.dim), pos).float().transpose(0, 1)
    k = rotary(k.view(n, layer.kv_heads, layer.dim), pos).float().transpose(0, 1).repeat_interleave(layer.q_heads // layer.kv_heads, 0)
    v = v.view(n, layer.kv_heads, layer.dim).float().transpose(0, 1).repeat_interleave(layer.q_heads // layer.kv_heads, 0)
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * layer.dim ** -0.5
    s = s.masked_fill(pos[None, :] > pos[:, None], float("-inf"))
    y = torch.matmul(torch.softmax(s, -1), v).transpose(0, 1).reshape(n, -1)
    return _b.razer_linear(layer.wo, y.to(torch.bfloat16).contiguous())


def run(hidden=1024, q_heads=8, kv_heads=2, head_dim=128, prompts=(37, 200, 64), steps=20, page=32, seed=0):
    """Prompts in one step, then `steps` tokens of every request: relative error of all outputs against uncached()."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    w = lambda rows, cols: _b.razer_quantize(torch.randn(rows, cols, generator=gen, device="cuda") * cols ** -0.5, _b.WEIGHT, (5.0, 8.0))
    total = [p + steps for p in prompts]
    pages = sum(-(-t // page) for t in total)
    layer = CachedAttention(w(q_heads * head_dim, hidden), w(kv_heads * head_dim, hidden), w(kv_heads * head_dim, hidden), w(hidden, q_heads * head_dim),
                            head_dim, pages, page)
    pool = PagePool(pages, len(prompts), max(total), page)
    x = [torch.randn(t, hidden, generator=gen, device="cuda").bfloat16() for t in total]
    out = [[] for _ in prompts]
    at = [0] * len(prompts)
    for fresh in [list(prompts)] + [[1] * len(prompts)] * steps:
        plan, known = pool.step(fresh)
        y = layer(torch.cat([x[r][at[r]:at[r] + n] for r, n in enumerate(fresh)]), plan, pool.table, **known)
        for r, part in enumerate(y.split(fresh)):
            out[r].append(part)
            at[r] += fresh[r]
    got, want = torch.cat([torch.cat(o) for o in out]).float(), torch.cat([uncached(layer, t) for t in x]).float()
    return float((got - want).norm() / want.norm())


def main():
    print("cached against uncached attention: relative error %.4f (8-bit keys and values)" % run())


if __name__ == "__main__":
    main()
