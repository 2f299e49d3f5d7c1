"""The operators of the 8-bit paged key/value cache, as cases that a measuring program can prepare, run and check.

A case is one of three kinds of call:

  plan       one serving step's bookkeeping: block tables, slots, positions and offsets from the requests' lengths
  append     the step's new keys and values, quantised into the pages that the slots name
  attention  the step's queries over the cached keys and values of their own request

The cache holds E4M3 codes in pages of `page` tokens with one power-of-two scale (an exponent byte, bias 127) for each
page and head, keys as [pages][heads][page][dim], values as [pages][heads][dim][page].  Keys have a few channels that
are 8 times as large as the others, values a small mean per channel; a page's unused places hold whatever was there
before, NaN codes among it.  Everything is drawn on the GPU from the seed; lengths come from the case's "pick".
"""
import math
import random

import numpy as np
import torch

own = False

B_MIN, B_MAX = 77, 177                 # range of the exponent byte


def listed():
    return [
        # a decode step of one short chat: latency of the bookkeeping
        dict(name="plan_single", op="plan", requests=1, tokens=1, len_hi=1000, new_hi=1, page=16, pick=1),
        # a step of a loaded server: decoding requests and a few prompts in pages of 16, padded to a fixed token count
        dict(name="plan_loaded", op="plan", requests=257, tokens=16384, len_hi=32000, new_hi=2048, page=16, pick=2),
        # new tokens of a decode batch of 64, grouped heads of a 70B-class layer
        dict(name="append_decode", op="append", requests=64, kv_heads=8, dim=128, page=64, len_hi=2000, new_lo=1, new_hi=1, f32=False, pick=3),
        # prompts of a 7B-class layer, ragged, in pages of 16, keys and values straight from a 32-bit rotary step
        dict(name="append_prompts", op="append", requests=5, kv_heads=32, dim=128, page=16, len_hi=700, new_lo=37, new_hi=2048, f32=True, pick=4),
        # one chat, one token: a 7B-class layer's attention at batch 1
        dict(name="decode_single", op="attention", requests=1, q_heads=32, kv_heads=32, dim=128, page=16, len_lo=1000, len_hi=1000, new_lo=1, new_hi=1, cap=0.0, window=0, bias=False, prefix=0, pick=5),
        # a decode batch of 64 ragged requests, a 70B-class layer with 8 query heads on each key/value head
        dict(name="decode_batch", op="attention", requests=64, q_heads=64, kv_heads=8, dim=128, page=64, len_lo=200, len_hi=8192, new_lo=1, new_hi=1, cap=0.0, window=0, bias=False, prefix=0, pick=6),
        # long documents, few requests: the keys have to be spread over the whole card
        dict(name="decode_long", op="attention", requests=3, q_heads=64, kv_heads=8, dim=128, page=128, len_lo=40000, len_hi=131001, new_lo=1, new_hi=1, cap=0.0, window=0, bias=False, prefix=0, pick=7),
        # a few drafted tokens per request to verify, capped scores, sliding window behind a few tokens that stay visible, wide heads
        dict(name="draft_capped", op="attention", requests=13, q_heads=16, kv_heads=4, dim=256, page=32, len_lo=33, len_hi=5000, new_lo=2, new_hi=5, cap=50.0, window=1024, bias=False, prefix=4, pick=8),
        # a whole prompt of a 7B-class layer
        dict(name="prompt", op="attention", requests=1, q_heads=32, kv_heads=32, dim=128, page=64, len_lo=2048, len_hi=2048, new_lo=2048, new_hi=2048, cap=0.0, window=0, bias=False, prefix=0, pick=9),
        # the next part of a long prompt, a 70B-class layer
        dict(name="prompt_part", op="attention", requests=1, q_heads=64, kv_heads=8, dim=128, page=128, len_lo=16384, len_hi=16384, new_lo=2048, new_hi=2048, cap=0.0, window=0, bias=False, prefix=0, pick=10),
        # short prompts beside decoding requests, small heads in odd groups, a bias by distance and prefixes seen from both sides
        dict(name="mixed_biased", op="attention", requests=9, q_heads=21, kv_heads=3, dim=64, page=16, len_lo=65, len_hi=2500, new_lo=1, new_hi=333, cap=0.0, window=0, bias=True, prefix=200, pick=11),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "attention", "attention", "attention"])
    page, pick = rng.choice([16, 32, 64, 128]), rng.randrange(1 << 20)
    if op == "plan":
        requests = _log_int(rng, 1, 257)
        new_hi = rng.choice([1, _log_int(rng, 1, 2048)])
        return dict(op=op, requests=requests, tokens=min(16384, requests * new_hi + rng.choice([0, rng.randrange(64)])), len_hi=_log_int(rng, 1, 32000), new_hi=new_hi, page=page, pick=pick)
    dim = rng.choice([64, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 16])
    if op == "append":
        new_hi = rng.choice([1, _log_int(rng, 1, 1024)])
        requests = _log_int(rng, 1, max(1, min(64, 2048 // new_hi)))
        return dict(op=op, requests=requests, kv_heads=kv_heads, dim=dim, page=page, len_hi=_log_int(rng, 1, 4096), new_lo=1, new_hi=new_hi, f32=rng.random() < 0.3, pick=pick)
    group = rng.choice([1, 2, 4, 5, 7, 8])
    new_hi = rng.choice([1, 1, rng.randint(1, 8), _log_int(rng, 8, 1024)])
    len_hi = _log_int(rng, max(16, new_hi), 16384)
    # the plain form pads to the longest: what it holds stays under that of the largest listed case
    most = min(64, (1 << 31) // (kv_heads * group * new_hi * len_hi), (1 << 30) // (kv_heads * dim * len_hi))
    requests = _log_int(rng, 1, max(1, most))
    return dict(op=op, requests=requests, q_heads=kv_heads * group, kv_heads=kv_heads, dim=dim, page=page, len_lo=rng.randint(1, len_hi), len_hi=len_hi, new_lo=1, new_hi=new_hi,
                cap=rng.choice([0.0, 0.0, 30.0]), window=rng.choice([0, 0, rng.randint(1, len_hi)]), bias=rng.random() < 0.3, prefix=rng.choice([0, 0, rng.randint(1, len_hi)]), pick=pick)


# ---- lengths -------------------------------------------------------------------------------------------------

def lengths(case):
    """(cached, new) tokens of each request: the first request has the largest of both."""
    r = random.Random(case["pick"])
    n = case["requests"]
    new = [case["new_hi"]] + [_log_int(r, case["new_lo"], case["new_hi"]) for _ in range(n - 1)]
    if case["op"] == "append":
        return [r.randint(0, case["len_hi"]) for _ in range(n)], new
    total = [case["len_hi"]] + [_log_int(r, case["len_lo"], case["len_hi"]) for _ in range(n - 1)]
    return [max(t - m, 0) for t, m in zip(total, new)], new


def _pages(tokens, page):
    return -(-tokens // page)


# ---- inputs --------------------------------------------------------------------------------------------------

def _normal(shape, gen, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _keys(shape, gen):
    """Keys [..., dim] with every 32nd channel 8 times as large."""
    k = _normal(shape, gen)
    k[..., 5::32] *= 8.0
    return k


def _values(shape, gen):
    return _normal(shape, gen) + 0.3 * _normal((shape[-1],), gen)


def _exponent(amax):
    """The smallest exponent byte b with amax <= 448 * 2^(b-127), in its range."""
    bits = amax.contiguous().view(torch.int32)
    return ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000)).clamp(B_MIN, B_MAX)


def _power(b):
    """2^(b-127) for 1 <= b <= 254."""
    return (b.to(torch.int32) << 23).view(torch.float32)


def _to_e4m3(x):
    return x.to(torch.float8_e4m3fn)


def _cache(case, pages, gen):
    """A cache whose pages are full of earlier tokens (as if appended at once)."""
    heads, dim, page = case["kv_heads"], case["dim"], case["page"]
    kc = torch.empty((pages, heads, page, dim), dtype=torch.uint8, device="cuda")
    vc = torch.empty((pages, heads, dim, page), dtype=torch.uint8, device="cuda")
    ks = torch.empty((pages, heads), dtype=torch.uint8, device="cuda")
    vs = torch.empty((pages, heads), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (heads * page * dim))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        for x, codes, scales in ((_keys((n, heads, page, dim), gen), kc, ks),
                                 (_values((n, heads, page, dim), gen).transpose(2, 3).contiguous(), vc, vs)):
            b = _exponent(x.abs().amax(dim=(2, 3)))
            codes[p:p + n] = _to_e4m3(x * _power(254 - b)[:, :, None, None]).view(torch.uint8)
            scales[p:p + n] = b.to(torch.uint8)
    return kc, vc, ks, vs


def _garbage(kc, vc, where, used, page):
    """Random bytes, NaN codes among them, in the unused places of the pages `where` (used tokens of each)."""
    free = torch.arange(page, device="cuda")[None, :] >= used[:, None]
    k, v = kc[where], vc[where]
    junk = (torch.arange(k.shape[1] * k.shape[2] * k.shape[3], device="cuda") % 257).to(torch.uint8)
    kc[where] = torch.where(free[:, None, :, None], junk.view(k.shape[1:]), k)
    vc[where] = torch.where(free[:, None, None, :], junk.view(v.shape[1:]), v)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dev = dict(device="cuda")
    s = dict(op=case["op"], page=case["page"])
    if case["op"] == "plan":
        n, tokens, page = case["requests"], case["tokens"], case["page"]
        r = random.Random(case["pick"] * 1000003 + seed)
        lens = [r.randint(0, case["len_hi"]) for _ in range(n)]
        new = [_log_int(r, 1, case["new_hi"]) if r.random() < 0.95 else 0 for _ in range(n)]
        over = sum(new) - tokens
        for i in range(n):                             # what does not fit the step's token count waits
            cut = min(max(over, 0), new[i])
            new[i], over = new[i] - cut, over - cut
        width = _pages(case["len_hi"] + case["new_hi"], page)
        held = [_pages(x, page) for x in lens]
        order = torch.randperm(sum(held) + tokens // page + n + 1, generator=gen, **dev).to(torch.int32)
        at = torch.arange(width, **dev)[None, :] + torch.tensor([0] + list(np.cumsum(held[:-1])), **dev)[:, None]
        filled = torch.arange(width, **dev)[None, :] < torch.tensor(held, **dev)[:, None]
        table = torch.where(filled, order[at.clamp(max=order.numel() - 1)], torch.full((), -1, dtype=torch.int32, **dev))
        i32 = dict(dtype=torch.int32, **dev)
        s.update(lens=torch.tensor(lens, **i32), new=torch.tensor(new, **i32), table=table.contiguous(), free=order[sum(held):].contiguous(), tokens=tokens,
                 out=(torch.empty(n + 1, **i32), torch.empty(n, **i32), torch.empty(tokens, dtype=torch.int64, **dev), torch.empty(tokens, **i32), torch.empty(tokens, **i32), torch.empty(1, **i32)))
        return s
    cached, new = lengths(case)
    total = [a + b for a, b in zip(cached, new)]
    page, heads, dim, n = case["page"], case["kv_heads"], case["dim"], case["requests"]
    held = [_pages(x, page) for x in total]
    pages, width = sum(held) + 1, max(held)
    order = torch.randperm(pages, generator=gen, **dev)
    kc, vc, ks, vs = _cache(case, pages, gen)
    first = torch.tensor([0] + list(np.cumsum(held[:-1])), **dev)
    at = torch.arange(width, **dev)[None, :] + first[:, None]
    filled = torch.arange(width, **dev)[None, :] < torch.tensor(held, **dev)[:, None]
    table = torch.where(filled, order[at.clamp(max=pages - 1)].to(torch.int32), torch.full((), -1, dtype=torch.int32, **dev)).contiguous()
    s.update(kc=kc, vc=vc, ks=ks, vs=vs)
    cu = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, **dev)
    tokens = sum(new)
    if case["op"] == "append":
        # new tokens as large as the cached ones, some requests' larger: their last page's scale has to grow
        dtype = torch.float32 if case["f32"] else torch.bfloat16
        row = torch.searchsorted(cu[1:].long(), torch.arange(tokens, **dev), right=True)
        pos = torch.arange(tokens, **dev) - cu[row] + torch.tensor(cached, **dev)[row]
        s["slots"] = table[row, pos // page].long() * page + pos % page
        gain = torch.where(row % 3 == 1, 3.0, 1.0)[:, None, None]
        s["k"] = (_keys((tokens, heads, dim), gen) * gain).to(dtype)
        s["v"] = (_values((tokens, heads, dim), gen) * gain).to(dtype)
        return s
    ends = torch.tensor(total, **dev)
    last = table[torch.arange(n, **dev), (ends - 1) // page].long()
    _garbage(kc, vc, last, (ends - 1) % page + 1, page)
    q_heads = case["q_heads"]
    s.update(q=_normal((tokens, q_heads, dim), gen, torch.bfloat16), cu=cu, total=ends.to(torch.int32), table=table, new_hi=max(new), len_hi=max(total), scale=dim ** -0.5,
             cap=case["cap"], window=case["window"], out=torch.empty((tokens, q_heads, dim), dtype=torch.bfloat16, **dev), slopes=None, prefix=None)
    if case["bias"]:
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, q_heads + 1, dtype=torch.float32, **dev) / q_heads)
    if case["prefix"]:
        r = random.Random(case["pick"] + 1)
        s["prefix"] = torch.tensor([min(t, r.randint(0, case["prefix"])) for t in total], dtype=torch.int32, **dev)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------

def _plain_plan(s):
    lens, new, table, free, page, tokens = s["lens"], s["new"], s["table"], s["free"], s["page"], s["tokens"]
    n, width = table.shape
    total = lens + new
    cu = torch.cat([new.new_zeros(1), new.cumsum(0, dtype=torch.int32)])
    had, need = (lens + (page - 1)) // page, (total + (page - 1)) // page
    begin = torch.cumsum(need - had, 0) - (need - had)
    col = torch.arange(width, device=lens.device)[None, :]
    fresh = (col >= had[:, None]) & (col < need[:, None])
    take = begin[:, None] + col - had[:, None]
    page_of = torch.where(take < free.numel(), free[take.clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where(fresh, page_of, table))
    t = torch.arange(tokens, device=lens.device)
    row = torch.searchsorted(cu[1:], t.to(torch.int32), right=True)
    real = row < n
    r = row.clamp(max=n - 1)
    pos = t - cu[r] + lens[r]
    block = table[r, (pos // page).clamp(0, width - 1)].long()
    slots = torch.where(real & (block >= 0), block * page + pos % page, -1)
    return dict(table=table, cu=cu, total=total, slots=slots, positions=torch.where(real, pos, 0).to(torch.int32), requests=torch.where(real, row, -1).to(torch.int32),
                used=(need - had).sum(dtype=torch.int32).view(1))


def _plain_append(s):
    kc, vc, ks, vs, page = s["kc"], s["vc"], s["ks"], s["vs"], s["page"]
    block, place = s["slots"] // page, s["slots"] % page
    starts = torch.cat([block.new_ones(1, dtype=torch.bool), block[1:] != block[:-1]])
    at = torch.nonzero(starts).squeeze(1)              # the first new token of each page
    group = torch.cumsum(starts, 0) - 1
    pages, kept = block[at], place[at]                 # tokens that each page keeps

    def side(x, codes, scales, tokens_last):
        x = x.to(torch.float32)
        amax = x.new_zeros((at.numel(), x.shape[1])).index_reduce_(0, group, x.abs().amax(2), "amax")
        before = torch.where((kept == 0)[:, None], B_MIN, scales[pages].to(torch.int32))
        b = torch.maximum(before, _exponent(amax))
        old = codes[pages]
        moved = _to_e4m3(old.view(torch.float8_e4m3fn).to(torch.float32) * _power((127 + before - b).clamp(min=1))[:, :, None, None]).view(torch.uint8)
        inside = torch.arange(page, device=x.device)[None, :] < kept[:, None]
        inside = inside[:, None, None, :] if tokens_last else inside[:, None, :, None]
        codes[pages] = torch.where(inside & (b > before)[:, :, None, None], moved, old)
        scales[pages] = b.to(torch.uint8)
        new = _to_e4m3(x * _power(254 - b)[group][:, :, None]).view(torch.uint8)
        if tokens_last:
            codes[block, :, :, place] = new
        else:
            codes[block, :, place] = new

    side(s["k"], kc, ks, False)
    side(s["v"], vc, vs, True)
    return _cache_out(s)


def _cache_out(s):
    return dict(k=s["kc"].view(torch.float8_e4m3fn), v=s["vc"].view(torch.float8_e4m3fn), k_exponents=s["ks"], v_exponents=s["vs"])


def _plain_attention(s):
    q, table, cu, total, page = s["q"], s["table"], s["cu"].long(), s["total"].long(), s["page"]
    tokens, q_heads, dim = q.shape
    n, width = table.shape
    heads, length, most = s["kc"].shape[1], width * page, s["new_hi"]
    group = q_heads // heads
    block = table.long().clamp(min=0)
    k = s["kc"][block].view(torch.float8_e4m3fn).to(torch.float32) * _power(s["ks"][block])[..., None, None]
    v = s["vc"][block].view(torch.float8_e4m3fn).to(torch.float32) * _power(s["vs"][block])[..., None, None]
    k = k.permute(0, 2, 4, 1, 3).reshape(n, heads, dim, length)                    # [n][heads][dim][length]
    v = v.permute(0, 2, 1, 4, 3).reshape(n, heads, length, dim)
    j = torch.arange(length, device=q.device)
    there = (j[None, :] < total[:, None]) & (table >= 0).repeat_interleave(page, 1)
    v = torch.where(there[:, None, :, None], v, 0.0)
    i = torch.arange(most, device=q.device)
    new = cu[1:] - cu[:-1]
    token = (cu[:-1, None] + i[None, :]).clamp(max=tokens - 1)                      # [n][most]
    real = i[None, :] < new[:, None]
    qs = q[token].to(torch.float32).view(n, most, heads, group, dim).permute(0, 2, 3, 1, 4).reshape(n, heads, group * most, dim)
    score = torch.matmul(qs, k).view(n, heads, group, most, length) * s["scale"]
    if s["cap"] > 0:
        score = s["cap"] * torch.tanh(score / s["cap"])
    p = (total - new)[:, None] + i[None, :]
    far = p[:, :, None] - j
    if s["slopes"] is not None:
        score = score - s["slopes"].view(heads, group, 1, 1) * far.abs().to(torch.float32)[:, None, None]
    seen = far >= 0
    if s["window"] > 0:
        seen = seen & (far < s["window"])
    if s["prefix"] is not None:
        seen = seen | (j < s["prefix"][:, None].long())[:, None, :]
    seen = (seen & there[:, None, :])[:, None, None]
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    w = torch.exp(score - torch.where(torch.isfinite(top), top, 0.0))
    del score
    total_w = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(n, heads, group * most, length), v).view(n, heads, group, most, dim) / torch.where(total_w > 0, total_w, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(n, most, q_heads, dim).to(torch.bfloat16)
    row = torch.searchsorted(cu[1:].contiguous(), torch.arange(tokens, device=q.device), right=True)
    return o[row, torch.arange(tokens, device=q.device) - cu[row]]


def run(s):
    if not own:
        return {"plan": _plain_plan, "append": _plain_append, "attention": _plain_attention}[s["op"]](s)
    import paper_2501_04052_amd as razer
    if s["op"] == "plan":
        p = razer.razer_cache_plan(s["lens"], s["new"], s["table"], s["free"], s["page"], s["tokens"], out=s["out"])
        return dict(table=s["table"], cu=p.cu, total=p.total, slots=p.slots, positions=p.positions, requests=p.requests, used=p.used)
    cache = razer.KVCache(s["kc"], s["vc"], s["ks"], s["vs"])
    if s["op"] == "append":
        razer.razer_cache_append(cache, s["k"], s["v"], s["slots"])
        return _cache_out(s)
    return razer.razer_cache_attention(cache, s["q"], s["cu"], s["total"], s["table"], max_new=s["new_hi"], max_len=s["len_hi"], scale=s["scale"], cap=s["cap"], window=s["window"],
                                       slopes=s["slopes"], prefix=s["prefix"], out=s["out"])


# ---- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    n, page = case["requests"], case["page"]
    if case["op"] == "plan":                           # lengths in; offsets, totals, slots, positions, requests and new table entries out
        return dict(bytes=8 * n + 4 * (2 * n + 2) + 16 * case["tokens"] + 8 * _pages(case["tokens"], page), flops=case["tokens"])
    heads, dim = case["kv_heads"], case["dim"]
    cached, new = lengths(case)
    if case["op"] == "append":
        tokens = sum(new)
        touched = sum(_pages(a + b, page) - a // page for a, b in zip(cached, new))
        return dict(bytes=tokens * heads * dim * 2 * ((4 if case["f32"] else 2) + 1) + 8 * tokens + 2 * touched * heads, flops=4 * tokens * heads * dim)
    r = random.Random(case["pick"] + 1)
    pairs = keys = 0
    for a, b in zip(cached, new):
        total = a + b
        prefix = min(total, r.randint(0, case["prefix"])) if case["prefix"] else 0
        p = np.arange(a, total, dtype=np.int64)
        low = np.maximum(0, p - case["window"] + 1) if case["window"] > 0 else np.zeros_like(p)
        pairs += int((np.maximum(p + 1 - np.maximum(low, prefix), 0) + prefix).sum())
        keys += max(0, total - max(int(low[0]), prefix)) + prefix if b else 0
    rows = sum(new) * case["q_heads"] * dim
    return dict(bytes=4 * rows + keys * heads * 2 * dim + 2 * heads * _pages(keys, page) + 4 * _pages(keys, page) + 8 * n, flops=4 * pairs * case["q_heads"] * dim)


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------

def _decode64(codes, exponent):
    """E4M3 bytes with an exponent byte, from the format's equation."""
    c = codes.to(torch.int64)
    e, m = (c >> 3) & 15, (c & 7).double()
    x = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2((e - 7).double()))
    return torch.where(c >= 128, -x, x) * torch.exp2(exponent.double() - 127)


def _round64(x):
    """The nearest E4M3 value (ties to the even code) of |x| <= 448, as float64."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    if case["op"] == "plan":
        return None                                    # whole numbers only
    s = prepare(case, seed)
    page, heads = s["page"], s["kc"].shape[1]
    if case["op"] == "append":
        cached, new = lengths(case)
        k, v = (_decode64(c, torch.tensor(127, device="cuda")) for c in (s["kc"], s["vc"]))
        t = 0
        for a, b in zip(cached, new):
            at = a
            while at < a + b:
                off = at % page
                count = min(page - off, a + b - at)
                pg = int(s["slots"][t]) // page
                for x, codes, scales in ((s["k"], k[pg], s["ks"][pg]), (s["v"], v[pg].transpose(1, 2), s["vs"][pg])):
                    rows = x[t:t + count].double().transpose(0, 1)                  # [heads][count][dim]
                    amax = rows.abs().amax((1, 2)).clamp(min=2.0 ** -120)
                    e = torch.ceil(torch.log2(amax / 448)).clamp(-50, 50)
                    before = scales.double() - 127 if off else torch.full_like(e, -50.0)
                    e = torch.maximum(e, before)
                    codes[:, :off] = _round64(codes[:, :off] * torch.exp2(before - e)[:, None, None])
                    codes[:, off:off + count] = _round64(rows * torch.exp2(-e)[:, None, None])
                t, at = t + count, at + count
        return dict(k=k, v=v, k_exponents=None, v_exponents=None)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    total, cu = s["total"].tolist(), s["cu"].tolist()
    group = s["q"].shape[1] // heads
    for r, length in enumerate(total):
        n = cu[r + 1] - cu[r]
        pages = s["table"][r, :_pages(length, page)].long()
        at = torch.arange(length, device="cuda")
        pos = torch.arange(length - n, length, device="cuda")
        far = pos[:, None] - at[None, :]
        seen = far >= 0
        if s["window"] > 0:
            seen &= far < s["window"]
        if s["prefix"] is not None:
            seen |= (at < s["prefix"][r])[None, :]
        for h in range(heads):
            k = _decode64(s["kc"][pages, h], s["ks"][pages, h][:, None, None]).reshape(-1, s["q"].shape[2])[:length]
            v = _decode64(s["vc"][pages, h], s["vs"][pages, h][:, None, None]).transpose(1, 2).reshape(-1, s["q"].shape[2])[:length]
            for g in range(h * group, (h + 1) * group):
                score = s["q"][cu[r]:cu[r + 1], g].double() @ k.t() * s["scale"]
                if s["cap"] > 0:
                    score = s["cap"] * torch.tanh(score / s["cap"])
                if s["slopes"] is not None:
                    score = score - s["slopes"][g].double() * far.abs()
                out[cu[r]:cu[r + 1], g] = torch.softmax(score.masked_fill(~seen, -math.inf), -1) @ v
    return out
