"""The 8-bit cache at the ends of its arguments' ranges: slots with gaps and skipped tokens, caps from the smallest to the largest, windows and offsets past 32 bits,
workspaces, many rows over many tiles."""
import numpy as np
import pytest
import torch

import cache_oracle as co
from gpu_util import launched_kernels
from test_gpu_cache import Batch, bf16_rows, dev, same_cache, some_rows, upload

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def razer():
    import paper_2501_04052_amd as r
    r.load_library()
    return r


def capped_attention(b, cap, scale):
    """(out, bound) of causal attention with capped scores in 64 bits.  The bound is made like the oracle's, with a cap that
    costs a score 2^-18 of itself, however large the cap is: from |s| = cap / 4 on the two roundings of 2y log2(e), the
    exponential's and the reciprocal's unit in the last place and three more roundings change tanh y by less than
    2^-19 of it, and below the series by less than 2^-21."""
    heads, dim = b.ref.heads, b.ref.dim
    group = b.q.shape[1] // heads
    q = b.q.astype(np.float64)
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    for r, length in enumerate(b.total):
        rows = slice(b.cu[r], b.cu[r + 1])
        n = b.cu[r + 1] - b.cu[r]
        seen = np.arange(length)[None, :] <= np.arange(length - n, length)[:, None]
        for h in range(b.q.shape[1]):
            k, v = (x[:length] for x in b.ref.keys_values(b.table[r, :-(-length // b.ref.page)], h // group))
            x = q[rows, h]
            s = cap * np.tanh(scale * (x @ k.T) / cap)
            err = (dim + 8) * 2.0 ** -24 * abs(scale) * (np.abs(x) @ np.abs(k).T) + 2.0 ** -18 * np.abs(s) + 8 * 2.0 ** -24 * (1 + np.abs(s))
            s = np.where(seen, s, -np.inf)
            top = s.max(1, keepdims=True)
            w = np.exp(s - top)
            w /= w.sum(1, keepdims=True)
            d = 2 * np.where(seen & (w > 1e-12), err, 0.0).max(1, keepdims=True) + 2 * np.abs(top) * 2.0 ** -23
            o, size = w @ v, w @ np.abs(v)
            out[rows, h] = o
            bound[rows, h] = 1.02 * (2.0 ** -8 * np.abs(o) + 2.0 ** -11 * size) + size * (d + 2 * length * 2.0 ** -24)
    return out, bound


@pytest.mark.parametrize("cap", [1e-40, 1e-3, 1.0, 30.0, 1e3, 1e4, 1e6, 1e8, 1e12, 3e38])
@pytest.mark.parametrize("dim,page,total,fresh,known,kernel", [
    (128, 64, [300, 5], [3, 5], dict(max_new=3, max_len=300), "rows_kernel"),
    (128, 64, [2500, 40], [3, 2], dict(max_new=3, max_len=2500), "shares_kernel"),
    (256, 32, [2500, 40], [3, 2], dict(max_new=3, max_len=2500), "shares_kernel"),
    (64, 16, [300, 40], [20, 40], dict(max_new=40, max_len=300), "tiles_kernel"),
    (256, 128, [300, 40], [20, 40], dict(max_new=40, max_len=300), "tiles_kernel")])
def test_attention_with_caps_of_any_size(razer, dim, page, total, fresh, known, kernel, cap):
    """A cap far above the scores leaves them as they are; one far below makes them its sign."""
    for seed, gain, scale in ((90, 1.0, dim ** -0.5), (91, 6.0, dim ** -0.5), (92, 2.0, -0.07), (93, 0.0, dim ** -0.5)):
        b = Batch(razer, seed, dim, page, 2, 4, total, fresh, gain=gain)
        want, bound = capped_attention(b, cap, scale)
        call = lambda: b.call(cap=cap, scale=scale, **known)
        if seed == 90:
            assert any(kernel in n for n in launched_kernels(call))
        got = call().float().cpu().numpy().astype(np.float64)
        bad = ~(np.abs(got - want) <= bound)
        assert not bad.any(), "seed %d: %d of %d off: %s instead of %s" % (seed, bad.sum(), bad.size, got[bad][:3], want[bad][:3])


# ---- append ---------------------------------------------------------------------------------------------------

class AnyBytes(co.Cache):
    """A cache whose pages may be gone on with before they are begun: an earlier exponent byte outside the range counts as the
    nearer end of it."""

    def _side(self, x, codes, scales, pg, h, off):
        if off:
            scales[pg, h] = np.clip(scales[pg, h], co.B_MIN, co.B_MAX)
        super()._side(x, codes, scales, pg, h, off)


def append_and_compare(razer, seed, slots, pages, page, dim=64, heads=2, f32=False):
    """Twice into the same pages, so that scales have to grow, or not, in the middle of a page."""
    rng = np.random.default_rng(seed)
    ref = AnyBytes(pages, heads, dim, page, rng)
    got = upload(razer, ref)
    slots = np.array(slots)
    for gain in (1.0, 20.0):
        k, v = (some_rows(rng, len(slots), heads, dim) * (gain * 2.0 ** rng.integers(-4, 5, (len(slots), 1, 1))).astype(np.float32) for _ in range(2))
        if f32:
            kd, vd = dev(k), dev(v)
        else:
            (kd, k), (vd, v) = bf16_rows(k), bf16_rows(v)
        razer.razer_cache_append(got, kd, vd, dev(slots, torch.int64))
        ref.append(k, v, slots)
        same_cache(got, ref)


def test_append_of_a_page_with_skipped_tokens(razer):
    for slots in ([16, 17, -1, 19], [17, -1, 18], [16, 18, 21], [33, -1, -1, 34, 35, -1, 40, 0, -1, 2], [-1, 5, -9, 1 << 50, 7, 48], [16, -1, 17, 32, -1, 33]):
        append_and_compare(razer, 1, slots, 4, 16)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_append_of_a_page_whose_first_and_last_rows_are_far_apart(razer, page):
    """Nothing but skipped rows between a page's tokens, at every place of the windows of rows that are looked at together."""
    for lead in (0, 1, 15, 16, 17, 63, 64, 130):
        for between in sorted({1, 13, 14, page // 2, page - 3, page - 2}):
            slots = [-1] * lead + [page + 1] + [-1] * between + [2 * page - 1, 3 * page, -1, 3 * page + 2] + [-1] * (page + 3) + [4 * page + 5]
            append_and_compare(razer, lead * 131 + between, slots, 6, page, heads=1)


def masked_pages(rng, pages, page, tokens):
    """Slots of pages in any order: whole, single, thinned out, with gaps, and skipped rows before, between and behind."""
    slots = []
    for p in rng.permutation(pages):
        a = int(rng.integers(page))
        b = int(rng.integers(a, page))
        rows = [p * page + np.arange(page), p * page + np.array([a]), np.where(rng.random(page) < 0.5, p * page + np.arange(page), -1),
                p * page + np.arange(a, b + 1)[rng.random(b + 1 - a) < 0.7], np.where(rng.random(b + 1 - a) < 0.95, p * page + np.arange(a, b + 1), pages * page + 3)]
        slots += list(rows[rng.integers(len(rows))]) + [-1] * int(rng.choice([0, 0, 0, 1, 7, 20, 70]))
        if len(slots) >= tokens:
            break
    return slots


@pytest.mark.parametrize("tokens", [200, 900, 2500])
@pytest.mark.parametrize("page,dim,f32", [(16, 64, False), (16, 192, True), (32, 128, False), (64, 64, True), (128, 128, False), (128, 256, False)])
def test_append_of_masked_steps(razer, page, dim, f32, tokens):
    for seed in range(3):
        slots = masked_pages(np.random.default_rng(seed * 7 + page + tokens), 3 * tokens // page + 4, page, tokens)
        append_and_compare(razer, seed, slots, 3 * tokens // page + 4, page, dim, 1 + seed, f32)


# ---- workspace ------------------------------------------------------------------------------------------------

def test_one_workspace_serves_every_window_and_shorter_length(razer):
    """The size that is told for the longest length is enough for calls that are cut up in another way; what lies behind it is not touched."""
    heads, dim, page, tokens, most = 8, 128, 64, 512, 8256
    gen = torch.Generator(device="cuda").manual_seed(5)
    codes = lambda *s: torch.randint(0, 0x70, s, generator=gen, device="cuda", dtype=torch.uint8)
    held = most // page
    cache = razer.KVCache(codes(held, heads, page, dim), codes(held, heads, dim, page), torch.full((held, heads), 120, dtype=torch.uint8, device="cuda"),
                          torch.full((held, heads), 120, dtype=torch.uint8, device="cuda"))
    q = torch.randn((tokens, heads, dim), generator=gen, device="cuda").to(torch.bfloat16)
    cu, total, table = dev([0, tokens], torch.int32), dev([most], torch.int32), torch.arange(held, dtype=torch.int32, device="cuda").view(1, -1)
    need = razer.razer_attention_workspace_bytes(cache, q, cu, total, table, tokens, most)
    ws = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    for length, window in ((most, 0), (most, 7488), (8192, 0), (8192, 3000), (most, 700), (2048, 0), (600, 0)):
        total[0] = length
        kw = dict(max_new=tokens, max_len=length, window=window)
        got = razer.razer_cache_attention(cache, q, cu, total, table, workspace=ws[:need], **kw)
        assert (ws[need:] == 171).all()
        assert torch.equal(got, razer.razer_cache_attention(cache, q, cu, total, table, **kw))


# ---- windows --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fresh,kernel", [(1, "shares_kernel"), (20, "tiles_kernel")])
def test_attention_with_windows_and_positions_past_30_bits(razer, fresh, kernel):
    """A request of more than 2^30 keys, of which only the first page is there: what a window leaves of it is what the same window,
    shortened by the keys that are not there, leaves of a short request."""
    dim, page, heads, far = 64, 128, 2, (1 << 30) - 200
    rng = np.random.default_rng(17)
    ref = co.Cache(1, 1, dim, page)
    k, v = (rng.standard_normal((page, 1, dim)).astype(np.float32) for _ in range(2))
    ref.append(k, v, np.arange(page))
    cache = upload(razer, ref)
    q = torch.from_numpy(rng.standard_normal((fresh, heads, dim)).astype(np.float32)).to(torch.bfloat16)
    total = far + 240
    table = torch.full((1, -(-total // page)), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    for window in ((1 << 30) - 1, 1 << 30, (1 << 30) + 10, (1 << 30) + 25, (1 << 31) - 1):
        want, bound = co.attention(ref, q.float().numpy(), [0, fresh], [240], np.array([[0, -1]]), dim ** -0.5, window=window - far)
        call = lambda: razer.razer_cache_attention(cache, q.cuda(), dev([0, fresh], torch.int32), dev([total], torch.int32), table, max_new=fresh, max_len=total, window=window)
        if window == 1 << 30:
            assert any(kernel in n for n in launched_kernels(call))
        assert (np.abs(call().float().cpu().numpy() - want) <= bound).all(), window


# ---- many rows over many tiles --------------------------------------------------------------------------------

@pytest.fixture(scope="module", params=[(64, 16, 2, 3), (128, 64, 1, 4), (192, 32, 1, 5), (256, 128, 2, 2)], ids=str)
def long_batch(request, razer):
    """A prompt's part, whole units and cut ones, a draft and a prompt: up to 47 tiles of 64 keys."""
    dim, page, heads, group = request.param
    return Batch(razer, dim + page, dim, page, heads, group, [3000, 1500, 129, 40], [40, 90, 3, 40])


LONG = [{}, {"prefix": [700, 0, 64, 10 ** 6], "window": 1500, "cap": 5.0, "bias": True}, {"prefix": [1, 1300, 0, 3], "window": 700}, {"bias": True}]


def long_options(b, opt):
    kw = dict(opt)
    if kw.pop("bias", False):
        kw["slopes"] = (2.0 ** (-8.0 * np.arange(1, b.q.shape[1] + 1) / b.q.shape[1])).astype(np.float32)
    if "prefix" in kw:
        kw["prefix"] = np.array(kw["prefix"])
    return kw


@pytest.mark.parametrize("opt", LONG, ids=str)
def test_attention_of_many_rows_over_many_tiles(razer, long_batch, opt):
    """One workgroup a unit, however many tiles it has: the announced length is too short to cut the keys."""
    kw = dict(long_options(long_batch, opt), max_new=90, max_len=64)
    names = launched_kernels(lambda: long_batch.call(**kw))
    assert any("tiles_kernel" in n for n in names) and not any("join_kernel" in n for n in names), names
    long_batch.check(**kw)


@pytest.mark.parametrize("opt", LONG, ids=str)
def test_attention_of_many_rows_with_the_keys_cut(razer, long_batch, opt):
    """Chunks that end in the middle of a prefix, of a window and behind a unit's last tile, put together by the join."""
    kw = dict(long_options(long_batch, opt), max_new=90, max_len=3000)
    names = launched_kernels(lambda: long_batch.call(**kw))
    cut = (min(opt.get("window", 3000) + 90, 3000) // 64 + 3) // 8 > 1     # at least 8 tiles a chunk
    assert any("tiles_kernel" in n for n in names) and any("join_kernel" in n for n in names) == cut, names
    out = long_batch.check(**kw)
    assert torch.equal(long_batch.call(**kw), out)


@pytest.mark.parametrize("max_new,max_len,kernel", [(40, 300, "tiles_kernel"), (1, 300, "rows_kernel"), (1, 0, "shares_kernel")])
def test_attention_of_pages_past_32_bit_offsets(razer, max_new, max_len, kernel):
    heads, dim, page, tokens = 8, 128, 128, 40
    pages = (1 << 32) // (heads * dim * page) + 40
    cache = razer.KVCache.allocate(pages, heads, dim, page)
    rng = np.random.default_rng(19)
    ref = co.Cache(6, heads, dim, page)
    k, v = some_rows(rng, 300, heads, dim), some_rows(rng, 300, heads, dim)
    ref.append(k, v, np.arange(300))
    first = pages - 6
    razer.razer_cache_append(cache, dev(k), dev(v), dev(np.arange(300) + first * page, torch.int64))
    wide = np.full((1, 400), -1)
    wide[0, :3] = [0, 1, 2]
    q = torch.from_numpy(rng.standard_normal((tokens, 16, dim)).astype(np.float32)).to(torch.bfloat16)
    want, bound = co.attention(ref, q.float().numpy(), [0, tokens], [300], wide, dim ** -0.5)
    table = dev(np.where(wide >= 0, wide + first, -1), torch.int32)
    call = lambda: razer.razer_cache_attention(cache, q.cuda(), dev([0, tokens], torch.int32), dev([300], torch.int32), table, max_new=max_new, max_len=max_len)
    assert any(kernel in n for n in launched_kernels(call))
    assert (np.abs(call().float().cpu().numpy() - want) <= bound).all()


def test_attention_of_some_requests_of_a_step(razer):
    """Rows of cu, total and table from the middle of a step, with the step's q and out: the other requests' rows are not touched."""
    b = Batch(razer, 94, 128, 32, 2, 4, [300, 1000, 40, 700], [40, 1, 12, 2])
    want, bound = b.want()
    for first, last, new in ((0, 1, 40), (1, 2, 1), (1, 4, 12), (2, 3, 12), (3, 4, 2)):
        out = torch.full_like(b.qd, 9.0)
        razer.razer_cache_attention(b.cache, b.qd, b.cud[first:last + 1], b.totald[first:last], b.tabled[first:last], max_new=new, max_len=1000, out=out)
        rows = np.zeros(b.tokens, bool)
        rows[b.cu[first]:b.cu[last]] = True
        got = out.float().cpu().numpy()
        assert (got[~rows] == 9).all() and (np.abs(got - want)[rows] <= bound[rows]).all(), (first, last)
