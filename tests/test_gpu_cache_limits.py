"""Attention over the 8-bit cache at the ends of its arguments' ranges: caps from the smallest to the largest."""
import numpy as np
import pytest
import torch

from gpu_util import launched_kernels
from test_gpu_cache import Batch

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
