"""The 8-bit paged key/value cache from its definition, in 64 bits on the host: plain loops over requests and runs."""
import numpy as np

B_MIN, B_MAX = 77, 177


def e4m3_values():
    """Value of every code (FP8 equation: E=0: M/512, else 2^(E-7)(1+M/8)); 0x7F and 0xFF are NaN."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    x = np.where(e == 0, m / 512.0, np.ldexp(1 + m / 8.0, e - 7))
    x = np.where(c >= 128, -x, x)
    x[[0x7F, 0xFF]] = np.nan
    return x


VALUES = e4m3_values()


def encode(x):
    """Codes of the nearest values (ties to the even code), |x| <= 448; the sign of zero is kept."""
    x = np.asarray(x, dtype=np.float64)
    pos = VALUES[:127]
    mid = (pos[1:] + pos[:-1]) / 2
    a = np.abs(x)
    code = np.searchsorted(mid, a, side="left")                      # a == mid[i] -> i
    tie = (code < 126) & (a == mid[np.minimum(code, 125)])
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    code = np.where(np.isnan(x), 127, code)                          # (a NaN code that is moved stays one)
    return np.where(np.signbit(x), code | 128, code).astype(np.uint8)


def exponent(amax):
    """Smallest b in range with amax <= 448 * 2^(b-127)."""
    b = B_MIN
    while b < B_MAX and amax > np.ldexp(448.0, b - 127):
        b += 1
    return b


class Cache:
    """Codes and exponent bytes as the ABI lays them out."""

    def __init__(self, pages, heads, dim, page, rng=None):
        fill = (lambda s: rng.integers(0, 256, s, dtype=np.uint8)) if rng is not None else (lambda s: np.zeros(s, np.uint8))
        self.k, self.v = fill((pages, heads, page, dim)), fill((pages, heads, dim, page))
        self.ks, self.vs = fill((pages, heads)), fill((pages, heads))
        self.pages, self.heads, self.dim, self.page = pages, heads, dim, page

    def append(self, k, v, slots):
        t, n = 0, len(slots)
        while t < n:
            s = int(slots[t])
            if s < 0 or s >= self.pages * self.page:
                t += 1
                continue
            pg, off, run = s // self.page, s % self.page, 1
            while t + run < n and off + run < self.page and slots[t + run] == s + run:
                run += 1
            for h in range(self.heads):
                self._side(k[t:t + run, h], self.k[pg, h], self.ks, pg, h, off)
                self._side(v[t:t + run, h], self.v[pg, h].T, self.vs, pg, h, off)
            t += run

    def _side(self, x, codes, scales, pg, h, off):                   # codes [page][dim] (a view)
        x = x.astype(np.float64)
        finite = np.abs(x[np.isfinite(x)])
        b = exponent(finite.max() if finite.size else 0.0)
        if off:
            before = int(scales[pg, h])
            b = max(b, before)
            if b > before:
                codes[:off] = encode(VALUES[codes[:off]] * np.ldexp(1.0, before - b))
        scales[pg, h] = b
        y = np.where(np.isnan(x), 0.0, x) * np.ldexp(1.0, 127 - b)
        codes[off:off + len(x)] = encode(np.clip(y, -448, 448))

    def keys_values(self, pages, h):
        """[tokens][dim] of the pages, one head."""
        k = [VALUES[self.k[p, h]] * np.ldexp(1.0, int(self.ks[p, h]) - 127) for p in pages]
        v = [VALUES[self.v[p, h]].T * np.ldexp(1.0, int(self.vs[p, h]) - 127) for p in pages]
        return np.concatenate(k), np.concatenate(v)


def plan(lens, fresh, table, free, page, tokens):
    table = table.copy()
    n, width = table.shape
    cu, total = np.zeros(n + 1, np.int64), np.zeros(n, np.int64)
    slots, positions, request = np.full(tokens, -1, np.int64), np.zeros(tokens, np.int64), np.full(tokens, -1, np.int64)
    taken = t = 0
    for r in range(n):
        total[r] = lens[r] + fresh[r]
        cu[r + 1] = cu[r] + fresh[r]
        for i in range(-(-int(lens[r]) // page), -(-int(total[r]) // page)):
            if i < width:
                table[r, i] = free[taken] if taken < len(free) else -1
            taken += 1
        for pos in range(int(lens[r]), int(total[r])):
            pg = table[r, pos // page] if pos // page < width else -1
            slots[t] = -1 if pg < 0 else int(pg) * page + pos % page
            positions[t], request[t] = pos, r
            t += 1
    return dict(table=table, cu=cu, total=total, slots=slots, positions=positions, requests=request, used=np.array([taken]))


def attention(cache, q, cu, total, table, scale, cap=0.0, window=0, slopes=None, prefix=None):
    """(out, bound): out [tokens][q_heads][dim] in 64 bits, and how far a bf16 result may be from it.

    What the bound is made of: the result is rounded to bf16 (8 significant bits: half a unit is up to 2^-8 of it);
    the weights are rounded to f16 for the product with the values (11 bits: 2^-11 of sum w|v|; what is 2^-38 of the
    largest or less may be lost); a score's error d (fp32 products and sums, the cap and the bias in
    fp32, the difference to the running maximum) changes a weight by the factor e^d; sums over n keys in fp32."""
    tokens, q_heads, dim = q.shape
    q = q.astype(np.float64)
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    group = q_heads // cache.heads
    for r in range(len(total)):
        n, length = int(cu[r + 1] - cu[r]), int(total[r])
        if n <= 0:
            continue
        pages = table[r][: -(-length // cache.page)]
        there = np.zeros(length, bool)
        ok = [i for i, p in enumerate(pages) if 0 <= p < cache.pages]
        for i in ok:
            there[i * cache.page:(i + 1) * cache.page] = True
        j, p = np.arange(length), np.arange(length - n, length)
        far = p[:, None] - j[None, :]
        seen = far >= 0
        if window > 0:
            seen &= far < window
        if prefix is not None:
            seen |= (j < prefix[r])[None, :]
        seen &= there[None, :]
        for h in range(q_heads):
            k, v = np.zeros((length, dim)), np.zeros((length, dim))
            if ok:
                kk, vv = cache.keys_values([pages[i] for i in ok], h // group)
                kk, vv = kk[: there.sum()], vv[: there.sum()]
                k[there], v[there] = kk, vv
            x = q[cu[r]:cu[r + 1], h]
            s = scale * (x @ k.T)
            err = (dim + 8) * 2.0 ** -24 * abs(scale) * (np.abs(x) @ np.abs(k).T)
            if cap > 0:
                s = cap * np.tanh(s / cap)
                err = err + 8 * 2.0 ** -24 * cap
            if slopes is not None:
                bias = slopes[h] * np.abs(far)
                s = s - bias
                err = err + 4 * 2.0 ** -24 * bias
            err = err + 8 * 2.0 ** -24 * (1 + np.abs(s))
            s = np.where(seen, s, -np.inf)
            top = s.max(1, keepdims=True) if length else np.zeros((n, 1))
            w = np.exp(s - np.where(np.isfinite(top), top, 0.0))
            w = np.where(seen, w, 0.0)
            sums = w.sum(1, keepdims=True)
            w = w / np.where(sums > 0, sums, 1.0)
            o, size = w @ v, w @ np.abs(v)
            d = 2 * np.where(seen & (w > 1e-12), err, 0.0).max(1, keepdims=True) if length else 0.0
            d = d + 2 * np.where(np.isfinite(top), np.abs(top), 0.0) * 2.0 ** -23
            out[cu[r]:cu[r + 1], h] = o
            bound[cu[r]:cu[r + 1], h] = 1.02 * (2.0 ** -8 * np.abs(o) + 2.0 ** -11 * size) + size * (d + 2 * length * 2.0 ** -24)
    return out, bound
