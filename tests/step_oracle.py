"""The operators of include/razer_step.h from their definition, in numpy and 64 bits, with bounds of what the roundings
that the header names can add up to."""
import math

import numpy as np

U32, U16 = 2.0 ** -24, 2.0 ** -8         # half a step of fp32 and of bf16, relative


def bf16(x):
    """x rounded to bf16 (nearest, ties to even), as float32."""
    b = np.ascontiguousarray(x, np.float32).view(np.uint32)
    b = (b + 0x7FFF + ((b >> 16) & 1)) & np.uint32(0xFFFF0000)
    return b.astype(np.uint32).view(np.float32)


# ---- norm -----------------------------------------------------------------------------------------------------

def norm(x, weight, eps, residual=None, offset=0.0):
    """(y, h) in float64."""
    h = x.astype(np.float64) + (0 if residual is None else residual.astype(np.float64))
    return h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * (offset + weight.astype(np.float64)), h


def norm_steps(x, weight, eps, residual=None, offset=0.0):
    """y in float32, operation by operation as the header has it."""
    f = np.float32
    h = x.astype(f) if residual is None else x.astype(f) + residual.astype(f)
    h64 = h.astype(np.float64)
    with np.errstate(divide="ignore"):
        s = (1.0 / np.sqrt((h64 * h64).sum(1, keepdims=True) / x.shape[1] + np.float64(f(eps)))).astype(f)
    return (h * s) * (f(offset) + weight.astype(f)), h


# ---- routing --------------------------------------------------------------------------------------------------

def route(logits, top_k, score="softmax", bias=None, renormalize=True, scale=1.0):
    """(ids, weights, gap): gap is the least difference of neighbours in a row's order around its top_k."""
    l = logits.astype(np.float64)
    l = np.where(np.isnan(l), -np.inf, np.minimum(l, np.finfo(np.float32).max))
    with np.errstate(over="ignore", invalid="ignore"):
        p = 1.0 / (1.0 + np.exp(-l)) if score == "sigmoid" else None
        key = (l if p is None else p) + (0 if bias is None else bias.astype(np.float64)[None])
        if p is None:
            m = l.max(1, keepdims=True)
            e = np.where(l > -np.inf, np.exp(l - np.where(np.isfinite(m), m, 0.0)), 0.0)
            p = e / np.where(e.sum(1, keepdims=True) > 0, e.sum(1, keepdims=True), 1.0)
    key = np.where(np.isnan(key), -np.inf, key)
    order = np.argsort(-key, axis=1, kind="stable")
    ids = order[:, :top_k]
    w = np.take_along_axis(p, ids, 1)
    if renormalize:
        s = w.sum(1, keepdims=True)
        w = np.where(s > 0, w / np.where(s > 0, s, 1.0), 0.0)
    ranked = np.take_along_axis(key, order[:, :top_k + 1], 1)
    with np.errstate(invalid="ignore"):
        gap = np.abs(np.diff(ranked, axis=1)).min(1) if ranked.shape[1] > 1 else np.full(len(l), np.inf)
    return ids, w * scale, gap


# ---- experts --------------------------------------------------------------------------------------------------

def activation(z, act):
    """(act(z), a bound of its slope)"""
    with np.errstate(over="ignore"):
        if act == "relu":
            return np.maximum(z, 0.0), 1.0
        if act == "silu":
            return z / (1.0 + np.exp(-z)), 1.1
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))), 1.13


def experts(x, ids, weights, gate, up, down, act="silu", between=U16):
    """(y, bound) in float64; gate, up, down: lists of float64 matrices; between: the rounding of what stands between the products."""
    x = x.astype(np.float64)
    y = np.zeros((x.shape[0], down[0].shape[0]))
    bound = np.zeros_like(y)
    for t in range(x.shape[0]):
        for j in range(ids.shape[1]):
            e, w = int(ids[t, j]), float(weights[t, j])
            if not 0 <= e < len(gate):
                continue
            z = gate[e] @ x[t]
            dz = (x.shape[1] + 2) * U32 * (np.abs(gate[e]) @ np.abs(x[t]))         # fp32 sum in any order, tensor scale
            a, slope = activation(z, act)
            da = slope * dz + 16 * U32 * np.abs(a)                                  # exp, sum, quotient and their like
            if up is not None:
                u = up[e] @ x[t]
                du = (x.shape[1] + 2) * U32 * (np.abs(up[e]) @ np.abs(x[t]))
                a, da = a * u, da * (np.abs(u) + du) + np.abs(a) * du + U32 * np.abs(a * u)
            da = da + between * (np.abs(a) + da)                                    # rounded to bf16, or its rest rounded again
            y[t] += w * (down[e] @ a)
            bound[t] += abs(w) * (np.abs(down[e]) @ (da + (down[e].shape[1] + 4) * U32 * (np.abs(a) + da)))
    return y, bound + ids.shape[1] * U32 * np.abs(y) + U16 * (np.abs(y) + bound) + 1e-38


# ---- sampling -------------------------------------------------------------------------------------------------

def sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, largest=np.finfo(np.float32).max):
    """largest: of the logits' type.  (tokens, logprobs, margin): margin is how far, in shares of the row's weight, a border is from where it would
    choose another token."""
    tokens, logprobs, margins = [], [], []
    for r in range(logits.shape[0]):
        l = logits[r].astype(np.float64)
        l = np.where(np.isnan(l), -np.inf, np.minimum(l, np.float64(largest)))
        order = np.argsort(-l, kind="stable")
        order = order[l[order] > -np.inf]
        if not len(order):
            tokens.append(-1), logprobs.append(-np.inf), margins.append(np.inf)
            continue
        t = 1.0 if temperature is None else float(temperature[r])
        if not t > 0:
            tokens.append(int(order[0])), logprobs.append(0.0), margins.append(np.inf)
            continue
        w = np.exp((l[order] - l[order[0]]) / t)
        margin = np.inf
        if top_k is not None and top_k[r] > 0:
            w = w[:int(top_k[r])]
        n = len(w)
        if top_p is not None and top_p[r] < 1:
            run, want = np.cumsum(w), max(float(top_p[r]), 0.0) * w.sum()
            n = min(n, 1 + int((run < want).sum()))
            margin = np.abs(run - want).min() / w.sum()
        if min_p is not None and min_p[r] > 0:
            m = min(float(min_p[r]), 1.0)
            margin = min(margin, np.abs(w - m).min() if m < 1.0 else np.inf)
            n = min(n, int((w >= m).sum()))
        w = w[:n]
        u = float(uniform[r])
        run, want = np.cumsum(w), (0.0 if not u > 0 else min(u, 1.0)) * w.sum()
        last = int((w > 0).sum()) - 1
        at = min(last, int((run <= want).sum()))
        if 0 < want < w.sum():
            margin = min(margin, np.abs(run - want).min() / w.sum())
        tokens.append(int(order[at])), logprobs.append(float(np.log(w[at] / w.sum()))), margins.append(margin)
    return np.array(tokens), np.array(logprobs), np.array(margins)
