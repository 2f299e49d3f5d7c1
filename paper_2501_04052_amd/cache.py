"""The 8-bit paged key/value cache: ctypes binding of include/razer_cache.h.

Same names, same arguments; torch supplies device memory and the current stream, nothing else.

    cache = razer.KVCache.allocate(pages, kv_heads, head_dim, page=64)
    plan = razer.razer_cache_plan(lens, fresh, table, free_pages, cache.page, tokens)       # once per step
    razer.razer_cache_append(cache, k, v, plan.slots)                                       # once per layer
    y = razer.razer_cache_attention(cache, q, plan.cu, plan.total, table)                   # once per layer
"""
import ctypes
import struct
from collections import namedtuple

import torch

from . import binding as _b

# a razer_cache and a razer_attention in one pass (see binding._pack_tensor)
_pack_cache = struct.Struct("@PPPPqiii4x").pack
_pack_attention = struct.Struct("@PqPqqiiPPPqiiqffi4xPP").pack

CachePlan = namedtuple("CachePlan", "cu total slots positions requests used")
CachePlan.__doc__ = """What razer_cache_plan returns: int32 cu [requests + 1], total [requests], positions and requests
[tokens], used [1]; int64 slots [tokens]."""


class KVCache:
    """A cache: four uint8 device tensors (razer_cache in the ABI).

    k_codes [pages][kv_heads][page][head_dim], v_codes [pages][kv_heads][head_dim][page], k_scales and v_scales
    [pages][kv_heads].  The object describes the tensors it was made of; they are not to be replaced."""

    __slots__ = ("k_codes", "v_codes", "k_scales", "v_scales", "pages", "kv_heads", "page", "head_dim", "_struct")

    def __init__(self, k_codes, v_codes, k_scales, v_scales):
        pages, heads, page, dim = k_codes.shape
        assert v_codes.shape == (pages, heads, dim, page) and k_scales.shape == (pages, heads) and v_scales.shape == (pages, heads)
        assert k_codes.dtype is torch.uint8 and k_codes.is_cuda and k_codes.is_contiguous()
        assert v_codes.dtype is torch.uint8 and v_codes.is_cuda and v_codes.is_contiguous()
        assert k_scales.dtype is torch.uint8 and k_scales.is_cuda and k_scales.is_contiguous()
        assert v_scales.dtype is torch.uint8 and v_scales.is_cuda and v_scales.is_contiguous()
        self.k_codes, self.v_codes, self.k_scales, self.v_scales = k_codes, v_codes, k_scales, v_scales
        self.pages, self.kv_heads, self.page, self.head_dim = pages, heads, page, dim
        self._struct = _pack_cache(k_codes.data_ptr(), v_codes.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), pages, heads, dim, page)

    @staticmethod
    def allocate(pages, kv_heads, head_dim, page=64, device="cuda"):
        """An uninitialised cache: a page holds nothing until its first token is appended."""
        new = lambda *s: torch.empty(s, dtype=torch.uint8, device=device)
        return KVCache(new(pages, kv_heads, page, head_dim), new(pages, kv_heads, head_dim, page), new(pages, kv_heads), new(pages, kv_heads))

    def values_of(self, page_ids, dtype=torch.float32):
        """The keys and the values that the pages `page_ids` hold, [n][kv_heads][page][head_dim] each (for inspection;
        places that no token was appended to hold anything)."""
        def side(codes, scales):
            return (codes[page_ids].view(torch.float8_e4m3fn).to(torch.float32)
                    * torch.exp2(scales[page_ids].to(torch.float32) - 127.0)[..., None, None]).to(dtype)
        return side(self.k_codes, self.k_scales), side(self.v_codes, self.v_scales).transpose(2, 3)


_i32, _i64, _f32, _bf16 = torch.int32, torch.int64, torch.float32, torch.bfloat16


def razer_cache_plan(lens, fresh, table, free_pages, page, tokens, out=None):
    """The bookkeeping of one step: request r has lens[r] cached tokens and fresh[r] new ones (int32), `tokens` is the
    step's number of rows (their sum, or more: padding).  table [requests][width] (int32) gets the pages that the new
    tokens begin, taken from free_pages (int32) in order.  out: a CachePlan (or its six tensors) to be filled.
    Returns a CachePlan."""
    L = _b.load_library()
    n, count = lens.numel(), free_pages.numel()
    rows, width = table.shape
    # (each property that is asked for costs about 0.1 us on every call: none is asked for twice)
    assert lens.dtype is _i32 and lens.is_cuda and lens.is_contiguous()
    assert fresh.dtype is _i32 and fresh.is_cuda and fresh.is_contiguous() and fresh.numel() == n
    assert free_pages.dtype is _i32 and free_pages.is_cuda and free_pages.is_contiguous()
    assert table.dtype is _i32 and table.is_cuda and rows == n and (table.stride(1) == 1 or width <= 1 or n == 0)
    if out is None:
        i32 = dict(dtype=_i32, device=lens.device)
        out = CachePlan(torch.empty(n + 1, **i32), torch.empty(n, **i32), torch.empty(tokens, dtype=_i64, device=lens.device),
                        torch.empty(tokens, **i32), torch.empty(tokens, **i32), torch.empty(1, **i32))
        cu, total, slots, positions, requests, used = out
    else:
        cu, total, slots, positions, requests, used = out
        if type(out) is not CachePlan:
            out = CachePlan(cu, total, slots, positions, requests, used)
        assert cu.dtype is _i32 and cu.is_cuda and cu.is_contiguous() and cu.numel() == n + 1
        assert total.dtype is _i32 and total.is_cuda and total.is_contiguous() and total.numel() == n
        assert slots.dtype is _i64 and slots.is_cuda and slots.is_contiguous() and slots.numel() == tokens
        assert positions.dtype is _i32 and positions.is_cuda and positions.is_contiguous() and positions.numel() == tokens
        assert requests.dtype is _i32 and requests.is_cuda and requests.is_contiguous() and requests.numel() == tokens
        assert used.dtype is _i32 and used.is_cuda and used.numel() == 1
    st = L.razer_cache_plan(lens.data_ptr(), fresh.data_ptr(), n, table.data_ptr(), width, table.stride(0) if n > 1 else width, free_pages.data_ptr(),
                            count, page, tokens, cu.data_ptr(), total.data_ptr(), slots.data_ptr(), positions.data_ptr(), requests.data_ptr(),
                            used.data_ptr(), _b._stream())
    if st != 0:
        raise _b.RazerError(st, "razer_cache_plan")
    return out


def _token_stride(t, n, heads, dim):
    """Elements from one token of t [tokens][heads][dim] to the next; heads lie side by side."""
    s0, s1, s2 = t.stride()
    assert s2 == 1 and (heads == 1 or s1 == dim)
    return s0 if n > 1 else max(s0, heads * dim)


def razer_cache_append(cache, k, v, slots):
    """Quantises k and v [tokens][kv_heads][head_dim] (float32 or bfloat16; rows may be longer) into the cache at
    slots [tokens] (int64, a CachePlan's; negative: skipped)."""
    L = _b.load_library()
    tokens, heads, dim = k.shape
    dtype = k.dtype
    assert (dtype is _bf16 or dtype is _f32) and k.is_cuda and heads == cache.kv_heads and dim == cache.head_dim
    assert v.dtype is dtype and v.is_cuda and v.shape == k.shape
    assert slots.dtype is _i64 and slots.is_cuda and slots.is_contiguous() and slots.numel() == tokens
    st = L.razer_cache_append(cache._struct, k.data_ptr(), _token_stride(k, tokens, heads, dim), v.data_ptr(), _token_stride(v, tokens, heads, dim),
                              _b.BF16 if dtype is _bf16 else _b.F32, tokens, slots.data_ptr(), _b._stream())
    if st != 0:
        raise _b.RazerError(st, "razer_cache_append")


def _attention_struct(cache, q, cu, total, table, max_new, max_len, scale, cap, window, slopes, prefix, out):
    tokens, heads, dim = q.shape
    n, width = table.shape
    assert q.dtype is _bf16 and q.is_cuda and dim == cache.head_dim
    assert out.dtype is _bf16 and out.is_cuda and (out is q or out.shape == q.shape)
    assert cu.dtype is _i32 and cu.is_cuda and cu.is_contiguous() and cu.numel() == n + 1
    assert total.dtype is _i32 and total.is_cuda and total.is_contiguous() and total.numel() == n
    assert table.dtype is _i32 and table.is_cuda and (table.stride(1) == 1 or width <= 1 or n == 0)
    sp = pp = 0
    if slopes is not None:
        assert slopes.dtype is _f32 and slopes.is_cuda and slopes.is_contiguous() and slopes.numel() == heads
        sp = slopes.data_ptr()
    if prefix is not None:
        assert prefix.dtype is _i32 and prefix.is_cuda and prefix.is_contiguous() and prefix.numel() == n
        pp = prefix.data_ptr()
    return _pack_attention(q.data_ptr(), _token_stride(q, tokens, heads, dim), out.data_ptr(), _token_stride(out, tokens, heads, dim), tokens, heads, n,
                           cu.data_ptr(), total.data_ptr(), table.data_ptr(), table.stride(0) if n > 1 else width, width,
                           max_new or 0, max_len or 0, dim ** -0.5 if scale is None else scale, cap, window, sp, pp)


def razer_attention_workspace_bytes(cache, q, cu, total, table, max_new=None, max_len=None):
    """Bytes of device workspace that razer_cache_attention needs for these sizes, whatever its other options; enough for every
    smaller max_len too."""
    return int(_b.load_library().razer_attention_workspace_bytes(
        cache._struct, _attention_struct(cache, q, cu, total, table, max_new, max_len, None, 0.0, 0, None, None, q)))


def razer_cache_attention(cache, q, cu, total, table, max_new=None, max_len=None, scale=None, cap=0.0, window=0, slopes=None,
                          prefix=None, out=None, workspace=None):
    """Attention of the new tokens' queries q [tokens][q_heads][head_dim] (bfloat16; rows may be longer) over the cache.

    cu, total, table: of razer_cache_plan.  max_new, max_len: about how many new tokens a request has at most and how
    long it is; they only choose kernels.  scale: 1 / sqrt(head_dim) if not given.  cap: scores are cap * tanh(s / cap).
    window: a query sees the last `window` keys up to its own.  slopes [q_heads] (float32): the score loses slope *
    distance.  prefix [requests] (int32): tokens that every query of the request sees.  cu, total, table and prefix may be
    slices of a step's: the other requests' rows of out are left alone.  Returns bfloat16, q's shape."""
    L = _b.load_library()
    if out is None:
        out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    args = _attention_struct(cache, q, cu, total, table, max_new, max_len, scale, cap, window, slopes, prefix, out)
    if workspace is None:
        need = L.razer_attention_workspace_bytes(cache._struct, args)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    ws, size = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    st = L.razer_cache_attention(cache._struct, args, ws, size, _b._stream())
    if st != 0:
        raise _b.RazerError(st, "razer_cache_attention")
    return out


def declare(L):
    """Argument types of the cache's entry points."""
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    L.razer_cache_plan.restype = ctypes.c_int
    L.razer_cache_plan.argtypes = [vp, vp, i32, vp, i32, i64, vp, i32, i32, i64, vp, vp, vp, vp, vp, vp, vp]
    L.razer_cache_append.restype = ctypes.c_int
    L.razer_cache_append.argtypes = [vp, vp, i64, vp, i64, i32, i64, vp, vp]
    L.razer_attention_workspace_bytes.restype = sz
    L.razer_attention_workspace_bytes.argtypes = [vp, vp]
    L.razer_cache_attention.restype = ctypes.c_int
    L.razer_cache_attention.argtypes = [vp, vp, vp, sz, vp]
