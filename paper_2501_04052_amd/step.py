"""Norm, mixture of experts and sampling: ctypes binding of include/razer_step.h.

Same names, same arguments; torch supplies device memory and the current stream, nothing else.

    y, h = razer.razer_norm(x, weight, eps, residual=h)                                     # between the layers
    q, h = razer.razer_norm_quantize(x, weight, tensor_scale, eps=eps, residual=h)          # ... as 4-bit activations
    ids, weights = razer.razer_moe_route(y, router, top_k)                                  # a layer's experts
    y = razer.razer_moe_experts(y, ids, weights, gate, up, down)
    tokens, logprobs = razer.razer_sample(logits, uniform, temperature, top_k, top_p, min_p)
"""
import ctypes
import struct

import torch

from . import binding as _b

# the argument structures in one pass (see binding._pack_tensor)
_pack_norm = struct.Struct("@PqPqPqPPqPPPiffii4xqqiiiiff").pack
_pack_route = struct.Struct("@PqPPqPPPqiiiiiif4x").pack
_pack_experts = struct.Struct("@PPPqqiiffii").pack
_pack_moe = struct.Struct("@PqPPPqqiiPPP").pack
_pack_sample = struct.Struct("@PqPPPPPPPqqi4x").pack

_i32, _f32, _bf16, _u8 = torch.int32, torch.float32, torch.bfloat16, torch.uint8
_DTYPE = {torch.float32: _b.F32, torch.bfloat16: _b.BF16}
SCORES = {"softmax": 0, "sigmoid": 1}
ACTS = {"silu": 0, "gelu": 1, "relu": 2}


# (a call of a few microseconds on the GPU is bound by what follows here: one launch takes 4 us of host time, torch.empty
# 1.6, torch.empty_like 1.1, current_device() 0.2; a tensor's property 0.03)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _device(t):
    """Index of t's device, which has to be the current one: kernels go to its current stream."""
    at = t.get_device()
    assert at >= 0 and at == _current_device(), "the tensors have to be on the current device"
    return at


def _stream(at):
    return _b._stream() if _b._raw_stream is None else _b._raw_stream(at)


def _rows(t, at):
    """(address, leading dimension) of a 2-D tensor on device `at` whose rows are dense."""
    rows, cols = t.shape
    s0, s1 = t.stride()
    assert t.get_device() == at and (s1 == 1 or cols <= 1)
    return t.data_ptr(), s0 if rows > 1 else max(s0, cols)


def _vector(t, n, dtype, at):
    """Address of a dense tensor of n elements, 0 for None."""
    if t is None:
        return 0
    assert t.dtype is dtype and t.get_device() == at and t.numel() == n and t.is_contiguous()
    return t.data_ptr()


def _workspace(t, at):
    """(address, bytes) of a caller's workspace, or of none."""
    if t is None:
        return None, 0
    assert t.get_device() == at and t.is_contiguous(), "the workspace has to be dense and on the tensors' device"
    return t.data_ptr(), t.numel() * t.element_size()


def _like(t, dtype):
    """A dense tensor of t's shape."""
    if t.dtype is dtype and t.is_contiguous():
        return torch.empty_like(t)
    return torch.empty(t.shape, dtype=dtype, device=t.device)


def _norm(x, weight, eps, residual, sum_out, out, q, block, sv, offset, dtype=None):
    """(out, sum): out is made here where dtype says of what type."""
    L = _b.load_library()
    rows, cols = x.shape
    at = _device(x)
    px, ld_x = _rows(x, at)
    assert weight.get_device() == at and weight.numel() == cols and weight.is_contiguous()
    pr = ld_r = ps = ld_s = po = ld_o = pc = pk = pt = 0
    r_type = o_type = _b.BF16
    if residual is not None:
        assert residual.shape == x.shape
        pr, ld_r = _rows(residual, at)
        r_dtype = residual.dtype
        r_type = _DTYPE[r_dtype]
        if sum_out is None:
            sum_out = _like(residual, r_dtype)
            ps, ld_s = sum_out.data_ptr(), cols
        else:
            assert sum_out.shape == x.shape and sum_out.dtype is r_dtype
            ps, ld_s = _rows(sum_out, at)
    else:
        assert sum_out is None, "without a residual there is no sum"
    if out is not None:
        assert out.shape == x.shape
        po, ld_o = _rows(out, at)
        o_type = _DTYPE[out.dtype]
    elif dtype is not None:
        out = _like(x, dtype)
        po, ld_o, o_type = out.data_ptr(), cols, _DTYPE[dtype]
    if q is not None:
        pc = _vector(q.codes, rows * (cols // 2), _u8, at)
        pk = _vector(q.scales, rows * (cols // block), _u8, at)
        pt = _vector(q.tensor_scale, 1, _f32, at)
    st = L.razer_norm(_pack_norm(px, ld_x, pr, ld_r, ps, ld_s, weight.data_ptr(), po, ld_o, pc, pk, pt, _b.ACT, sv[0], 0.0, block, 0, rows, cols,
                                 _DTYPE[x.dtype], r_type, _DTYPE[weight.dtype], o_type, eps, offset), _stream(at))
    if st != 0:
        raise _b.RazerError(st, "razer_norm")
    return out, sum_out


def razer_norm(x, weight, eps=1e-6, residual=None, dtype=torch.bfloat16, out=None, sum_out=None, offset=0.0):
    """Root-mean-square norm of the rows of h = x + residual: h / sqrt(mean(h^2) + eps) * (offset + weight).

    x, residual [rows][cols] and weight [cols]: float32 or bfloat16 each; rows may be longer.  out: to be written (dtype is
    then its own); it may be x.  sum_out: takes h, of residual's type; it may be residual.
    Returns (y, h), h None without a residual."""
    return _norm(x, weight, eps, residual, sum_out, out, None, 16, (5.0,), offset, dtype)


def razer_norm_quantize(x, weight, tensor_scale, sv=(5.0,), block=16, eps=1e-6, residual=None, sum_out=None, offset=0.0, q=None, out=None):
    """razer_norm with its output as 4-bit activations for a given tensor scale (a float32 device tensor of one element): the
    codes and scale bytes that razer_quantize writes for the float32 output.  q: a RazerTensor to be filled (its block,
    special value and tensor scale count).  out: takes the output itself as well.
    Returns (RazerTensor, h), h None without a residual."""
    rows, cols = x.shape
    if q is None:
        new = lambda n: torch.empty((rows, n), dtype=_u8, device=x.device)
        q = _b.RazerTensor(new(cols // 2), new(cols // block), tensor_scale, rows, cols, _b.ACT, sv, block)
    assert (q.rows, q.cols, q.fmt) == (rows, cols, _b.ACT)
    return q, _norm(x, weight, eps, residual, sum_out, out, q, q.block, q.sv, offset)[1]


def _route(x, router, logits, top_k, score, bias, renormalize, scale, out, workspace):
    L = _b.load_library()
    ref = logits if x is None else x
    dev, tokens = _device(ref), ref.shape[0]
    if x is None:
        experts, hidden, px, ld_x, pw = logits.shape[1], 0, 0, 0, 0
        pl, ld_l = _rows(logits, dev)
    else:
        experts, hidden = router.shape
        assert x.dtype is _bf16 and x.shape[1] == hidden
        px, ld_x = _rows(x, dev)
        pw = _vector(router, experts * hidden, _bf16, dev)
        pl = ld_l = 0
    if out is None:
        ids = torch.empty((tokens, top_k), dtype=_i32, device=ref.device)
        weights = torch.empty_like(ids, dtype=_f32)
    else:
        ids, weights = out
    args = _pack_route(px, ld_x, pw, pl, ld_l, _vector(bias, experts, _f32, dev), _vector(ids, tokens * top_k, _i32, dev), _vector(weights, tokens * top_k, _f32, dev),
                       tokens, hidden, experts, top_k, SCORES[score], 1 if renormalize else 0, _b.F32 if x is not None else _DTYPE[logits.dtype], scale)
    if workspace is None and x is not None:
        need = L.razer_moe_route_workspace_bytes(args)
        if need:
            workspace = torch.empty(need, dtype=_u8, device=ref.device)
    ws, size = _workspace(workspace, dev)
    st = L.razer_moe_route(args, ws, size, _stream(dev))
    if st != 0:
        raise _b.RazerError(st, "razer_moe_route")
    return ids, weights


def razer_moe_route(x, router, top_k, score="softmax", bias=None, renormalize=True, scale=1.0, out=None, workspace=None):
    """The experts of the tokens x [tokens][hidden] (bfloat16; rows may be longer) by router [experts][hidden] (bfloat16).

    score: "softmax" or "sigmoid" of the products.  bias [experts] (float32) counts where experts are chosen, not in their
    weights: with "sigmoid" it is added to the score, with "softmax" to the product (not to the probability).  A NaN is
    chosen last, with weight 0.  renormalize: a token's weights add up to scale.  Returns (ids int32, weights float32), both
    [tokens][top_k], best first; out: the two to be written."""
    return _route(x, router, None, top_k, score, bias, renormalize, scale, out, workspace)


def razer_moe_select(logits, top_k, score="softmax", bias=None, renormalize=True, scale=1.0, out=None):
    """razer_moe_route from given products, logits [tokens][experts] (float32 or bfloat16; rows may be longer)."""
    return _route(None, None, logits, top_k, score, bias, renormalize, scale, out, None)


class RazerExperts:
    """One projection of all experts (razer_experts in the ABI): uint8 codes [experts][rows][cols/2] and scales
    [experts][rows][cols/block], float32 tensor_scales [experts], in the weight format with special values sv.  The object
    describes the tensors it was made of; they are not to be replaced."""

    __slots__ = ("codes", "scales", "tensor_scales", "experts", "rows", "cols", "sv", "block", "device", "_struct", "_address")

    def __init__(self, codes, scales, tensor_scales, sv=(5.0, 8.0), block=16):
        experts, rows, half = codes.shape
        dev = codes.get_device()
        assert dev >= 0
        _vector(codes, experts * rows * half, _u8, dev)
        _vector(scales, experts * rows * (2 * half // block), _u8, dev)
        _vector(tensor_scales, experts, _f32, dev)
        self.codes, self.scales, self.tensor_scales = codes, scales, tensor_scales
        self.experts, self.rows, self.cols, self.sv, self.block, self.device = experts, rows, 2 * half, tuple(sv), block, dev
        self._struct = ctypes.create_string_buffer(_pack_experts(codes.data_ptr(), scales.data_ptr(), tensor_scales.data_ptr(), rows, 2 * half, experts,
                                                                 _b.WEIGHT, sv[0], sv[1], block, 0))
        self._address = ctypes.addressof(self._struct)

    @staticmethod
    def stack(tensors):
        """Copies RazerTensors of equal shape and configuration (one per expert) behind one another."""
        t = tensors[0]
        assert all((x.rows, x.cols, x.fmt, x.sv, x.block, x.layout) == (t.rows, t.cols, _b.WEIGHT, t.sv, t.block, _b.LAYOUT_CANONICAL) for x in tensors)
        return RazerExperts(torch.stack([x.codes for x in tensors]), torch.stack([x.scales for x in tensors]), torch.cat([x.tensor_scale.view(1) for x in tensors]),
                            t.sv, t.block)

    def expert(self, e):
        """Expert e's weights as a RazerTensor on the same memory (what razer_linear and razer_dequant take)."""
        return _b.RazerTensor(self.codes[e], self.scales[e], self.tensor_scales[e:e + 1], self.rows, self.cols, _b.WEIGHT, self.sv, self.block)


def _moe_struct(x, ids, weights, gate, up, down, act, out):
    dev = _device(x)
    tokens, top_k = ids.shape
    assert x.dtype is _bf16 and x.shape[0] == tokens and x.shape[1] == gate.cols
    assert out.dtype is _bf16 and out.shape[0] == tokens and out.shape[1] == down.rows
    assert gate.device == dev and down.device == dev and (up is None or up.device == dev)
    px, ld_x = _rows(x, dev)
    py, ld_y = _rows(out, dev)
    return _pack_moe(px, ld_x, _vector(ids, tokens * top_k, _i32, dev), _vector(weights, tokens * top_k, _f32, dev), py, ld_y, tokens, top_k, ACTS[act],
                     gate._address, 0 if up is None else up._address, down._address)


def razer_moe_workspace_bytes(x, ids, weights, gate, up, down):
    """Bytes of device workspace that razer_moe_experts needs for these sizes; enough for fewer tokens too."""
    y = x if down.rows == gate.cols else x.new_empty((x.shape[0], down.rows))
    return int(_b.load_library().razer_moe_workspace_bytes(_moe_struct(x, ids, weights, gate, up, down, "silu", y)))


def razer_moe_experts(x, ids, weights, gate, up, down, act="silu", out=None, workspace=None):
    """sum_j weights[t][j] * down_e(act(gate_e(x[t])) * up_e(x[t])), e = ids[t][j], for the tokens x [tokens][hidden]
    (bfloat16; rows may be longer).  ids int32 and weights float32 [tokens][top_k] (an id that is no expert: left out);
    gate, up (or None), down: RazerExperts; act: "silu", "gelu" or "relu".  Returns bfloat16 [tokens][down.rows]."""
    L = _b.load_library()
    if out is None:
        out = _like(x, _bf16) if down.rows == x.shape[1] else torch.empty((x.shape[0], down.rows), dtype=_bf16, device=x.device)
    args = _moe_struct(x, ids, weights, gate, up, down, act, out)
    if workspace is None:
        need = L.razer_moe_workspace_bytes(args)
        if need:
            workspace = torch.empty(need, dtype=_u8, device=x.device)
    ws, size = _workspace(workspace, gate.device)
    st = L.razer_moe_experts(args, ws, size, _stream(gate.device))
    if st != 0:
        raise _b.RazerError(st, "razer_moe_experts")
    return out


def razer_sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None, logprobs=None, workspace=None):
    """One token of each row of logits [rows][vocab] (float32 or bfloat16; rows may be longer) by uniform [rows] (float32,
    random numbers in [0, 1)).  temperature, top_p, min_p (float32) and top_k (int32) [rows]: each row's own settings, or
    None.  A row whose logits are all -infinity or NaN gives -1.  Returns (tokens int32, logprobs float32) [rows]."""
    L = _b.load_library()
    rows, vocab = logits.shape
    dev = _device(logits)
    pl, ld = _rows(logits, dev)
    if tokens is None:
        tokens = torch.empty_like(uniform, dtype=_i32)
    if logprobs is None:
        logprobs = torch.empty_like(uniform)
    args = _pack_sample(pl, ld, _vector(uniform, rows, _f32, dev), _vector(temperature, rows, _f32, dev), _vector(top_k, rows, _i32, dev), _vector(top_p, rows, _f32, dev),
                        _vector(min_p, rows, _f32, dev), _vector(tokens, rows, _i32, dev), _vector(logprobs, rows, _f32, dev), rows, vocab, _DTYPE[logits.dtype])
    if workspace is None:
        need = L.razer_sample_workspace_bytes(args)
        if need:
            workspace = torch.empty(need, dtype=_u8, device=logits.device)
    ws, size = _workspace(workspace, dev)
    st = L.razer_sample(args, ws, size, _stream(dev))
    if st != 0:
        raise _b.RazerError(st, "razer_sample")
    return tokens, logprobs


def declare(L):
    """Argument types of the step's entry points."""
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    L.razer_norm.restype = ctypes.c_int
    L.razer_norm.argtypes = [vp, vp]
    for name in ("razer_moe_route", "razer_moe", "razer_sample"):
        f = getattr(L, name + "_workspace_bytes")
        f.restype, f.argtypes = sz, [vp]
    for name in ("razer_moe_route", "razer_moe_experts", "razer_sample"):
        f = getattr(L, name)
        f.restype, f.argtypes = ctypes.c_int, [vp, vp, sz, vp]
