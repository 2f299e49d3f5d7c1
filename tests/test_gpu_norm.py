"""razer_norm on the GPU: values against the formula in 64 bits within the roundings that the header names, codes to the bit
against the encoder's oracle on the same float32 output."""
import itertools

import numpy as np
import pytest
import torch

import paper_2501_04052_amd as razer
import step_oracle as so

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "f32": torch.float32}


def inputs(rows, cols, seed, x="bf16", residual="bf16", weight="bf16", pad=0):
    rng = np.random.default_rng(seed)

    def make(shape, dtype, scale=1.0):
        a = (rng.standard_normal(shape) * scale).astype(np.float32)
        return so.bf16(a) if dtype == "bf16" else a
    host = [make((rows, cols), x, 2.0), None if residual == "none" else make((rows, cols), residual, 5.0), make(cols, weight)]

    def up(a, dtype):
        if a is None:
            return None
        t = torch.from_numpy(a).cuda().to(T[dtype])
        if pad and a.ndim == 2:
            wide = torch.full((rows, cols + pad), float("nan"), device="cuda", dtype=T[dtype])
            wide[:, :cols] = t
            return wide[:, :cols]
        return t
    return host, [up(host[0], x), up(host[1], residual), up(host[2], weight)]


def check(got, want, dtype):
    got = got.double().cpu().numpy()
    # h one rounding, its mean as many again, root, two products and 1 + w one each
    bound = (7 * so.U32 + (so.U16 if dtype == "bf16" else so.U32)) * np.abs(want) * (1 + 1e-3) + 1e-38
    bad = np.abs(got - want) > bound
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])


SIZES = [(1, 1), (3, 7), (1, 63), (2, 64), (5, 65), (1, 1000), (7, 1024), (3, 1032), (2, 4096), (1, 8191), (2, 8192), (3, 8200), (1, 16384), (2, 32767), (2, 32768), (70, 96)]


@pytest.mark.parametrize("rows,cols", SIZES)
def test_values(rows, cols):
    for i, (x, residual, weight, out) in enumerate(itertools.product(("bf16", "f32"), ("none", "bf16", "f32"), ("bf16", "f32"), ("bf16", "f32"))):
        pad = (0, 8, 3)[i % 3]
        host, dev = inputs(rows, cols, 10 * cols + i, x, residual, weight, pad)
        offset = float(i % 2)
        want, h = so.norm(host[0], host[2], 1e-5, host[1], offset)
        y, total = razer.razer_norm(dev[0], dev[2], eps=1e-5, residual=dev[1], dtype=T[out], offset=offset)
        check(y, want, out)
        if residual == "none":
            assert total is None
        else:
            h32 = host[0] + host[1]
            assert np.array_equal(total.float().cpu().numpy(), so.bf16(h32) if residual == "bf16" else h32)


def test_rows_behind_and_between_stay_as_they_were():
    for cols, pad in ((64, 8), (61, 3)):
        host, dev = inputs(5, cols, 3)
        buf = torch.full((7, cols + pad), 9.0, device="cuda")
        total = torch.full((7, cols + pad), 8.0, device="cuda", dtype=torch.bfloat16)
        razer.razer_norm(dev[0], dev[2], residual=dev[1], out=buf[1:6, :cols], sum_out=total[1:6, :cols])
        for t, v in ((buf, 9.0), (total, 8.0)):
            assert (t[0] == v).all() and (t[6] == v).all() and (t[:, cols:] == v).all() and not (t[1:6, :cols] == v).all()


def test_in_place():
    for cols in (4096, 999):
        for dtype in ("bf16", "f32"):
            host, dev = inputs(4, cols, 5, dtype, dtype, "f32")
            y, total = razer.razer_norm(dev[0], dev[2], residual=dev[1], dtype=T[dtype])
            razer.razer_norm(dev[0], dev[2], residual=dev[1], out=dev[0], sum_out=dev[1])
            assert torch.equal(dev[0], y) and torch.equal(dev[1], total)


def test_zero_rows_large_and_small_values():
    w = torch.ones(256, device="cuda")
    x = torch.zeros(6, 256, device="cuda")
    x[1] = 1e-30
    x[2] = 1e25
    x[3, 0] = 3e38
    x[4, 7] = float("inf")
    x[5, 9] = float("nan")
    y, _ = razer.razer_norm(x, w, eps=0.0, dtype=torch.float32)
    assert torch.isnan(y[0]).all()                      # 0 / 0, as the formula has it
    y, _ = razer.razer_norm(x, w, eps=1e-6, dtype=torch.float32)
    want, _ = so.norm(x[:4].cpu().numpy(), w.cpu().numpy(), 1e-6)
    assert (y[0] == 0).all()
    check(y[:4], want, "f32")
    assert torch.isnan(y[4, 7]) and (y[4, :7] == 0).all() and torch.isnan(y[5]).all()


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(1, 128), (3, 256), (2, 4096), (5, 4224), (1, 8192), (2, 16512), (1, 32768), (33, 384)])
def test_codes(oracle, rows, cols, block):
    for i, (x, residual, sv) in enumerate((("bf16", "none", 5.0), ("bf16", "bf16", 5.0), ("f32", "f32", 7.5))):
        host, dev = inputs(rows, cols, cols + block + i, x, residual, "f32" if i else "bf16", 8 * i)
        y32, _ = so.norm_steps(host[0], host[2], 1e-6, host[1])
        ts = np.float32(np.abs(y32).max() / 2688.0 * (1.0, 0.6, 3.0)[i])
        q, total = razer.razer_norm_quantize(dev[0], dev[2], torch.tensor([ts], device="cuda"), sv=(sv,), block=block, residual=dev[1])
        codes, scales, _ = oracle.quantize(oracle.ACT, y32, sv=(sv, 0.0), given_tensor_scale=float(ts), block=block)
        assert np.array_equal(q.scales.cpu().numpy(), scales) and np.array_equal(q.codes.cpu().numpy(), codes)
        # and the same as the two calls
        y, _ = razer.razer_norm(dev[0], dev[2], residual=dev[1], dtype=torch.float32)
        assert np.array_equal(y.cpu().numpy(), y32)
        two = razer.razer_quantize(y, razer.ACT, (sv,), tensor_scale=q.tensor_scale, block=block)
        assert torch.equal(two.codes, q.codes) and torch.equal(two.scales, q.scales)


def test_codes_and_values_of_one_call_feed_the_linear_layer():
    host, dev = inputs(7, 512, 1)
    w = razer.razer_quantize(torch.randn(96, 512, device="cuda") * 0.05, razer.WEIGHT, (5.0, 8.0))
    ts = torch.tensor([12.0 / 2688], device="cuda")
    out = torch.empty(7, 512, device="cuda")
    q, _ = razer.razer_norm_quantize(dev[0], dev[2], ts, residual=dev[1], out=out)
    y = razer.razer_linear(w, q).double()
    want = razer.razer_dequant(q, torch.float32).double() @ razer.razer_dequant(w, torch.float32).double().t()
    assert float((y - want).abs().max()) <= 8e-3 * float(want.abs().max())
    ref, _ = razer.razer_norm(dev[0], dev[2], residual=dev[1], dtype=torch.float32)
    assert torch.equal(out, ref)


def test_on_another_stream_and_many_rows():
    host, dev = inputs(5000, 128, 2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y, total = razer.razer_norm(dev[0], dev[2], residual=dev[1])
    s.synchronize()
    want, _ = so.norm(host[0], host[2], 1e-6, host[1])
    check(y, want, "bf16")


def test_refusals_through_the_binding():
    x, w = torch.zeros(2, 64, device="cuda"), torch.zeros(64, device="cuda")
    with pytest.raises(AssertionError):
        razer.razer_norm(x, w, sum_out=x)
    with pytest.raises(AssertionError):
        razer.razer_norm(x, w.cpu())
    with pytest.raises(AssertionError):
        razer.razer_norm(x, w, residual=x[:1])
    with pytest.raises(razer.RazerError):
        razer.razer_norm(x, w, eps=-1.0)
    with pytest.raises(razer.RazerError):
        razer.razer_norm_quantize(torch.zeros(2, 48, device="cuda"), w[:48], w[:1])
