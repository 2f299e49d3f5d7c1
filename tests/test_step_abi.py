"""The C entry points of include/razer_step.h refuse bad arguments before any GPU work, the binding's structures have the
header's layout, workspaces grow with the number of tokens, and the tests' own oracle agrees with torch (runs without a GPU)."""
import os
import random
import re
import struct

import numpy as np
import pytest
import torch

import step_oracle as so

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, ODD = 0x1000, 0x1004
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    import paper_2501_04052_amd as r
    if not os.path.exists(r.lib_path()):
        from paper_2501_04052_amd import build
        build.build()
    return r.load_library()


def test_header_symbols_are_exported(lib):
    from paper_2501_04052_amd import binding
    text = open(os.path.join(ROOT, "include", "razer_step.h")).read()
    names = set(re.findall(r"^(?:razer_status|size_t) (razer_[a-z_]+)\(", text, re.M))
    assert names == set(binding.STEP_EXPORTS)
    for n in names:
        assert hasattr(lib, n), n


def test_header_is_plain_c_and_the_structures_match(tmp_path):
    import subprocess
    from paper_2501_04052_amd import step
    fields = {"razer_norm_args": ["cfg", "rows", "x_dtype", "weight_offset"], "razer_moe_route_args": ["tokens", "hidden", "logits_dtype", "scale"],
              "razer_experts": ["tensor_scales", "experts", "cfg"], "razer_moe_args": ["ld_y", "top_k", "down"], "razer_sample_args": ["min_p", "logprobs", "vocab", "dtype"]}
    src = tmp_path / "s.c"
    src.write_text('#include "razer_step.h"\n#include <stdio.h>\nint main(void){' + "".join(
        'printf("%%zu%s\\n",sizeof(%s)%s);' % (" %zu" * len(f), t, "".join(",offsetof(%s,%s)" % (t, x) for x in f)) for t, f in fields.items()) + 'return 0;}\n')
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [[int(x) for x in line.split()] for line in subprocess.run([str(exe)], capture_output=True, check=True).stdout.splitlines()]
    at = lambda fmt, data, off: struct.unpack_from(fmt, data, off)[0]
    a, (size, cfg, rows, xd, off) = step._pack_norm(*range(1, 13), 13, 14.0, 15.0, 16, 17, 18, 19, 20, 21, 22, 23, 24.0, 25.0), got[0]
    assert len(a) == size and at("i", a, cfg) == 13 and at("q", a, rows) == 18 and at("i", a, xd) == 20 and at("f", a, off) == 25.0
    a, (size, tokens, hidden, ld, scale) = step._pack_route(*range(1, 16), 16.0), got[1]
    assert len(a) == size and at("q", a, tokens) == 9 and at("i", a, hidden) == 10 and at("i", a, ld) == 15 and at("f", a, scale) == 16.0
    a, (size, ts, experts, cfg) = step._pack_experts(1, 2, 3, 4, 5, 6, 7, 8.0, 9.0, 10, 11), got[2]
    assert len(a) == size and at("P", a, ts) == 3 and at("i", a, experts) == 6 and at("i", a, cfg) == 7
    a, (size, ld, k, down) = step._pack_moe(*range(1, 13)), got[3]
    assert len(a) == size and at("q", a, ld) == 6 and at("i", a, k) == 8 and at("P", a, down) == 12
    a, (size, minp, lp, vocab, dtype) = step._pack_sample(*range(1, 13)), got[4]
    assert len(a) == size and at("P", a, minp) == 7 and at("P", a, lp) == 9 and at("q", a, vocab) == 11 and at("i", a, dtype) == 12


def test_norm_refusals(lib):
    from paper_2501_04052_amd import step

    def norm(**kw):
        d = dict(x=FAKE, ld_x=64, res=FAKE, ld_r=64, sum=FAKE, ld_s=64, w=FAKE, out=FAKE, ld_o=64, codes=0, scales=0, ts=0, fmt=1, sv0=5.0, sv1=0.0, block=16, layout=0, rows=3, cols=64,
                 xt=1, rt=1, wt=1, ot=1, eps=1e-6, offset=0.0)
        d.update(kw)
        return lib.razer_norm(step._pack_norm(*d.values()), None)
    q = dict(codes=FAKE, scales=FAKE, ts=FAKE)
    assert lib.razer_norm(None, None) == 1
    for bad in (dict(xt=2), dict(rt=-1), dict(wt=5), dict(ot=2), dict(eps=-1e-6), dict(eps=NAN), dict(q, fmt=0), dict(q, fmt=2, block=128), dict(q, sv0=6.0), dict(q, block=24), dict(q, layout=1)):
        assert norm(**bad) == 4, bad
    for bad in (dict(rows=-1), dict(rows=1 << 22), dict(cols=-1), dict(cols=32769, ld_x=40000, ld_r=40000, ld_s=40000, ld_o=40000), dict(ld_x=63), dict(ld_r=63), dict(ld_s=63), dict(ld_o=0),
                dict(q, cols=48), dict(q, cols=32, block=64)):
        assert norm(**bad) == 2, bad
    for bad in (dict(x=0), dict(w=0), dict(out=0, sum=0), dict(res=0), dict(q, scales=0), dict(q, ts=0)):
        assert norm(**bad) == 1, bad
    for bad in (dict(x=0x1001), dict(xt=0, x=0x1002), dict(w=0x1001), dict(res=0x1001), dict(sum=0x1001), dict(out=0x1001), dict(q, x=ODD), dict(q, ld_x=68), dict(q, codes=ODD), dict(q, scales=ODD),
                dict(q, ts=0x1002)):
        assert norm(**bad) == 3, bad
    assert norm(rows=0, x=0) == 0 and norm(cols=0, out=0) == 0


def test_route_refusals(lib):
    from paper_2501_04052_amd import step

    def args(**kw):
        d = dict(x=FAKE, ld_x=64, router=FAKE, logits=0, ld_l=0, bias=0, ids=FAKE, weights=FAKE, tokens=3, hidden=64, experts=8, top_k=2, score=0, renorm=1, lt=0, scale=1.0)
        d.update(kw)
        return step._pack_route(*d.values())

    def route(ws=FAKE, size=1 << 30, **kw):
        return lib.razer_moe_route(args(**kw), ws, size, None)
    given = dict(x=0, logits=FAKE, ld_l=8)
    assert lib.razer_moe_route(None, FAKE, 1 << 30, None) == 1 and lib.razer_moe_route_workspace_bytes(None) == 0
    for bad in (dict(score=2), dict(score=-1), dict(given, lt=2)):
        assert route(**bad) == 4, bad
    for bad in (dict(tokens=-1), dict(tokens=(1 << 20) + 1), dict(experts=0), dict(experts=513), dict(top_k=0), dict(top_k=9), dict(experts=64, top_k=33), dict(hidden=0), dict(hidden=48), dict(ld_x=56),
                dict(given, ld_l=7)):
        assert route(**bad) == 2, bad
    for bad in (dict(router=0), dict(ids=0), dict(weights=0), dict(given, logits=0)):
        assert route(**bad) == 1, bad
    for bad in (dict(x=ODD), dict(router=ODD), dict(ld_x=68), dict(ids=0x1002), dict(weights=0x1001), dict(bias=0x1001), dict(given, logits=0x1002)):
        assert route(**bad) == 3, bad
    need = lib.razer_moe_route_workspace_bytes(args())
    assert need > 0 and route(ws=None) == 5 and route(ws=ODD) == 5 and route(size=need - 1) == 5
    assert lib.razer_moe_route_workspace_bytes(args(**given)) == 0 and route(tokens=0, x=FAKE, ids=0) == 0


def experts_struct(**kw):
    import ctypes
    from paper_2501_04052_amd import step
    d = dict(codes=FAKE, scales=FAKE, ts=FAKE, rows=64, cols=64, experts=8, fmt=0, sv0=5.0, sv1=8.0, block=16, layout=0)
    d.update(kw)
    return ctypes.create_string_buffer(step._pack_experts(*d.values()))


def moe_args(gate=None, up=None, down=None, no_up=False, **kw):
    import ctypes
    from paper_2501_04052_amd import step
    g, u, w = experts_struct(**(gate or {})), experts_struct(**(up or gate or {})), experts_struct(**(down or {}))
    d = dict(x=FAKE, ld_x=64, ids=FAKE, weights=FAKE, y=FAKE, ld_y=64, tokens=3, top_k=2, act=0, gate=ctypes.addressof(g), up=0 if no_up else ctypes.addressof(u), down=ctypes.addressof(w))
    d.update(kw)
    return step._pack_moe(*d.values()), (g, u, w)


def test_experts_refusals(lib):
    def moe(ws=FAKE, size=1 << 40, **kw):
        a, keep = moe_args(**kw)
        return lib.razer_moe_experts(a, ws, size, None)
    assert lib.razer_moe_experts(None, FAKE, 1 << 40, None) == 1 and lib.razer_moe_workspace_bytes(None) == 0
    for bad in (dict(act=3), dict(act=-1), dict(gate=dict(fmt=1)), dict(down=dict(fmt=2, block=128)), dict(gate=dict(layout=1)), dict(gate=dict(block=20)), dict(down=dict(sv0=6.0)),
                dict(up=dict(sv1=7.0)), dict(up=dict(block=32)), dict(up=dict(fmt=1))):
        assert moe(**bad) == 4, bad
    for bad in (dict(gate=dict(rows=48)), dict(gate=dict(rows=0)), dict(gate=dict(cols=48)), dict(gate=dict(cols=32, block=64)), dict(gate=dict(experts=0)), dict(gate=dict(experts=1025)),
                dict(gate=dict(rows=1 << 21)), dict(down=dict(cols=32)), dict(down=dict(experts=7)), dict(up=dict(rows=32)), dict(up=dict(cols=32)), dict(up=dict(experts=9)),
                dict(tokens=-1), dict(top_k=0), dict(top_k=33), dict(tokens=(1 << 19) + 1), dict(gate=dict(rows=2048), down=dict(cols=2048), tokens=1 << 19), dict(ld_x=56), dict(ld_y=56), dict(ld_x=1 << 30)):
        assert moe(**bad) == 2, bad
    for bad in (dict(gate=dict(codes=0)), dict(up=dict(scales=0)), dict(down=dict(ts=0)), dict(gate=None, x=0), dict(ids=0), dict(weights=0), dict(y=0), dict(down=None) | dict(y=0)):
        assert moe(**bad) == 1, bad
    from paper_2501_04052_amd import step
    a, keep = moe_args()
    import ctypes
    assert lib.razer_moe_experts(step._pack_moe(FAKE, 64, FAKE, FAKE, FAKE, 64, 3, 2, 0, 0, 0, ctypes.addressof(keep[2])), FAKE, 1 << 40, None) == 1
    for bad in (dict(x=ODD), dict(y=ODD), dict(ld_x=68), dict(ld_y=68), dict(ids=0x1002), dict(weights=0x1002), dict(gate=dict(codes=ODD)), dict(down=dict(scales=ODD)), dict(down=dict(ts=0x1002))):
        assert moe(**bad) == 3, bad
    need = lib.razer_moe_workspace_bytes(a)
    assert need > 0 and moe(ws=None) == 5 and moe(ws=ODD) == 5 and moe(size=need - 1) == 5
    assert moe(tokens=0, x=0) == 0


def test_experts_workspace_grows_with_the_tokens(lib):
    rng = random.Random(5)
    for _ in range(60):
        k, e, rows, cols = rng.randint(1, 8), rng.choice([1, 2, 8, 64, 1000]), 32 * rng.randint(1, 40), 32 * rng.randint(1, 40)
        last = 0
        for tokens in [*range(1, 130), 500, 501, 5000, 100000]:
            a, keep = moe_args(gate=dict(rows=cols, cols=rows, experts=e), down=dict(rows=rows, cols=cols, experts=e), tokens=tokens, top_k=k)
            need = lib.razer_moe_workspace_bytes(a)
            assert need >= last > -1 and need > 0, (k, e, rows, cols, tokens)
            last = need


def test_sample_refusals(lib):
    from paper_2501_04052_amd import step

    def args(**kw):
        d = dict(logits=FAKE, ld=100, uniform=FAKE, t=0, k=0, p=0, m=0, tokens=FAKE, logprobs=0, rows=3, vocab=100, dtype=0)
        d.update(kw)
        return step._pack_sample(*d.values())
    sample = lambda **kw: lib.razer_sample(args(**kw), FAKE, 1 << 40, None)
    assert lib.razer_sample(None, None, 0, None) == 1 and lib.razer_sample_workspace_bytes(None) == 0
    assert sample(dtype=2) == 4 and sample(dtype=-1) == 4
    for bad in (dict(rows=-1), dict(rows=1 << 22), dict(vocab=0), dict(vocab=(1 << 24) + 1, ld=1 << 25), dict(ld=99)):
        assert sample(**bad) == 2, bad
    for bad in ("logits", "uniform", "tokens"):
        assert sample(**{bad: 0}) == 1, bad
    for bad in (dict(logits=0x1002), dict(dtype=1, logits=0x1001), dict(uniform=0x1002), dict(t=0x1001), dict(k=0x1002), dict(p=0x1001), dict(m=0x1003), dict(tokens=0x1002), dict(logprobs=0x1002)):
        assert sample(**bad) == 3, bad
    assert sample(rows=0, logits=0) == 0
    for rows in (1, 2, 40, 300):
        for vocab in (5, 5000, 128000):
            need = lib.razer_sample_workspace_bytes(args(rows=rows, vocab=vocab, ld=vocab))
            if need:
                for ws, size in ((None, need), (ODD, need), (FAKE, need - 1)):
                    assert lib.razer_sample(args(rows=rows, vocab=vocab, ld=vocab), ws, size, None) == 5


def test_binding_refuses_tensors_that_are_not_on_the_current_device():
    from paper_2501_04052_amd import step
    with pytest.raises(AssertionError):
        step._rows(torch.zeros(2, 3).t().contiguous().t(), -1)
    with pytest.raises(AssertionError):
        step._vector(torch.zeros(4, dtype=torch.float64), 4, torch.float32, -1)
    with pytest.raises(AssertionError):
        step._device(torch.zeros(4))


# ---- the oracle itself ------------------------------------------------------------------------------------------

def test_oracle_bf16():
    x = np.concatenate([np.random.default_rng(0).standard_normal(10000), [0.0, 1.00390625, 1.01171875, 3e38]]).astype(np.float32)
    assert np.array_equal(so.bf16(x), torch.from_numpy(x).bfloat16().float().numpy())


def test_oracle_norm_and_experts_against_torch():
    g = torch.Generator().manual_seed(1)
    x, r, w = (torch.randn(s, generator=g) for s in ((5, 96), (5, 96), (96,)))
    y, h = so.norm(x.numpy(), w.numpy(), 1e-3, r.numpy(), offset=1.0)
    want = torch.nn.functional.rms_norm((x.double() + r.double()), (96,), w.double() + 1.0, 1e-3)
    assert np.allclose(y, want.numpy(), rtol=1e-12)
    steps, _ = so.norm_steps(x.numpy(), w.numpy(), 1e-3, r.numpy(), offset=1.0)
    assert (np.abs(steps - y) <= 8 * so.U32 * np.abs(y)).all()
    gate, up, down = ([torch.randn(s, generator=g).double().numpy() for _ in range(3)] for s in ((64, 96), (64, 96), (32, 64)))
    ids, ws = np.array([[0, 2], [1, 1], [-1, 2], [5, -7], [2, 0]]), np.abs(np.random.default_rng(2).standard_normal((5, 2)))
    y, bound = so.experts(x.numpy(), ids, ws, gate, up, down, "gelu")
    t = lambda m: torch.from_numpy(m)
    f = lambda e, v: (torch.nn.functional.gelu(t(gate[e]) @ v, approximate="tanh") * (t(up[e]) @ v)).numpy()
    v = x.double()
    assert np.allclose(y[0], ws[0, 0] * (down[0] @ f(0, v[0])) + ws[0, 1] * (down[2] @ f(2, v[0])))
    assert np.allclose(y[1], ws[1].sum() * (down[1] @ f(1, v[1]))) and not y[3].any() and (bound > 0).all()


def test_oracle_route_and_sample_small():
    ids, w, gap = so.route(np.array([[1.0, 3.0, 3.0, np.nan]]), 3)
    assert ids.tolist() == [[1, 2, 0]] and np.isclose(w[0, 0], w[0, 1]) and np.isclose(w.sum(), 1.0) and gap[0] == 0.0
    l = np.log(np.array([[0.1, 0.4, 0.2, 0.3]], np.float32))
    for u, want in ((0.0, 1), (0.39, 1), (0.41, 3), (0.69, 3), (0.71, 2), (0.95, 0)):
        assert so.sample(l, [u])[0][0] == want
    assert so.sample(l, [0.99], top_k=[2])[0][0] == 3 and so.sample(l, [0.99], top_p=[0.65])[0][0] == 3 and so.sample(l, [0.99], top_p=[0.75])[0][0] == 2
    assert so.sample(l, [0.99], min_p=[0.6])[0][0] == 3 and so.sample(l, [0.99], temperature=[0.0])[0][0] == 1
    assert so.sample(np.full((1, 3), -np.inf, np.float32), [0.5])[0][0] == -1
