"""The cache's C entry points refuse bad arguments before any GPU work, the binding's structures have the header's
layout, and the tests' own oracle agrees with torch's E4M3 casts (runs without a GPU)."""
import ctypes
import os
import re
import struct

import numpy as np
import pytest

import cache_oracle as co

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, ODD = 0x1000, 0x1004


@pytest.fixture(scope="module")
def lib():
    import paper_2501_04052_amd as r
    if not os.path.exists(r.lib_path()):
        from paper_2501_04052_amd import build
        build.build()
    return r.load_library()


def test_header_symbols_are_exported(lib):
    from paper_2501_04052_amd import binding
    text = open(os.path.join(ROOT, "include", "razer_cache.h")).read()
    names = set(re.findall(r"^(?:razer_status|size_t) (razer_[a-z_]+)\(", text, re.M))
    assert names == set(binding.CACHE_EXPORTS)
    for n in names:
        assert hasattr(lib, n), n


def test_header_is_plain_c_and_the_structures_match(tmp_path):
    import subprocess
    from paper_2501_04052_amd import cache
    src = tmp_path / "s.c"
    src.write_text('#include "razer_cache.h"\n#include <stdio.h>\nint main(void){printf("%zu %zu %zu %zu %zu\\n",sizeof(razer_cache),sizeof(razer_attention),'
                   'offsetof(razer_attention,cu),offsetof(razer_attention,scale),offsetof(razer_attention,slopes));return 0;}\n')
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    sizes = [int(x) for x in subprocess.run([str(exe)], capture_output=True, check=True).stdout.split()]
    assert sizes[0] == len(cache._pack_cache(1, 2, 3, 4, 5, 6, 7, 8))
    a = cache._pack_attention(1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 0.5, 0.25, 15, 16, 17)
    assert sizes[1] == len(a)
    assert struct.unpack_from("P", a, sizes[2])[0] == 8 and struct.unpack_from("f", a, sizes[3])[0] == 0.5 and struct.unpack_from("P", a, sizes[4])[0] == 16


def cache_struct(**kw):
    from paper_2501_04052_amd import cache
    d = dict(k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, pages=4, heads=2, dim=128, page=64)
    d.update(kw)
    return cache._pack_cache(d["k"], d["v"], d["ks"], d["vs"], d["pages"], d["heads"], d["dim"], d["page"])


BAD_CACHES = [(dict(page=48), 4), (dict(page=8), 4), (dict(page=256), 4), (dict(dim=96), 4), (dict(dim=0), 4), (dict(dim=512), 4), (dict(pages=0), 2), (dict(pages=1 << 31), 2),
              (dict(heads=0), 2), (dict(heads=-1), 2), (dict(heads=16385), 2), (dict(k=0), 1), (dict(v=0), 1), (dict(ks=0), 1), (dict(vs=0), 1), (dict(k=ODD), 3), (dict(v=ODD), 3)]


def test_plan_refusals(lib):
    def plan(**kw):
        d = dict(lens=FAKE, fresh=FAKE, requests=4, table=FAKE, width=8, ld=8, free=FAKE, count=9, page=16, tokens=5, cu=FAKE, total=FAKE, slots=FAKE, pos=None, req=None, used=FAKE)
        d.update(kw)
        return lib.razer_cache_plan(*d.values(), None)
    for page in (0, 1, 17, 48, 256, -16):
        assert plan(page=page) == 4
    for bad in (dict(requests=-1), dict(width=-1), dict(ld=7), dict(count=-1), dict(tokens=-1), dict(tokens=1 << 31)):
        assert plan(**bad) == 2, bad
    for bad in ("lens", "fresh", "table", "free", "cu", "total", "slots", "used"):
        assert plan(**{bad: None}) == 1, bad


def test_append_refusals(lib):
    def append(cache=None, **kw):
        d = dict(k=FAKE, ld_k=256, v=FAKE, ld_v=256, dtype=1, tokens=3, slots=FAKE)
        d.update(kw)
        return lib.razer_cache_append(cache_struct() if cache is None else cache, *d.values(), None)
    assert lib.razer_cache_append(None, FAKE, 256, FAKE, 256, 1, 3, FAKE, None) == 1
    for kw, want in BAD_CACHES:
        assert append(cache_struct(**kw)) == want, kw
    assert append(dtype=2) == 4 and append(dtype=-1) == 4
    for bad in (dict(tokens=-1), dict(tokens=1 << 24), dict(ld_k=255), dict(ld_v=128)):
        assert append(**bad) == 2, bad
    assert append(cache_struct(heads=64, dim=64), tokens=1 << 20, ld_k=4096, ld_v=4096) == 2
    for bad in ("k", "v", "slots"):
        assert append(**{bad: None}) == 1
    for bad in (dict(k=ODD), dict(v=ODD), dict(ld_k=260), dict(ld_v=257), dict(dtype=0, ld_k=258)):
        assert append(**bad) == 3, bad
    assert append(tokens=0, k=None, v=None, slots=None) == 0


def test_attention_refusals(lib):
    from paper_2501_04052_amd import cache as pc

    def args(**kw):
        d = dict(q=FAKE, ld_q=1024, out=FAKE, ld_out=1024, tokens=3, q_heads=8, requests=2, cu=FAKE, total=FAKE, table=FAKE, ld_table=10, width=10, max_new=0, max_len=0, scale=0.1, cap=0.0,
                 window=0, slopes=0, prefix=0)
        d.update(kw)
        return pc._pack_attention(*d.values())

    def call(cache=None, ws=None, size=0, **kw):
        return lib.razer_cache_attention(cache_struct() if cache is None else cache, args(**kw), ws, size, None)
    assert lib.razer_cache_attention(None, args(), None, 0, None) == 1 and lib.razer_cache_attention(cache_struct(), None, None, 0, None) == 1
    for kw, want in BAD_CACHES:
        assert call(cache_struct(**kw)) == want, kw
    for bad in (dict(tokens=-1), dict(requests=-1), dict(q_heads=0), dict(q_heads=7), dict(width=-1), dict(ld_q=1023), dict(ld_out=8), dict(ld_table=9), dict(tokens=(1 << 24) + 1),
                dict(requests=(1 << 21) + 1)):
        assert call(**bad) == 2, bad
    for bad in (dict(window=-1), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**bad) == 4, bad
    for bad in ("q", "out", "cu", "total", "table"):
        assert call(**{bad: 0}) == 1, bad
    for bad in (dict(q=ODD), dict(out=ODD), dict(ld_q=1028), dict(ld_out=1025)):
        assert call(**bad) == 3, bad
    assert call(tokens=0, q=0, out=0) == 0 and call(requests=0) == 0
    # a few requests over long tables: the keys are split, and the parts meet in a workspace
    long = dict(width=4096, ld_table=4096, requests=1, tokens=1)
    need = lib.razer_attention_workspace_bytes(cache_struct(), args(**long))
    assert need > 0 and lib.razer_attention_workspace_bytes(cache_struct(), args(**dict(long, q_heads=7))) == 0
    assert call(**long) == 5 and call(ws=FAKE, size=need - 1, **long) == 5 and call(ws=ODD, size=need, **long) == 5
    assert lib.razer_attention_workspace_bytes(cache_struct(), args(**dict(long, tokens=0))) == 0


def test_oracle_codes_against_the_library_cast():
    import torch
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, co.VALUES, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 20001), np.linspace(-0.05, 0.05, 20001), (co.VALUES[:126] + co.VALUES[1:127]) / 2]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(co.encode(x), want)
    for a, b in ((0.0, 77), (448.0, 127), (448.1, 128), (224.0, 126), (1e-40, 77), (3e38, 177), (1.0, 119)):
        assert co.exponent(a) == b, a


def test_oracle_attention_of_one_key_is_its_value():
    c = co.Cache(1, 1, 64, 16)
    v = np.arange(64, dtype=np.float32).reshape(1, 1, 64)
    c.append(v, v, np.array([0]))
    out, bound = co.attention(c, np.ones((1, 2, 64), np.float32), [0, 1], [1], np.array([[0]]), 0.1)
    held = c.keys_values([0], 0)[1][0]
    assert np.array_equal(out[0, 0], held) and np.allclose(held, v[0, 0], rtol=2.0 ** -4) and (bound >= 2.0 ** -9 * np.abs(out)).all()
