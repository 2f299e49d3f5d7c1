"""The workspace that attention over the cache asks for: one allocation serves every window and every shorter length
(runs without a GPU)."""
import os
import random

import pytest

FAKE = 0x1000


@pytest.fixture(scope="module")
def lib():
    import paper_2501_04052_amd as r
    if not os.path.exists(r.lib_path()):
        from paper_2501_04052_amd import build
        build.build()
    return r.load_library()


def need(lib, heads, dim, page, q_heads, requests, tokens, max_new, max_len, width, window=0):
    from paper_2501_04052_amd import cache as pc
    cache = pc._pack_cache(FAKE, FAKE, FAKE, FAKE, 1 << 20, heads, dim, page)
    row = q_heads * dim
    return lib.razer_attention_workspace_bytes(cache, pc._pack_attention(FAKE, row, FAKE, row, tokens, q_heads, requests, FAKE, FAKE, FAKE, width, width, max_new, max_len,
                                                                         0.1, 0.0, window, 0, 0))


def sizes(rng):
    heads, page = rng.choice([1, 2, 3, 8, 32]), rng.choice([16, 32, 64, 128])
    requests, max_new = rng.choice([1, 1, 2, 7, 64]), rng.choice([1, 2, 5, 9, 33, 128, 512, 2048])
    return dict(heads=heads, dim=rng.choice([64, 128, 192, 256]), page=page, q_heads=heads * rng.choice([1, 4, 7, 8]), requests=requests, tokens=rng.randint(max_new, requests * max_new),
                max_new=max_new, width=(1 << 20) // page)


def test_the_size_without_a_window_serves_every_window(lib):
    one = dict(heads=8, dim=128, page=64, q_heads=8, requests=1, tokens=512, max_new=512, max_len=8256, width=129)
    assert need(lib, window=7488, **one) <= need(lib, **one)
    rng = random.Random(3)
    asked = 0
    for _ in range(4000):
        s = dict(sizes(rng), max_len=int(2 ** rng.uniform(0, 20)))
        bytes_ = need(lib, **s)
        asked += bytes_ > 0
        assert need(lib, window=int(2 ** rng.uniform(0, 20)), **s) <= bytes_, s
    assert asked > 1000


def test_the_size_grows_with_the_length(lib):
    one = dict(heads=8, dim=128, page=64, q_heads=8, requests=1, tokens=512, max_new=512, width=200)
    assert need(lib, max_len=8192, **one) <= need(lib, max_len=8256, **one)
    rng = random.Random(4)
    for _ in range(300):
        s = sizes(rng)
        s["window"] = rng.choice([0, int(2 ** rng.uniform(0, 20))])
        most = need(lib, max_len=0, **s)
        last = 0
        for n in sorted(int(2 ** rng.uniform(0, 20)) for _ in range(30)):
            now = need(lib, max_len=n, **s)
            assert last <= now <= most, (s, n)
            last = now
