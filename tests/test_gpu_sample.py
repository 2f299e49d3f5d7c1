"""razer_sample on the GPU against its definition in 64 bits: the tokens exactly (no border of these rows lies within 1e-9 of
where it would choose another one), the logarithms within fp32."""
import numpy as np
import pytest
import torch

import paper_2501_04052_amd as razer
import step_oracle as so

pytestmark = pytest.mark.gpu


def up(a, dtype=torch.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def check(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, sure=True):
    """logits: a device tensor"""
    f32 = lambda a: None if a is None else np.asarray(a, np.float32)
    u, t, p, m = f32(uniform), f32(temperature), f32(top_p), f32(min_p)
    want, logp, margin = so.sample(logits.float().cpu().numpy(), u, t, top_k, p, m, torch.finfo(logits.dtype).max)
    tok, lp = razer.razer_sample(logits, up(u), up(t), None if top_k is None else up(np.asarray(top_k), torch.int32), up(p), up(m))
    tok, lp = tok.cpu().numpy(), lp.double().cpu().numpy()
    if sure:
        assert (margin > 1e-9).all()
    bad = tok != want
    assert not bad.any(), (np.flatnonzero(bad)[:5], tok[bad][:5], want[bad][:5])
    fin = np.isfinite(logp)
    assert np.array_equal(fin, np.isfinite(lp)) and np.allclose(lp[fin], logp[fin], rtol=2 * so.U32, atol=1e-9)
    return tok


def rows_of(rng, rows, vocab, dtype, pad=0):
    x = rng.standard_normal((rows, vocab)) * 2 + 6 * rng.random((rows, vocab)) ** 100
    x[:, 3::97] = -np.inf
    wide = torch.full((rows, vocab + pad), float("inf"), dtype=dtype, device="cuda")
    wide[:, :vocab] = up(x).to(dtype)
    return wide[:, :vocab]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,pad", [(1, 1, 0), (1, 2, 0), (4, 63, 1), (5, 64, 0), (3, 1000, 5), (2, 1025, 0), (9, 4096, 0), (2, 32000, 0), (40, 5003, 0), (3, 131072, 3), (1, 200001, 0), (300, 700, 1)])
def test_sample(rows, vocab, pad, dtype):
    rng = np.random.default_rng(rows * vocab)
    l = rows_of(rng, rows, vocab, dtype, pad)
    u = rng.random(rows)
    t = rng.uniform(0.4, 1.6, rows)
    k = rng.integers(1, max(2, min(vocab, 2000)), rows)
    check(l, u)
    check(l, u, t)
    check(l, u, t, top_k=k)
    check(l, u, t, top_p=rng.uniform(0.05, 0.999, rows))
    check(l, u, t, min_p=rng.uniform(0.0005, 0.4, rows))
    check(l, u, t, k, rng.uniform(0.3, 0.999, rows), rng.uniform(0.001, 0.2, rows))
    # all settings in one call, some off
    t2 = np.where(np.arange(rows) % 4 == 1, 0.0, t)
    check(l, u, t2, np.where(np.arange(rows) % 3 == 0, 0, k), np.where(np.arange(rows) % 5 == 0, 1.0, 0.8), np.where(np.arange(rows) % 2 == 0, 0.0, 0.05))


def test_greedy_takes_the_first_of_the_largest():
    for dtype in (torch.float32, torch.bfloat16):
        l = torch.zeros(3, 3000, device="cuda", dtype=dtype)
        l[0, [2999, 77, 1500]] = 4.0
        l[1] = -7.0
        l[2, 64:] = 1.0
        tok, lp = razer.razer_sample(l, up(np.full(3, 0.99)), up(np.zeros(3)))
        assert tok.tolist() == [77, 0, 64] and (lp == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [8, 1000, 5000, 70000])
def test_equal_logits(vocab, dtype):
    """All weights are one: borders are counts."""
    l = torch.full((7, vocab), -2.5, device="cuda", dtype=dtype)
    u = np.array([0.0, 0.25, 0.5, 0.75, 0.999, 0.25, 0.875], np.float32)
    assert check(l, u, sure=False).tolist() == [int(np.floor(v * vocab)) for v in u.astype(np.float64)]
    assert check(l, u, top_k=np.full(7, vocab // 4), sure=False).tolist() == [int(np.floor(float(v) * (vocab // 4))) for v in u]
    assert check(l, u, top_p=np.full(7, 0.5), sure=False).tolist() == [int(np.floor(float(v) * (vocab // 2))) for v in u]
    check(l, u, min_p=np.full(7, 1.0), sure=False)
    check(l, u, top_k=np.full(7, 5), top_p=np.full(7, 0.375), sure=False)     # 1.875 of 5 ones: two stay


def test_borders_between_equal_logits():
    """Borders of top_k and top_p inside runs of equal logits: the lower indexes stay."""
    rng = np.random.default_rng(8)
    for vocab in (50, 3000, 40000):
        l = up(rng.integers(-3, 4, (24, vocab)).astype(np.float32))
        u = rng.random(24)
        for k in (1, 2, vocab // 9, vocab // 2, vocab - 1, vocab, vocab + 1):
            check(l, u, top_k=np.full(24, k))
            check(l, u, rng.uniform(0.5, 2, 24), top_k=np.full(24, k), top_p=rng.uniform(0.1, 0.99, 24), min_p=rng.uniform(0.0001, 0.9, 24))


def test_random_numbers_at_and_past_the_ends():
    rng = np.random.default_rng(9)
    l = rows_of(rng, 6, 2000, torch.float32)
    nan = float("nan")
    u = np.array([0.0, 1.0, 2.0, -1.0, nan, np.nextafter(np.float32(1), np.float32(0))], np.float32)
    check(l, u, top_k=np.full(6, 30), sure=False)
    check(l, u, top_p=np.full(6, 0.7), sure=False)


def test_settings_at_and_past_the_ends():
    rng = np.random.default_rng(10)
    l = rows_of(rng, 8, 2500, torch.bfloat16)
    u, nan, inf = rng.random(8), float("nan"), float("inf")
    check(l, u, top_p=np.array([0.0, -1.0, 1.0, 2.0, nan, 1e-9, 0.5, 1.0]), sure=False)
    check(l, u, min_p=np.array([0.0, -1.0, 1.0, 2.0, nan, 1e-9, 0.5, 1e-30]), sure=False)
    check(l, u, top_k=np.array([0, -5, 1, 2500, 2499, 2 ** 31 - 1, -2 ** 31, 2]), sure=False)
    check(l, u, np.array([nan, -1.0, 0.0, 1e-30, 1e-3, 1e3, 1e30, inf]), sure=False)
    check(l, u, np.array([nan, -1.0, 0.0, 1e-30, 1e-3, 1e3, 1e30, inf]), np.full(8, 50), np.full(8, 0.9), np.full(8, 0.5), sure=False)


def test_infinities_nan_and_rows_without_tokens():
    inf, nan = float("inf"), float("nan")
    l = torch.full((9, 300), -inf, device="cuda")
    l[1] = nan
    l[2, 250] = -3e38
    l[3, 5:9] = torch.tensor([nan, 1.0, nan, 1.0], device="cuda")
    l[4, [7, 100]] = inf
    l[4, 8] = 3e38
    l[5, ::2] = 0.0
    l[5, 1::4] = -0.0
    l[6] = 1e-40
    l[7, 3] = -inf
    l[7, 299] = 1e-45
    l[8] = torch.arange(300, device="cuda") * -1e36
    for dtype in (torch.float32, torch.bfloat16):
        for u in (0.0, 0.3, 0.6, 0.99):
            tok = check(l.to(dtype), np.full(9, u), sure=False)
            assert tok[0] == tok[1] == -1 and tok[2] == 250 and tok[3] in (6, 8) and tok[4] in (7, 100)
            check(l.to(dtype), np.full(9, u), np.full(9, 0.7), np.full(9, 4), np.full(9, 0.8), np.full(9, 0.1), sure=False)


def test_one_row_does_not_touch_another_and_logprobs_are_optional():
    from paper_2501_04052_amd import binding as b, step
    rng = np.random.default_rng(12)
    l = rows_of(rng, 5, 3001, torch.float32)
    u = up(rng.random(5))
    tok, lp = razer.razer_sample(l, u)
    out = torch.full((7,), -9, dtype=torch.int32, device="cuda")
    need = razer.load_library().razer_sample_workspace_bytes(step._pack_sample(l.data_ptr(), l.stride(0), u.data_ptr(), 0, 0, 0, 0, out[1:].data_ptr(), 0, 5, 3001, b.F32))
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    assert razer.load_library().razer_sample(step._pack_sample(l.data_ptr(), l.stride(0), u.data_ptr(), 0, 0, 0, 0, out[1:].data_ptr(), 0, 5, 3001, b.F32), ws.data_ptr(), ws.numel(), b._stream()) == 0
    assert out[0] == -9 and out[6] == -9 and torch.equal(out[1:6], tok)
    for r in range(5):
        one = razer.razer_sample(l[r:r + 1], u[r:r + 1])
        assert one[0][0] == tok[r] and one[1][0] == lp[r]


def test_frequencies_follow_the_weights():
    """65536 evenly spaced random numbers count each token floor or ceil of its share times their number."""
    rng = np.random.default_rng(13)
    n = 65536
    l = rng.standard_normal(40).astype(np.float32)
    tok, lp = razer.razer_sample(up(np.tile(l, (n, 1))), up((np.arange(n) + 0.5) / n))
    share = np.exp(l.astype(np.float64) - l.max())
    share /= share.sum()
    count = np.bincount(tok.cpu().numpy(), minlength=40)
    assert (np.abs(count - share * n) <= 1.0 + 1e-6).all()


def test_on_another_stream():
    rng = np.random.default_rng(14)
    l = rows_of(rng, 17, 9000, torch.bfloat16)
    u = up(rng.random(17))
    want = razer.razer_sample(l, u)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = razer.razer_sample(l, u)[0]
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_flat_rows_and_vocabularies_beyond_the_bins(dtype):
    """Rows whose places lie among more tokens than can be weighed one by one, and more than 2^18 tokens."""
    rng = np.random.default_rng(20)
    for rows, vocab in ((3, 30000), (2, 120000), (2, 300001)):
        l = rows_of(rng, rows, vocab, dtype, 3)
        u = rng.random(rows)
        flat = np.full(rows, 60.0)
        check(l, u, flat, sure=False)
        check(l, u, flat, top_k=np.full(rows, vocab // 3), sure=False)
        check(l, u, flat, top_p=np.full(rows, 0.7), sure=False)
        check(l, u, flat, np.full(rows, vocab // 2), np.full(rows, 0.5), np.full(rows, 0.9), sure=False)
        check(l, u, np.full(rows, 1.0), np.full(rows, 300), np.full(rows, 0.9), np.full(rows, 0.01))
        check(l, u, np.zeros(rows))


def test_places_far_below_the_largest():
    """Weights below 2^-32 of the largest: top_k and min_p that reach there, and a draw that falls there because little else stays."""
    rng = np.random.default_rng(21)
    for rows, vocab in ((4, 3000), (2, 90000)):
        l = rows_of(rng, rows, vocab, torch.float32)
        u = np.full(rows, 0.25)
        cold = np.full(rows, 0.2)                      # most tokens lie beyond 32 octaves
        for k in (50, vocab // 2, vocab - vocab // 90 - 5):
            check(l, u, cold, top_k=np.full(rows, k), sure=False)
            check(l, u, cold, top_k=np.full(rows, k), top_p=np.full(rows, 0.999), sure=False)
        for m in (1e-3, 1e-12, 1e-30):
            check(l, u, cold, min_p=np.full(rows, m), sure=False)
        # one token far above two groups of equal ones, of which the lower is beyond 32 octaves
        x = torch.full((rows, vocab), -40.0, device="cuda")
        x[:, 17] = 0.0
        x[:, 30:40] = -1.0
        assert check(x, np.full(rows, 0.999999), sure=False).tolist() == [39] * rows
        assert check(x, np.full(rows, 0.1), sure=False).tolist() == [17] * rows


def test_two_pieces_of_a_row_and_odd_addresses():
    """Rows that begin at any element, at lengths around those at which a row is cut, and pieces of odd length."""
    rng = np.random.default_rng(22)
    for dtype in (torch.float32, torch.bfloat16):
        for vocab in (40005, 40006, 40007, 45057, 65537):
            flat = torch.full((vocab + 9,), float("inf"), dtype=dtype, device="cuda")
            for off in (0, 1, 3, 7):
                flat[off:off + vocab] = up(rng.standard_normal(vocab) * 2).to(dtype)
                l = flat[off:off + vocab].view(1, vocab)
                check(l, rng.random(1), None, None, np.array([0.9]))
                flat[off:off + vocab] = float("inf")


def test_many_rows():
    rng = np.random.default_rng(23)
    l = rows_of(rng, 70000, 40, torch.bfloat16)
    u = rng.random(70000)
    tok, _ = razer.razer_sample(l, up(u), top_k=torch.full((70000,), 9, dtype=torch.int32, device="cuda"))
    for a in (0, 65530, 69990):
        want, _, margin = so.sample(l[a:a + 10].float().cpu().numpy(), u[a:a + 10].astype(np.float32), top_k=[9] * 10)
        assert (margin > 1e-9).all() and tok[a:a + 10].tolist() == want.tolist()
    none = razer.razer_sample(l[:0], up(u[:0]))
    assert none[0].shape == (0,)


@pytest.mark.parametrize("listed", [1, 2, 3, 63, 64, 65, 128, 129, 511, 513, 1023, 1024, 1025, 2047, 2049, 4095, 4096, 4097])
@pytest.mark.parametrize("vocab", [4200, 60000])
def test_many_tokens_in_a_bin(listed, vocab):
    """So many logits lie in a hundredth of an octave, in one bin, the others far below: each of them is a place on its own."""
    rng = np.random.default_rng(listed + vocab)
    rows = 8
    x = rng.standard_normal((rows, vocab)) - 60.0
    for r in range(rows):
        x[r, rng.permutation(vocab)[:listed]] = rng.uniform(0.0, 0.007, listed)
    l, u = up(x), rng.random(rows)
    check(l, u)
    check(l, u, top_k=rng.integers(1, listed + 1, rows), top_p=rng.uniform(0.2, 0.999, rows))
    check(l, u, min_p=np.exp(-rng.uniform(0.0, 0.007, rows)))
