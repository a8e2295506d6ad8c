"""Attention over the cache where a row meets scores of very different size: running maxima that climb from far below, rows of one tile
that do and do not."""
import numpy as np
import pytest

import cache_ref
import quantized_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


def _ints(values):
    import torch
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _reference(k, v, q, scale, ends, dtype):
    """(out, lse, bar of out, bar of lse) in fp64 for rows q [M, D] against k, v [T, D], row i seeing the first ends[i].

    Bars: a score is an fp32 sum of D products, off by at most (D + 8) 2^-24 of the magnitudes it adds up; exponentials and logarithms are good to
    2^-21 and a part that grows with the exponent.  A token more than 64 below the row's largest score has less than e^-60 of its weight, errors of
    its score (at most 1e-5 of it here) included: only the others' errors count."""
    M, D = q.shape
    out, lse, bar, lse_bar = np.zeros((M, D)), np.zeros(M), np.zeros((M, D)), np.zeros(M)
    half = ref.HALF_STEP[dtype]
    for i in range(M):
        z, size = scale * (k[:ends[i]] @ q[i]), scale * (np.abs(k[:ends[i]]) @ np.abs(q[i]))
        top = z.max()
        near = z >= top - 64
        p = np.exp(z - top)
        out[i], lse[i] = p @ v[:ends[i]] / p.sum(), top + np.log(p.sum())
        delta = (D + 8) * 2.0 ** -24 * size[near].max() + 2.0 ** -21 * (1 + np.abs(z - top)[near].max() * 2.0 ** -3)
        bar[i] = (half + 2 * delta + 2 * ends[i] * 2.0 ** -24) * (p @ np.abs(v[:ends[i]]) / p.sum()) * 1.01 + half * np.abs(out[i])
        lse_bar[i] = delta + ends[i] * 2.0 ** -24 + 2.0 ** -21 * max(1.0, abs(lse[i]))
    return out, lse, bar, lse_bar


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("low", [1e5, 1e7, 1e10])
@pytest.mark.parametrize("M,D", [(1, 64), (20, 64), (40, 64), (1, 128), (20, 128)])
def test_maxima_that_climb(B, M, D, low, dtype):
    """The first tokens that every wave walks score near -low, later ones a few units; every third row scores a few units all along."""
    import torch
    rng = np.random.default_rng(M + D)
    page, T = 32, 900
    cache = B.kv_cache(30, 1, page, D)
    table = rng.permutation(30)[None].astype(np.int32)
    k = rng.standard_normal((T, D))
    k[:, 0] = np.where(np.arange(T) < 300, -1.0, 0.0)
    v = rng.standard_normal((T, D))
    on_gpu = lambda x: torch.from_numpy(x.astype(np.float32)).view(1, -1, 1, D).cuda()
    B.cache_append(on_gpu(k), on_gpu(v), cache, _ints(table), _ints([T]))
    kk, vv, there = cache_ref.Model(cache).sequence(0, table, T)
    assert there.all()
    q = 2.0 * rng.standard_normal((M, D))
    q[:, 0] = np.where(np.arange(M) % 3 == 1, 0.0, low / 0.125)
    qt = on_gpu(q).to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype])
    qe = qt.double().cpu().numpy()[0, :, 0]
    want, want_lse, bar, lse_bar = _reference(kk[:, 0], vv[:, 0], qe, 0.125, T - (M - 1 - np.arange(M)), dtype)
    assert (np.abs(want_lse) < 50).all()
    for limit in (1, 500, None):
        out, lse = B.cache_attention(qt, cache, _ints(table), _ints([T]), 0.125, max_length=limit)
        err, lse_err = np.abs(out.double().cpu().numpy()[0, :, 0] - want), np.abs(lse.double().cpu().numpy()[0, 0] - want_lse)
        print(f"[climb {M} {D} {low} {dtype} {limit}] worst err/bar {float((err / bar).max()):.3f}, lse {float((lse_err / lse_bar).max()):.3f}", flush=True)
        assert (err <= bar).all() and (lse_err <= lse_bar).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,D", [(1, 64), (20, 64), (40, 64), (1, 128), (20, 128)])
def test_differences_of_large_scores(B, M, D, dtype):
    """Whole numbers near 2^22 as scores, exact in fp32, a quarter of which is what the exponential takes: rows are ordinary softmax rows of the differences, however
    the walk is shared out.  Bars: exponentials and logarithms (2^-21, a part that grows with the difference), sums of the weights, the result's rounding."""
    import torch
    rng = np.random.default_rng(M + D)
    page, T = 16, 800
    cache = B.kv_cache(51, 1, page, D)
    table = rng.permutation(51)[None].astype(np.int32)
    k = np.zeros((T, D))
    k[:, 0], k[:, 1:5] = 8, rng.integers(-4, 5, (T, 4))
    v = rng.standard_normal((T, D))
    on_gpu = lambda x: torch.from_numpy(x.astype(np.float32)).view(1, -1, 1, D).cuda()
    B.cache_append(on_gpu(k), on_gpu(v), cache, _ints(table), _ints([T]))
    kk, vv, _ = cache_ref.Model(cache).sequence(0, table, T)
    np.testing.assert_array_equal(kk[:, 0], k)
    q = np.zeros((M, D))
    q[:, 0], q[:, 1:5] = 2.0 ** 19, rng.choice([-1.0, 1.0], (M, 4))
    qt = on_gpu(q).to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype])
    half = ref.HALF_STEP[dtype]
    for limit in (1, 300, None):
        out, lse = B.cache_attention(qt, cache, _ints(table), _ints([T]), 0.25, max_length=limit)
        for i in range(M):
            n = T - (M - 1 - i)
            z = 0.25 * (k[:n] @ q[i])
            p = np.exp(z - z.max())
            want, want_lse = p @ vv[:n, 0] / p.sum(), z.max() + np.log(p.sum())
            delta = 2.0 ** -21 * (1 + (z.max() - z.min()) / 8)
            bar = (half + 2 * delta + 2 * n * 2.0 ** -24) * (p @ np.abs(vv[:n, 0]) / p.sum()) * 1.01 + half * np.abs(want)
            assert (np.abs(out.double().cpu().numpy()[0, i, 0] - want) <= bar).all(), (limit, i)
            assert abs(float(lse[0, 0, i]) - want_lse) <= 2.0 ** -21 * want_lse, (limit, i)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("M,D", [(1, 64), (20, 64), (40, 64), (20, 128)])
def test_scores_that_pass_fp32_when_scaled(B, M, D, sign, dtype):
    """Scores of up to 2^108 times a scale of 2^30, all of one sign: the row is the mean of its best tokens' values, lse is infinite."""
    import torch
    rng = np.random.default_rng(M + D)
    page, T = 32, 700
    cache = B.kv_cache(24, 1, page, D)
    table = rng.permutation(24)[None].astype(np.int32)
    k = rng.integers(1, 9, (T, D)).astype(np.float64)
    on_gpu = lambda x: torch.from_numpy(x.astype(np.float32)).view(1, -1, 1, D).cuda()
    B.cache_append(on_gpu(k), on_gpu(rng.standard_normal((T, D))), cache, _ints(table), _ints([T]))
    kk, vv, _ = cache_ref.Model(cache).sequence(0, table, T)
    np.testing.assert_array_equal(kk[:, 0], k)
    q = sign * rng.integers(1, 9, (M, D)) * 2.0 ** 96
    scores = q @ k.T                                                           # exact: whole numbers below 2^13 times 2^96
    scores[np.arange(T)[None, :] >= T - (M - 1 - np.arange(M))[:, None]] = -np.inf
    best = scores == scores.max(1, keepdims=True)
    want = best @ vv[:, 0] / best.sum(1, keepdims=True)
    bar = (2.0 ** -8 if dtype == "bf16" else 0.0) * np.abs(want) + 2.0 ** -20 * np.abs(vv).max()
    qt = on_gpu(q).to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype])
    for limit in (1, 300, None):
        out, lse = B.cache_attention(qt, cache, _ints(table), _ints([T]), 2.0 ** 30, max_length=limit)
        assert (np.abs(out.double().cpu().numpy()[0, :, 0] - want) <= bar).all()
        assert bool((lse == sign * float("inf")).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("power", [-70, -112, -120, -135])
@pytest.mark.parametrize("M,D", [(1, 64), (20, 64), (40, 64), (1, 128), (20, 128)])
def test_small_queries_against_large_keys(B, M, D, power, dtype):
    """Queries down to fp32's least numbers against keys of up to 2^120, ordinary scores; every third row of ordinary size, whose scores are huge."""
    import torch
    rng = np.random.default_rng(M + D - power)
    page, T = 32, 500
    cache = B.kv_cache(17, 1, page, D)
    table = rng.permutation(17)[None].astype(np.int32)
    up = min(-power - 2, 118)
    on_gpu = lambda x: torch.from_numpy(x.astype(np.float32)).view(1, -1, 1, D).cuda()
    B.cache_append(on_gpu(rng.standard_normal((T, D)) * 2.0 ** up), on_gpu(rng.standard_normal((T, D))), cache, _ints(table), _ints([T]))
    kk, vv, there = cache_ref.Model(cache).sequence(0, table, T)
    assert there.all()
    q = rng.standard_normal((M, D)) * 2.0 ** np.where(np.arange(M) % 3 == 1, 0, power)[:, None]
    qt = on_gpu(q).to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype])
    qe = qt.double().cpu().numpy()[0, :, 0]
    scale = 2.0 ** (-power - up - 2)
    want, want_lse, bar, lse_bar = _reference(kk[:, 0], vv[:, 0], qe, scale, T - (M - 1 - np.arange(M)), dtype)
    assert (bar[0] <= 0.02 * np.abs(vv).max()).all()
    for limit in (1, None):
        out, lse = B.cache_attention(qt, cache, _ints(table), _ints([T]), scale, max_length=limit)
        got_lse = lse.double().cpu().numpy()[0, 0]
        over = np.abs(want_lse) > 3.4028235e38               # rounds to an infinity of its sign
        assert (got_lse[over] == np.copysign(np.inf, want_lse[over])).all() and np.isfinite(got_lse[~over]).all()
        err, lse_err = np.abs(out.double().cpu().numpy()[0, :, 0] - want), np.where(over, 0.0, np.abs(got_lse - want_lse))
        print(f"[small {M} {D} {power} {dtype} {limit}] worst err/bar {float((err / bar).max()):.3f}, lse {float((lse_err / lse_bar).max()):.3f}", flush=True)
        assert (err <= bar).all() and (lse_err <= lse_bar).all()


@pytest.mark.parametrize("M,D", [(1, 64), (20, 64), (20, 128)])
def test_queries_next_to_the_largest_number(B, M, D):
    """fp32 queries that would round to infinity in bf16."""
    import torch
    rng = np.random.default_rng(M + D)
    page, T = 16, 200
    cache = B.kv_cache(14, 1, page, D)
    table = rng.permutation(14)[None].astype(np.int32)
    on_gpu = lambda x: torch.from_numpy(x.astype(np.float32)).view(1, -1, 1, D).cuda()
    B.cache_append(on_gpu(rng.standard_normal((T, D)) * 2.0 ** -110), on_gpu(rng.standard_normal((T, D))), cache, _ints(table), _ints([T]))
    kk, vv, _ = cache_ref.Model(cache).sequence(0, table, T)
    q = rng.choice([-1.0, 1.0], (M, D)) * float(np.float32(3.4028234e38)) * (1 - rng.integers(0, 100, (M, D)) * 2.0 ** -24)
    qt = on_gpu(q)
    assert torch.isfinite(qt).all() and torch.isinf(qt.to(torch.bfloat16)).all()
    scale = 2.0 ** -19
    want, want_lse, bar, lse_bar = _reference(kk[:, 0], vv[:, 0], qt.double().cpu().numpy()[0, :, 0], scale, T - (M - 1 - np.arange(M)), "fp32")
    out, lse = B.cache_attention(qt, cache, _ints(table), _ints([T]), scale)
    assert (np.abs(out.double().cpu().numpy()[0, :, 0] - want) <= bar).all() and (np.abs(lse.double().cpu().numpy()[0, 0] - want_lse) <= lse_bar).all()
