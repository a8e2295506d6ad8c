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
        near = z > top - 64
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
