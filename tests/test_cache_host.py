"""Host side of the cache of keys and values in e4m3: refusals of the C ABI (fake pointers, never dereferenced), workspace sizes, and the
reference's own pins."""
import ctypes

import numpy as np
import pytest

import cache_ref
import quantized_ref as ref

OK_PTR = 0x10000


@pytest.fixture(scope="module")
def B():
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


def _cache(B, **kw):
    a = dict(k=OK_PTR, v=OK_PTR, scales=OK_PTR, pages=4, heads=2, page=16, D=64)
    a.update(kw)
    return B.Cache(a["k"], a["v"], a["scales"], a["pages"], a["heads"], a["page"], a["D"])


BAD_CACHES = [(dict(page=8), -2), (dict(page=48), -2), (dict(page=256), -2), (dict(D=32), -2), (dict(D=96), -2), (dict(pages=0), -2), (dict(heads=0), -2),
              (dict(k=None), -1), (dict(v=None), -1), (dict(scales=None), -1), (dict(k=OK_PTR + 8), -5), (dict(v=OK_PTR + 4), -5)]
BAD_NAMES = [(dict(table=None), -1), (dict(lengths=None), -1), (dict(table=OK_PTR + 2), -5), (dict(lengths=OK_PTR + 1), -5), (dict(counts=OK_PTR + 2), -5),
             (dict(width=0), -2), (dict(ld=1), -2), (dict(width=1 << 28, ld=1 << 28), -7), (dict(Bsz=0), -2)]


def test_refusals_of_append(B):
    def rc(k=OK_PTR, v=OK_PTR, s=(128 * 3, 128, 64), dt=0, Bsz=2, T=3, cache={}, table=OK_PTR, width=2, ld=2, lengths=OK_PTR, counts=None):
        st = B.Strides(*s)
        return B.lib().dfa_cache_append(k, v, st, st, dt, Bsz, T, _cache(B, **cache), table, width, ld, lengths, counts, None)

    assert rc(k=None) == -1 and rc(v=None) == -1 and rc(dt=2) == -4 and rc(T=0) == -2 and rc(T=-1) == -2
    assert rc(k=OK_PTR + 2) == -5 and rc(s=(128 * 3, 128, 60)) == -5 and rc(s=(4, 128, 64)) == -5
    for bad, code in BAD_CACHES:
        assert rc(cache=bad) == code, bad
    for bad, code in BAD_NAMES:
        assert rc(**bad) == code, bad
    assert rc(Bsz=1 << 30, cache=dict(heads=1 << 20)) == -7


def test_refusals_of_attention(B):
    def rc(q=OK_PTR, s=(256 * 3, 256, 64), dt=0, Bsz=2, M=3, H=4, cache={}, table=OK_PTR, width=2, ld=2, lengths=OK_PTR, counts=None, scale=0.125, limit=32,
           out=OK_PTR, lse=None, ws=None, size=0):
        return B.lib().dfa_cache_attention(q, B.Strides(*s), dt, Bsz, M, H, _cache(B, **cache), table, width, ld, lengths, counts, 1, ctypes.c_float(scale),
                                           limit, out, lse, ws, size, None)

    assert rc(q=None) == -1 and rc(out=None) == -1 and rc(dt=-1) == -4
    for bad in (dict(M=0), dict(H=3), dict(H=0), dict(H=1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(limit=-1)):
        assert rc(**bad) == -2, bad
    for bad in (dict(q=OK_PTR + 2), dict(s=(256 * 3, 256, 4)), dict(out=OK_PTR + 8), dict(lse=OK_PTR + 2), dict(ws=OK_PTR + 8)):
        assert rc(**bad) == -5, bad
    for bad, code in BAD_CACHES:
        assert rc(cache=bad) == code, bad
    for bad, code in BAD_NAMES:
        assert rc(**bad) == code, bad
    assert rc(M=1 << 30, H=8) == -7


def test_workspace_sizes(B):
    size = B.lib().dfa_cache_attention_workspace_bytes
    assert size(1, 1, 12, 12, 64, 0, 64) == 0                       # a chunk of 64 tokens is nothing to share out
    assert size(1, 1, 12, 12, 64, 0, 4096) > 0 and size(1, 1, 12, 12, 64, 0, 4096) % 256 == 0
    assert size(0, 1, 12, 12, 64, 0, 4096) == 0 and size(1, 1, 12, 5, 64, 0, 4096) == 0 and size(1, 1, 12, 12, 64, 9, 4096) == 0
    assert size(4096, 1, 12, 12, 64, 0, 4096) == 0                  # enough workgroups without


def test_tensors_on_the_cpu_are_refused(B):
    import torch
    cache = B.kv_cache(2, 1, 16, 64, device="cpu")
    t, n, x = torch.zeros((1, 2), dtype=torch.int32), torch.ones((1,), dtype=torch.int32), torch.zeros((1, 1, 1, 64))
    for call in (lambda: B.cache_append(x, x, cache, t, n), lambda: B.cache_attention(x, cache, t, n, 1.0)):
        with pytest.raises(RuntimeError):
            call()


def test_reference_attention_is_textbook_attention(B):
    """On whole pages of exactly held numbers the reference is softmax attention; an appended token by token cache holds what one append leaves
    where no scale grows."""
    import torch
    rng = np.random.default_rng(4)
    n, heads, D = 40, 2, 64
    k, v = (rng.integers(-4, 5, (1, n, heads, D)).astype(np.float64) for _ in range(2))
    k[:, ::16, :, 0], v[:, ::16, :, 0] = 5, 5                       # every page's first token has its largest number
    q = rng.standard_normal((1, 3, heads, D))
    empty = B.kv_cache(3, heads, 16, D, device="cpu")
    once, steps = cache_ref.Model(empty), cache_ref.Model(empty)
    table = np.array([[2, 0, 1]])
    once.append(k, v, table, [n])
    for t in range(n):
        steps.append(k[:, t:t + 1], v[:, t:t + 1], table, [t + 1])
    np.testing.assert_array_equal(once.k, steps.k)
    np.testing.assert_array_equal(once.v, steps.v)
    np.testing.assert_array_equal(once.e, steps.e)
    out, lse = cache_ref.attention(once, q, table, [n], 0.125, True)[:2]
    for i in range(3):
        for h in range(heads):
            z = 0.125 * k[0, :n - 2 + i, h] @ q[0, i, h]
            p = np.exp(z)
            np.testing.assert_allclose(out[0, i, h], p @ v[0, :n - 2 + i, h] / p.sum(), rtol=1e-12, atol=1e-12)
            np.testing.assert_allclose(lse[0, h, i], np.log(p.sum()), rtol=1e-12)
    assert ref.NUMBERS.shape == (256,) and torch.float8_e4m3fn is not None
