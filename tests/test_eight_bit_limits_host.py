"""Sizes beyond what the operators on 8-bit operands count in are refused by the host (fake pointers, never dereferenced)."""
import ctypes

import pytest

OK_PTR = 0x10000


@pytest.fixture(scope="module")
def B():
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("dt,D", [(0, 64), (0, 128), (1, 64), (1, 128)])
def test_counts_of_tiles_beyond_64_bits(B, dt, D):
    """Sequences, heads and rows whose product is 2^64 and more."""
    L = B.lib()
    for Bsz, M, H, heads in ((1 << 30, 256, 1 << 30, 1 << 30), (1 << 30, 1, 1 << 30, 1 << 30), (1 << 20, 1 << 24, 1 << 24, 1 << 24)):
        assert L.dfa_cache_attention_workspace_bytes(Bsz, M, H, heads, D, dt, 4096) == 0
        cache = B.Cache(OK_PTR, OK_PTR, OK_PTR, 4, heads, 64, D)
        st = B.Strides(64 * D, 64 * D, D)
        assert L.dfa_cache_attention(OK_PTR, st, dt, Bsz, M, H, cache, OK_PTR, 2, 2, OK_PTR, None, 1, ctypes.c_float(0.125), 128, OK_PTR, None, None, 0, None) == -7


def test_grids_of_2_32_threads(B):
    """What a launch cannot hold is too large, not an error of the runtime."""
    L = B.lib()
    q = lambda rows, cols: ctypes.byref(B.Quantized(OK_PTR, OK_PTR, -(-cols // 128) * 128, -(-rows // 16) * 16))
    for rows, cols in ((1 << 29, 1 << 12), (1 << 30, 128 * 70)):
        assert L.dfa_quantize(OK_PTR, 0, rows, cols, cols, 1, q(rows, cols), None, None) == -7
    m = lambda rows: B.Quantized(OK_PTR, OK_PTR, 128, -(-rows // 16) * 16)
    assert L.dfa_quantized_product(m(1 << 30), m(1 << 30), OK_PTR, 0, 1 << 30, 1 << 30, 128, 1 << 30, None, 0, None) == -7
    st = B.Strides(1 << 20, 1 << 10, 128)
    cache = B.Cache(OK_PTR, OK_PTR, OK_PTR, 4, 1 << 10, 128, 128)
    append = lambda Bsz, T: L.dfa_cache_append(OK_PTR, OK_PTR, st, st, 0, Bsz, T, cache, OK_PTR, 1 << 20, 1 << 20, OK_PTR, None, None)
    assert append(1 << 12, 1) == -7 and append(1 << 30, 1 << 26) == -7
