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
