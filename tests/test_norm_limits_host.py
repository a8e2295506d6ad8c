"""How many rows the norm takes: what is refused is what a grid does not hold.  (Fake pointers, misaligned wherever the sizes are right: nothing is launched.)"""
import ctypes

import pytest

OK = 0x10000
# columns -> the most rows of a forward call
MOST_ROWS = [(1, 2 ** 26 - 4), (64, 2 ** 26 - 4), (128, 2 ** 26 - 4), (1024, 2 ** 26 - 4), (1025, 2 ** 24 - 1), (4096, 2 ** 24 - 1), (4097, 2 ** 23 - 1), (16384, 2 ** 23 - 1),
             (16385, 2 ** 22 - 1), (32768, 2 ** 22 - 1)]


@pytest.fixture(scope="module")
def B():
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("C,most", MOST_ROWS)
def test_rows_of_the_norm(B, C, most):
    def rc(M):
        return B.lib().dfa_rms_norm(OK + 1, C, None, 0, None, 0, 0, ctypes.c_float(1e-6), None, 0, OK, C, None, M, C, None)

    assert rc(1) == rc(2 ** 22 - 1) == rc(most) == -5
    assert rc(most + 1) == rc(2 ** 40) == rc(2 ** 63 - 1) == -7


@pytest.mark.parametrize("C", [1, 64, 1024, 4096, 32768])
def test_rows_of_its_gradients(B, C):
    def rc(M):
        return B.lib().dfa_rms_norm_backward(OK + 1, C, OK, C, None, 0, 0, ctypes.c_float(1e-6), None, 0, OK, C, OK, M, C, OK, 1 << 40, None)

    size = B.lib().dfa_rms_norm_backward_workspace_bytes
    for M in (2 ** 22 - 1, 2 ** 22, 2 ** 26, 2 ** 31 + 1):
        assert rc(M) == -5 and size(M, C) == size(2 ** 21, C) > 0
    assert rc(2 ** 48 // C + 1) == rc(2 ** 63 - 1) == -7 and size(2 ** 48 // C + 1, C) == size(2 ** 63 - 1, C) == 0


def test_what_quantized_may_be(B):
    """A word other than "both" is no answer to whether y is wanted in 8 bits."""
    import torch
    x = torch.zeros((2, 64))
    for word in ("yes", "true", "BOTH", ""):
        with pytest.raises(ValueError, match="quantized"):
            B.rms_norm(x, None, 1e-6, quantized=word)
