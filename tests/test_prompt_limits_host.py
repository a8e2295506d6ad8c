"""How large packed prompts may be.  (Fake pointers, a misaligned gradient wherever the sizes are right: nothing is launched.)"""
import ctypes

import pytest

OK = 0x10000


@pytest.fixture(scope="module")
def B():
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


def _backward(B, T, H, Hkv, D, dt=0, Bsz=8):
    es = 4 if dt else 2
    sq, sk = B.Strides(0, H * D, D), B.Strides(0, Hkv * D, D)
    assert H * D * es < 1 << 25
    return B.lib().dfa_prompt_attention_backward(OK, OK, OK, sq, sk, sk, OK, OK, OK + 2, dt, T, H, Hkv, D, OK, Bsz, 1, ctypes.c_float(0.125), OK, OK, OK, OK, 1 << 50, None)


@pytest.mark.parametrize("dt", [0, 1])
def test_gradients_of_many_elements(B, dt):
    """What a launch's grid does not hold is refused, and nothing else: 2^33 elements of k and more are not too many."""
    for T, H, Hkv, D in ((2 ** 21 + 7, 32, 32, 128), (2 ** 22 + 7, 32, 32, 64), (2 ** 24, 31, 31, 64), (2 ** 23, 32, 32, 128)):
        assert T * Hkv * D >= 2 ** 33
        assert _backward(B, T, H, Hkv, D, dt) == -5, (T, H, Hkv, D)
        assert B.lib().dfa_prompt_attention_backward_workspace_bytes(T, H, Hkv, D, 8) == -(-2 * H * T * 4 // 256) * 256
    for T, H, Bsz in ((2 ** 24, 32, 8), (1000, 64, 2 ** 18), (2 ** 29, 1, 8)):
        assert _backward(B, T, H, H, 64, dt, Bsz) == -7 and B.lib().dfa_prompt_attention_backward_workspace_bytes(T, H, H, 64, Bsz) == 0
