"""The sizes that the GPU tests run for one form of the operators on 8-bit operands in particular take that form, and every form has one."""
import ctypes

import pytest

import eight_bit_forms as forms


@pytest.fixture(scope="module")
def B():
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


def test_sizes_take_their_forms(B):
    for dtype, M, N, K, tile, splits in forms.PRODUCTS:
        assert forms.product(B, dtype, M, N, K) == (tile, splits), (dtype, M, N, K)
    for dtype, M, N, K, blocks, tile in forms.LINEARS:
        assert forms.linear(B, dtype, M, N, K) == (blocks, tile), (dtype, M, N, K)
    for dtype, M, N, K, *form in forms.GRADIENTS:
        assert forms.gradients(B, dtype, M, N, K) == tuple(form), (dtype, M, N, K)
    for *size, rows, tiles, splits in forms.ATTENTIONS:
        assert forms.attention(B, *size) == (rows, tiles, splits), size


def test_every_form_has_a_size(B):
    assert {(d, t, s > 1) for d, _, _, _, t, s in forms.PRODUCTS} == {(d, t, s) for d in ("bf16", "fp32") for t in (128, 256) for s in (False, True)}
    assert {(d, b) for d, _, _, _, b, _ in forms.LINEARS} == {(d, b) for d in ("bf16", "fp32") for b in (0, 1, 2, 4)}
    assert {(d, paired) for d, _, _, _, _, _, paired in forms.GRADIENTS} == {(d, p) for d in ("bf16", "fp32") for p in (False, True)}
    most = {("bf16", 64): 48, ("bf16", 128): 32, ("fp32", 64): 32, ("fp32", 128): 16}
    assert ({(d, D, r, t, s) for d, _, _, _, _, D, _, _, r, t, s in forms.ATTENTIONS if r > 16 or most[d, D] == 16} | {(d, D, 16, False, s) for d, D in most for s in (False, True)}
            == {(d, D, r, t, s) for (d, D), m in most.items() for r in range(16, m + 1, 16) for t in (False, True) for s in (False, True) if r > 16 or not t or m == 16})


def test_refusals(B):
    L, q, a = B.lib(), B.QuantizedForm(), B.CacheAttentionForm()
    for call, dt, size, code in ((0, 2, (1, 1, 1), -4), (-1, 0, (1, 1, 1), -2), (4, 0, (1, 1, 1), -2), (1, 0, (0, 1, 1), -2), (2, 0, (1 << 24, 64, 64), -7)):
        assert L.dfa_quantized_describe(call, dt, *size, ctypes.byref(q)) == code
    assert L.dfa_quantized_describe(0, 0, 1, 1, 1, None) == -1
    for size, dt, limit, code in (((1, 1, 3, 2, 64), 0, 64, -2), ((1, 1, 2, 2, 32), 0, 64, -2), ((1, 1, 2, 2, 64), 5, 64, -4), ((1, 1, 2, 2, 64), 0, -1, -2)):
        assert L.dfa_cache_attention_describe(*size, dt, limit, ctypes.byref(a)) == code
    assert L.dfa_cache_attention_describe(1, 1, 2, 2, 64, 0, 64, None) == -1
