"""Host side of the products of 8-bit operands: the reference's format against torch's e4m3 type, refusals of the C ABI (fake pointers, never
dereferenced: every refusal comes before a launch)."""
import ctypes

import numpy as np
import pytest

import quantized_ref as ref

OK_PTR = 0x10000


@pytest.fixture(scope="module")
def B():
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


def test_reference_numbers_are_torch_s():
    import torch
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(codes, ref.NUMBERS)
    y = np.concatenate([np.linspace(-448, 448, 20001), np.linspace(-0.05, 0.05, 20001), (ref.NUMBERS[:126] + ref.NUMBERS[1:127]) / 2])
    got = torch.from_numpy(y).float().to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ref.to_e4m3(y.astype(np.float32)), got)


def test_reference_scales():
    for amax, e in ((0.0, -126), (448.0, 0), (448.0001, 1), (447.0, 0), (224.0, -1), (1.75, -8), (1.76, -7), (3.4e38, 120), (1e-45, -126)):
        assert ref.scale_exponents(amax) == e


def _matrix(B, rows, cols, **kw):
    a = dict(values=OK_PTR, scales=OK_PTR, ld=-(-cols // 128) * 128, ld_scales=-(-rows // 16) * 16)
    a.update(kw)
    return B.Quantized(a["values"], a["scales"], a["ld"], a["ld_scales"])


def test_refusals_of_quantize(B):
    L = B.lib()

    def rc(x=OK_PTR, dt=0, rows=10, cols=200, ldx=200, block=1, q={}, qt=None):
        q = None if q is None else ctypes.byref(_matrix(B, rows, cols, **q))
        qt = None if qt is None else ctypes.byref(_matrix(B, cols, rows, **qt))
        return L.dfa_quantize(x, dt, rows, cols, ldx, block, q, qt, None)

    assert rc(x=None) == -1 and rc(q=None) == -1 and rc(q=dict(values=None)) == -1 and rc(qt=dict(scales=None)) == -1
    assert rc(dt=2) == -4 and rc(dt=-1) == -4
    for bad in (dict(rows=0), dict(cols=0), dict(rows=-3), dict(ldx=199), dict(block=0), dict(block=64), dict(q=dict(ld=128)),
                dict(q=dict(ld_scales=0)), dict(qt=dict(ld=0)), dict(qt=dict(ld_scales=192))):
        assert rc(**bad) == -2, bad
    for bad in (dict(q=dict(ld=264)), dict(q=dict(ld_scales=24)), dict(q=dict(values=OK_PTR + 8)), dict(qt=dict(scales=OK_PTR + 4)), dict(x=OK_PTR + 1)):
        assert rc(**bad) == -5, bad
    assert rc(cols=1 << 23, ldx=1 << 23) == -7                      # a row of 2^23 values
    assert rc(rows=(1 << 31) - 1, cols=1 << 20, ldx=1 << 20) == -7


def test_refusals_of_the_products(B):
    L = B.lib()

    def product(M=10, N=20, K=200, y=OK_PTR, dt=0, ldy=20, a={}, b={}, ws=None, size=0):
        return L.dfa_quantized_product(_matrix(B, M, K, **a), _matrix(B, N, K, **b), y, dt, M, N, K, ldy, ws, size, None)

    assert product(y=None) == -1 and product(a=dict(values=None)) == -1 and product(b=dict(scales=None)) == -1
    assert product(dt=7) == -4
    for bad in (dict(M=0), dict(N=-1), dict(K=0), dict(ldy=19), dict(a=dict(ld=128)), dict(b=dict(ld_scales=16))):
        assert product(**bad) == -2, bad
    for bad in (dict(a=dict(ld=257)), dict(y=OK_PTR + 1), dict(ws=OK_PTR + 8, size=64)):
        assert product(**bad) == -5, bad
    assert product(K=(1 << 23) + 1, a=dict(ld=1 << 24), b=dict(ld=1 << 24)) == -7

    def linear(M=10, N=20, K=200, x=OK_PTR, y=OK_PTR, dt=0, ldx=200, ldy=20, w={}, ws=None, size=0):
        return L.dfa_quantized_linear(x, dt, ldx, _matrix(B, N, K, **w), y, M, N, K, ldy, ws, size, None)

    assert linear(x=None) == -1 and linear(y=None) == -1 and linear(w=dict(values=None)) == -1
    assert linear(dt=3) == -4
    for bad in (dict(M=0), dict(ldx=199), dict(ldy=19), dict(w=dict(ld=128))):
        assert linear(**bad) == -2, bad
    assert linear(x=OK_PTR + 1) == -5 and linear(dt=1, y=OK_PTR + 2) == -5

    def backward(M=10, N=20, K=200, dy=OK_PTR, x=OK_PTR, dx=OK_PTR, dw=OK_PTR, dt=0, lddy=20, ldx=200, lddx=200, lddw=200, w={}, ws=None, size=0):
        return L.dfa_quantized_linear_backward(dy, lddy, x, ldx, dt, _matrix(B, K, N, **w), dx, lddx, dw, lddw, M, N, K, ws, size, None)

    assert backward(dy=None) == -1 and backward(dx=None, dw=None) == -1 and backward(x=None) == -1
    for bad in (dict(M=0), dict(lddy=19), dict(ldx=199), dict(lddx=199), dict(lddw=199)):
        assert backward(**bad) == -2, bad
    assert backward(dt=5) == -4 and backward(dw=OK_PTR + 2) == -5


def test_workspace_sizes(B):
    L = B.lib()
    assert L.dfa_quantized_linear_workspace_bytes(0, 1, 4096, 4096) == 0 and L.dfa_quantized_linear_workspace_bytes(1, 16, 512, 512) == 0
    assert L.dfa_quantized_linear_workspace_bytes(0, 64, 4096, 8192) >= 64 * 8192        # every workgroup quantising x would take longer
    assert L.dfa_quantized_linear_workspace_bytes(0, 65, 512, 512) >= 65 * 512
    assert L.dfa_quantized_linear_workspace_bytes(0, 0, 512, 512) == 0 and L.dfa_quantized_linear_workspace_bytes(2, 65, 512, 512) == 0
    assert L.dfa_quantized_linear_backward_workspace_bytes(1, 100, 300, 500) >= 100 * 384 + 300 * 128 + 500 * 128
    many = L.dfa_quantized_product_workspace_bytes(1, 128, 128, 1 << 16)       # one tile, long k: shared out
    assert many >= 2 * 128 * 128 * 4 and many % 256 == 0


def test_tensors_on_the_cpu_are_refused(B):
    import torch
    x = torch.zeros((4, 128), dtype=torch.bfloat16)
    q = B.QuantizedMatrix(torch.zeros((16, 128), dtype=torch.float8_e4m3fn), torch.zeros((1, 16), dtype=torch.uint8), 128)
    for call in (lambda: B.quantize(x), lambda: B.quantized_linear(x, q), lambda: B.quantized_product(q, q, torch.float32),
                 lambda: B.quantized_linear_backward(x, x, q)):
        with pytest.raises(RuntimeError):
            call()
