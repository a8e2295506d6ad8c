"""Root-mean-square norm and its gradients on rows at both ends of fp32's range, against the 64-bit references and bounds of packed_ref.

Scaling by a power of two is exact there, so the bounds are those of ordinary rows; a result below the normal range is half a subnormal step off besides."""
import pytest

import packed_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


def _type(name):
    import torch
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def _rows(seed, M, C, dtype, size=1.0):
    """Rows of about `size`, worked out in 64 bits (a normal number times it may be subnormal)."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (size * torch.randn((M, C), generator=gen, device="cuda", dtype=torch.float64)).to(_type(dtype))


def _close(got, want, tol, what):
    over = ((got.double() - want).abs() - tol).max().item()
    assert over <= 0, f"{what}: {over:.3e} over its bound"


def _check(B, h, dy, w, eps):
    """Forward and backward of rows h."""
    import torch
    u = ref.U[h.dtype]
    want, _ = ref.norm(h, w, eps)
    y, _ = B.rms_norm(h, w, eps)
    _close(y, want, want.abs() * (u + ref.NORM_OFF), "y")
    (want_dx, want_dw), (off, off_dw) = ref.norm_backward(dy, h, w, eps)
    dx, dw = B.rms_norm_backward(dy, h, w, eps)
    _close(dx, want_dx, off + u * want_dx.abs() + 2.0 ** -148, "dx")
    _close(dw, want_dw, off_dw, "dw")
    alone, _ = B.rms_norm_backward(torch.zeros_like(dy), h, w, eps)
    assert (alone == 0).all(), "no gradient, none of x"


# every form: threads and pieces of a row, and the gradients that read it again
SIZES = [(9, 500), (5, 2500), (1030, 96), (1100, 777), (4, 4097), (2, 9000), (2, 20001)]


@pytest.mark.parametrize("M,C", SIZES)
@pytest.mark.parametrize("dtype,size,dy_size,eps", [
    ("fp32", 1e-36, 1e-3, 0.0), ("fp32", 1e-39, 1e-10, 0.0), ("fp32", 1e-41, 1e-12, 0.0), ("fp32", 2e-44, 1e-15, 0.0), ("fp32", 1e-21, 1.0, 2.0 ** -140),
    ("fp32", 4e37, 1e10, 0.0), ("fp32", 4e37, 1e10, 1e-6), ("bf16", 1e-38, 1e-9, 0.0), ("bf16", 1e-39, 1e-10, 0.0), ("bf16", 4e37, 1e10, 0.0)])
def test_rows_at_the_ends_of_the_range(B, M, C, dtype, size, dy_size, eps):
    """Their root mean square, or one over it, is no normal fp32 number.  (Six times 4e37 is below 2^128.)"""
    _check(B, _rows(1, M, C, dtype, size).clamp(-3e38, 3e38), _rows(2, M, C, dtype, dy_size), _rows(3, 1, C, dtype)[0], eps)


@pytest.mark.parametrize("C", [64, 1000, 4097, 32768])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_least_number_in_a_row(B, C, dtype):
    """The smallest mean of squares there is, and zeros beside it."""
    import torch
    least = 2.0 ** -149 if dtype == "fp32" else 2.0 ** -133
    h = torch.zeros((3, C), dtype=torch.float64)
    h[0, 0], h[1, C // 2], h[2, C - 1] = least, -least, 3 * least
    _check(B, h.to(_type(dtype)).cuda(), _rows(2, 3, C, dtype, 1e-12), _rows(3, 1, C, dtype)[0], 0.0)


def test_eight_bits_and_the_sum_of_such_rows(B):
    import torch
    x, res, w = _rows(1, 7, 300, "fp32", 1e-40), _rows(2, 7, 300, "fp32", 1e-40), _rows(3, 1, 300, "fp32")[0]
    (y, q), h = B.rms_norm(x, w, 0.0, residual=res, quantized="both")
    want, sums = ref.norm(x, w, 0.0, res)
    assert torch.equal(h.double(), sums)                     # (sums of subnormal numbers are exact)
    _close(y, want, want.abs() * (ref.E + ref.NORM_OFF), "y")
    again = B.quantize(y)
    assert torch.equal(q.values.view(torch.uint8), again.values.view(torch.uint8)) and torch.equal(q.scales[:, :7], again.scales[:, :7])


def test_rows_of_zeros(B):
    """eps alone is what they are divided by; the largest and the least there is."""
    import torch
    for eps in (2.0 ** -149, 2.0 ** -140, 1e-30, 1e-6, 1e30):
        h, dy = torch.zeros((4, 600), device="cuda"), torch.full((4, 600), 2.0 ** -60, device="cuda")
        y, _ = B.rms_norm(h, None, eps)
        dx, dw = B.rms_norm_backward(dy, h, None, eps)
        assert (y == 0).all() and (dw == 0).all()
        want = dy.double() / torch.tensor(eps, dtype=torch.float32).double().sqrt().item()
        _close(dx, want, ref.NORM_OFF * want, "dx")


@pytest.mark.parametrize("M,C", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size,dy_size", [(1e10, 1e30), (1e17, 1e22), (1e3, 1e34)])
def test_gradients_whose_products_with_the_row_overflow(B, M, C, dtype, size, dy_size):
    """Rows that are summed up as they are, with gradients that fp32 holds and products that it does not."""
    _check(B, _rows(1, M, C, dtype, size), _rows(2, M, C, dtype, dy_size), _rows(3, 1, C, dtype)[0], 1e-6)


def test_more_rows_than_a_grid_has_places_for_one_each(B):
    """The norm of the heads of 131072 tokens and a few: forward and dx as of parts of the rows, dw against 64 bits."""
    import torch
    M, C, cut = 2 ** 22 + 5, 64, 1 << 21
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.randn((M, C), generator=gen, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn((C,), generator=gen, device="cuda").bfloat16()
    (y, q), _ = B.rms_norm(x, w, 1e-6, quantized="both")
    dx, dw = B.rms_norm_backward(dy, x, w, 1e-6)
    for rows in (slice(0, cut), slice(cut, 2 * cut), slice(M - 40, M)):
        (y1, q1), _ = B.rms_norm(x[rows], w, 1e-6, quantized="both")
        n = y1.shape[0]
        assert torch.equal(y[rows], y1) and torch.equal(q.values[rows].view(torch.uint8), q1.values.view(torch.uint8)) and torch.equal(q.scales[:, rows], q1.scales[:, :n])
        assert torch.equal(dx[rows], B.rms_norm_backward(dy[rows], x[rows], w, 1e-6, want_dw=False)[0])
    last = slice(M - 300, M)
    want, _ = ref.norm(x[last], w, 1e-6)
    _close(y[last], want, want.abs() * (2.0 ** -8 + ref.NORM_OFF), "y")
    # the workgroups that are resident take 4096 rows at once at least: 1025 of a column are added up one after the other, then three, and sixteen of the parts and eight
    u = x.double() / torch.sqrt(x.double().square().mean(1, keepdim=True) + 1e-6)
    products = dy.double() * u
    _close(dw, products.sum(0), (1025 + 3 + 16 + 8 + 2) * ref.E * products.abs().sum(0) + ref.NORM_OFF * products.abs().sum(0), "dw")


@pytest.mark.parametrize("given", [None, "h"])
def test_whatever_counts_as_true(B, given):
    """quantized=1 and numpy's True are True: y in 8 bits alone, in native code and in Python."""
    import numpy as np
    import torch
    x = _rows(1, 5, 200, "bf16")
    h = None if given is None else torch.empty_like(x)
    want, _ = B.rms_norm(x, None, 1e-6, quantized=True, h=h)
    for yes in (1, np.True_, torch.tensor(True)):
        q, _ = B.rms_norm(x, None, 1e-6, quantized=yes, h=h)
        assert isinstance(q, B.QuantizedMatrix) and torch.equal(q.values.view(torch.uint8), want.values.view(torch.uint8))
    for no in (0, np.False_, None):
        y, _ = B.rms_norm(x, None, 1e-6, quantized=no, h=h)
        assert isinstance(y, torch.Tensor)


@pytest.mark.parametrize("C", [96, 500, 4097, 20001])
def test_sums_of_such_rows_in_place(B, C):
    """h over x or over the residual, among ordinary rows; what is stored is the sum itself, not what it was scaled to."""
    import torch
    x, res = _rows(1, 6, C, "fp32"), _rows(2, 6, C, "fp32")
    for row, size in ((1, 2.0 ** -135), (2, 2.0 ** 120), (4, 2.0 ** -145), (5, 2.0 ** 124)):
        x[row], res[row] = _rows(10 + row, 1, C, "fp32", size)[0], _rows(20 + row, 1, C, "fp32", size)[0]
    want, _ = ref.norm(x, None, 0.0, res)
    sums = x + res
    for place in (None, 0, 1):
        a, b = x.clone(), res.clone()
        y, h = B.rms_norm(a, None, 0.0, residual=b, h=None if place is None else (a, b)[place])
        assert torch.equal(h, sums)
        _close(y, want, want.abs() * (2 * ref.E + ref.NORM_OFF), "y")         # (the sum's rounding and y's)
