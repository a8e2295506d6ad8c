"""Quantised matrices that are rows of larger ones: pointers into the larger arrays, with their pitches.  What lies around the rows stays as it was."""
import ctypes

import numpy as np
import pytest

import quantized_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


KEPT = 0xA5                                                  # no scale byte that these inputs have (2^38)


def _part(B, values, scales, row):
    """The C struct of the rows from `row` (a multiple of 16) on."""
    assert row % 16 == 0
    return B.Quantized(values.data_ptr() + row * values.stride(0), scales.data_ptr() + row, values.stride(0), scales.stride(0))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("transpose", [False, True, "both"])
@pytest.mark.parametrize("rows,cols", [(10, 40), (40, 10), (17, 300), (130, 129)])
def test_quantize_into_a_larger_matrix(B, rows, cols, transpose, block_rows, dtype):
    """Into the middle, and as the last rows of the arrays: the values and scale bytes of the rows up to a multiple of 16 are written, no others."""
    import torch
    rng = np.random.default_rng(rows + cols)
    x = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)).to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]).cuda()
    xe = x.double().cpu().numpy()
    code = B.DFA_F32 if dtype == "fp32" else B.DFA_BF16
    for behind in (160, 0):                                  # rows of the larger matrix behind these
        at, held = 32, []
        for want, src in ((transpose in (False, "both"), xe), (bool(transpose), xe.T)):
            R, C = src.shape
            R16, ld = -(-R // 16) * 16, -(-C // 128) * 128
            values = torch.full((at + R16 + behind, ld + 128), KEPT, dtype=torch.uint8, device="cuda")
            scales = torch.full((ld // 128, at + R16 + behind), KEPT, dtype=torch.uint8, device="cuda")
            held.append((values, scales, src, R16, _part(B, values, scales, at)) if want else None)
        rc = B.lib().dfa_quantize(x.data_ptr(), code, rows, cols, cols, block_rows, *(ctypes.byref(h[4]) if h else None for h in held),
                                  torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        for h in held:
            if h is None:
                continue
            values, scales, src, R16, _ = h
            R, C = src.shape
            ld = -(-C // 128) * 128
            want, exps = ref.quantize(src, block_rows)
            v, s = values.cpu().numpy(), scales.cpu().numpy()
            np.testing.assert_array_equal(ref.NUMBERS[v[at:at + R, :C]], want)
            assert (v[at:at + R, C:ld] == 0).all()
            np.testing.assert_array_equal(s[:, at:at + R].astype(np.int64) - 127, exps)
            assert (s[:, at + R:at + R16] == 1).all()
            assert (s[:, :at] == KEPT).all() and (s[:, at + R16:] == KEPT).all()
            assert (v[:at] == KEPT).all() and (v[at + R:] == KEPT).all() and (v[:, ld:] == KEPT).all()


@pytest.mark.parametrize("M,N,K", [(10, 40, 300), (70, 300, 130), (130, 17, 5000), (300, 200, 700)])
def test_products_of_slices(B, M, N, K):
    """Operands that are the first, middle and last rows of larger matrices: the bits that copies of these rows give."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    rows = lambda m, first, n: B.QuantizedMatrix(m.values[first:first + n], m.scales[:, first:first + -(-n // 16) * 16], m.cols)
    copy = lambda m: B.QuantizedMatrix(m.values.clone(), m.scales.contiguous().clone(), m.cols)
    for before, behind in ((0, 48), (32, 16), (112, 0)):
        a, b = B.quantize(normal(before + M + behind, K)), B.quantize(normal(before + N + behind, K))
        pa, pb = rows(a, before, M), rows(b, before, N)
        for dtype in (torch.float32, torch.bfloat16):
            assert torch.equal(B.quantized_product(pa, pb, dtype), B.quantized_product(copy(pa), copy(pb), dtype))
        x, dy = normal(M, K), normal(M, N)
        assert torch.equal(B.quantized_linear(x, pb), B.quantized_linear(x, copy(pb)))
        wt = rows(B.quantize(normal(before + K + behind, N)), before, K)
        for got, want in zip(B.quantized_linear_backward(dy, x, wt), B.quantized_linear_backward(dy, x, copy(wt))):
            assert torch.equal(got, want)
