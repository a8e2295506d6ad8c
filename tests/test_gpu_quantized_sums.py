"""What the sums of a product keep where large terms cancel: everything in fp32; in bf16 all but 16 * 2^-13 of the largest product of each 16 neighbouring k."""
import pytest

import eight_bit_forms as forms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("M,N,K", [(3, 40, 256), (300, 130, 256), (3801, 3801, 300)])
@pytest.mark.parametrize("at", [(0, 1, 2), (3, 9, 14), (5, 40, 200)])
def test_cancelling_terms(B, M, N, K, at):
    """256 - 256 + 2^-6, the three side by side, apart in one group of 16, and in groups of their own."""
    import torch
    for dtype, code in ((torch.float32, "fp32"), (torch.bfloat16, "bf16")):
        x, w = torch.zeros((M, K), device="cuda"), torch.zeros((N, K), device="cuda")
        for k, (a, b) in zip(at, ((256.0, 1.0), (256.0, -1.0), (2.0 ** -6, 1.0))):
            x[:, k], w[:, k] = a, b
        x, qw = x.to(dtype), B.quantize(w, 128)
        for y in (B.quantized_linear(x, qw), B.quantized_product(B.quantize(x), qw, dtype)):
            if code == "fp32":
                assert bool((y == 2.0 ** -6).all())
            else:
                assert bool(((y.double() - 2.0 ** -6).abs() <= 16 * 2.0 ** -13 * 256 + 2.0 ** -14).all())
    assert forms.product(B, "bf16", 3801, 3801, 300)[0] == 256
