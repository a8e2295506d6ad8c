"""Root-mean-square norm, its 8-bit result and its gradients against 64-bit references; bounds in packed_ref."""
import numpy as np
import pytest

import packed_ref as ref
import quantized_ref

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
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (size * torch.randn((M, C), generator=gen, device="cuda") * torch.exp2(torch.randn((M, 1), generator=gen, device="cuda"))).to(_type(dtype))


def _close(got, want, tol, what):
    over = ((got.double() - want).abs() - tol).max().item()
    assert over <= 0, f"{what}: {over:.3e} over its bound"


def _check_quantized(B, q, y):
    """Values and scale bytes of y within what y may be off by: the bytes of y's blocks, or of blocks a hair larger or smaller; values half a step off."""
    import torch
    M, C = y.shape
    ld = -(-C // 128) * 128
    full = torch.zeros((M, ld), dtype=torch.float64, device=y.device)
    full[:, :C] = y
    amax = full.view(M, ld // 128, 128).abs().amax(2).cpu().numpy()
    lo, hi = (quantized_ref.scale_exponents(amax * f) for f in (1 - ref.NORM_OFF, 1 + ref.NORM_OFF))
    e = q.scales[:, :M].t().cpu().numpy().astype(np.int64) - 127
    assert ((e == lo) | (e == hi)).all()
    assert (q.scales[:, M:-(-M // 16) * 16] == 1).all()
    unit = torch.from_numpy(np.exp2(e.astype(np.float64))).cuda().repeat_interleave(128, 1)
    got = q.values.double() * unit
    _close(got, full, full.abs() * (2.0 ** -4 + 2 * ref.NORM_OFF) + unit * 2.0 ** -10, "values")
    assert (q.values[:, C:].view(torch.uint8) == 0).all()


SIZES = [(1, 1), (1, 4096), (3, 7), (5, 129), (17, 1000), (2, 2049), (33, 768), (4, 4097), (2, 8200), (2, 16384), (1, 20001), (1, 32768), (1030, 96), (1100, 777), (1025, 1024),
         (5000, 300), (3500, 1000), (2000, 2100), (1100, 4000), (600, 4500), (300, 9000), (530, 20001)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,C", SIZES)
def test_norm(B, M, C, dtype):
    x, res, w = _rows(1, M, C, dtype), _rows(2, M, C, dtype), _rows(3, 1, C, dtype)[0]
    u = ref.U[x.dtype]
    for residual in (None, res):
        for weight in (w, None):
            (y, q), h = B.rms_norm(x, weight, 1e-6, residual=residual, quantized="both")
            want, sums = ref.norm(x, weight, 1e-6, residual)
            _close(y, want, want.abs() * (u + ref.NORM_OFF), "y")
            _check_quantized(B, q, want)
            if residual is None:
                assert h is None
            else:
                _close(h, sums, sums.abs() * u + 2 * ref.E * sums.abs(), "h")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,C", SIZES)
def test_backward(B, M, C, dtype):
    h, dy, dh, w = _rows(1, M, C, dtype), _rows(2, M, C, dtype), _rows(3, M, C, dtype), _rows(4, 1, C, dtype)[0]
    u = ref.U[h.dtype]
    for more, weight in ((dh, w), (None, w), (dh, None)):
        dx, dw = B.rms_norm_backward(dy, h, weight, 1e-6, dh=more)
        (want_dx, want_dw), (off, off_dw) = ref.norm_backward(dy, h, weight, 1e-6, more)
        _close(dx, want_dx, off + u * want_dx.abs(), "dx")
        _close(dw, want_dw, off_dw, "dw")
        alone, none = B.rms_norm_backward(dy, h, weight, 1e-6, dh=more, want_dw=False)
        assert none is None and (alone == dx).all()


def test_backward_against_differences(B):
    import torch
    h, dy, dh, w = _rows(1, 5, 40, "fp32"), _rows(2, 5, 40, "fp32"), _rows(3, 5, 40, "fp32"), _rows(4, 1, 40, "fp32")[0]
    dx, dw = B.rms_norm_backward(dy, h, w, 1e-3, dh=dh)
    (_, _), (off, off_dw) = ref.norm_backward(dy, h, w, 1e-3, dh)
    gen = torch.Generator(device="cuda").manual_seed(1)
    a, b = torch.randn(h.shape, generator=gen, device="cuda", dtype=torch.float64), torch.randn(w.shape, generator=gen, device="cuda", dtype=torch.float64)

    def value(step, which):
        hs = h.double() + (step * a if which == 0 else 0.0)
        ws = w.double() + (step * b if which else 0.0)
        y, _ = ref.norm(hs, ws, 1e-3)
        return (y * dy.double()).sum() + (hs * dh.double()).sum()

    for which, got, tol in ((0, (dx.double() * a).sum(), ((off + ref.E * dx.double().abs()) * a.abs()).sum()), (1, (dw.double() * b).sum(), (off_dw * b.abs()).sum())):
        slope = (value(1e-5, which) - value(-1e-5, which)) / 2e-5
        assert (got - slope).abs() <= tol + 1e-7 * slope.abs() + 1e-7


def test_bf16_rows_fp32_weight(B):
    x, w = _rows(1, 20, 300, "bf16"), _rows(2, 1, 300, "fp32")[0]
    y, _ = B.rms_norm(x, w, 1e-5)
    want, _ = ref.norm(x, w, 1e-5)
    _close(y, want, want.abs() * (2.0 ** -8 + ref.NORM_OFF), "y")
    dx, dw = B.rms_norm_backward(x, x, w, 1e-5)
    (want_dx, want_dw), (off, off_dw) = ref.norm_backward(x, x, w, 1e-5)
    _close(dx, want_dx, off + 2.0 ** -8 * want_dx.abs(), "dx")
    _close(dw, want_dw, off_dw, "dw")


@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("size", [1e30, 1e-18, 1e-25])
def test_rows_of_any_size(B, size, eps):
    """Sums of squares that fp32 does not hold."""
    import torch
    h, dy, w = _rows(1, 9, 500, "fp32", size), _rows(2, 9, 500, "fp32"), _rows(3, 1, 500, "fp32")[0]
    want, _ = ref.norm(h, w, eps)
    y, _ = B.rms_norm(h, w, eps)
    _close(y, want, want.abs() * (ref.E + ref.NORM_OFF), "y")
    (want_dx, want_dw), (off, off_dw) = ref.norm_backward(dy, h, w, eps)
    dx, dw = B.rms_norm_backward(dy, h, w, eps)
    # (results below fp32's normal range are a subnormal step off)
    _close(dx, want_dx, off + ref.E * want_dx.abs() + 2.0 ** -148, "dx")
    _close(dw, want_dw, off_dw, "dw")


def test_odd_rows(B):
    """Rows of zeros and values that are not finite stay in their rows."""
    import torch
    x, w = _rows(1, 6, 200, "bf16"), _rows(2, 1, 200, "bf16")[0]
    clean, _ = B.rms_norm(x, w, 1e-6, quantized="both")
    x[1], x[2, 5], x[4, 7] = 0.0, float("nan"), float("inf")
    (y, q), _ = B.rms_norm(x, w, 1e-6, quantized="both")
    for r in (0, 3, 5):
        assert torch.equal(y[r], clean[0][r]) and torch.equal(q.values[r].view(torch.uint8), clean[1].values[r].view(torch.uint8))
    assert (y[1] == 0).all() and y[2].isnan().all() and y[4, 7].isnan() and (q.values[1].float() == 0).all() and (q.scales[:, 1] == 1).all()
    assert q.values[2, :200].float().isnan().all() and (q.values[2, 200:].view(torch.uint8) == 0).all()


def test_in_place_views_and_repeats(B):
    """h over x or over the residual; rows of a wider matrix at any element; more than two dimensions; equal calls, equal bits."""
    import torch
    x, res, w = _rows(1, 40, 333, "bf16"), _rows(2, 40, 333, "bf16"), _rows(3, 1, 333, "bf16")[0]
    y, h = B.rms_norm(x, w, 1e-6, residual=res)
    for place in (0, 1):
        a, b = x.clone(), res.clone()
        y2, h2 = B.rms_norm(a, w, 1e-6, residual=b, h=(a, b)[place])
        assert torch.equal(y, y2) and torch.equal(h, (a, b)[place]) and h2 is (a, b)[place] and torch.equal((a, b)[1 - place], (x, res)[1 - place])
    wide = torch.zeros((40, 701), dtype=x.dtype, device="cuda")
    wide[:, 3:336], wide[:, 367:700] = x, res
    y3, h3 = B.rms_norm(wide[:, 3:336], w, 1e-6, residual=wide[:, 367:700])
    assert torch.equal(y, y3) and torch.equal(h, h3)
    y4, h4 = B.rms_norm(x.view(5, 8, 333), w, 1e-6, residual=res.view(5, 8, 333))
    assert y4.shape == (5, 8, 333) and torch.equal(y4.view(40, 333), y) and torch.equal(h4.view(40, 333), h)
    g = B.rms_norm_backward(x, h, w, 1e-6, dh=res)
    for again in (B.rms_norm_backward(x, h, w, 1e-6, dh=res), B.rms_norm_backward(wide[:, 3:336], h, w, 1e-6, dh=wide[:, 367:700])):
        assert all(torch.equal(m, n) for m, n in zip(g, again))


def test_the_product_takes_it(B):
    """What the norm leaves in 8 bits is what dfa_quantize would of the same fp32 rows, and goes into the product."""
    import torch
    x, w = _rows(1, 50, 640, "fp32"), _rows(2, 1, 640, "fp32")[0]
    (y, q), _ = B.rms_norm(x, w, 1e-6, quantized="both")
    again = B.quantize(y)
    assert torch.equal(q.values.view(torch.uint8), again.values.view(torch.uint8)) and torch.equal(q.scales[:, :50], again.scales[:, :50])
    weight = B.quantize(_rows(4, 96, 640, "fp32"), 128)
    assert torch.equal(B.quantized_product(q, weight, torch.float32), B.quantized_product(again, weight, torch.float32))


def test_refusals(B):
    import torch
    x, w = _rows(1, 4, 64, "bf16"), _rows(2, 1, 64, "bf16")[0]
    for bad in (lambda: B.rms_norm(x, w[:-1], 1e-6), lambda: B.rms_norm(x, w, -1.0), lambda: B.rms_norm(x, w, float("nan")), lambda: B.rms_norm(x, w, 1e-6, residual=x[:2]),
                lambda: B.rms_norm(x, w, 1e-6, residual=x.float()), lambda: B.rms_norm(x.half(), w, 1e-6), lambda: B.rms_norm(x.float(), w, 1e-6),
                lambda: B.rms_norm_backward(x, x[:, :32], w, 1e-6), lambda: B.rms_norm(x, w.half(), 1e-6), lambda: B.rms_norm_backward(x, x, w, 1e-6, workspace=None),
                lambda: B.rms_norm(torch.zeros((1, 32769), device="cuda"), None, 1e-6)):
        with pytest.raises(B.DfaError):
            bad()
    with pytest.raises(RuntimeError):
        B.rms_norm(x.cpu(), w, 1e-6)
    with pytest.raises(ValueError):
        B.rms_norm(x.t(), w[:4], 1e-6)


def test_captured(B):
    import torch
    x, res, w, dy = _rows(1, 600, 512, "bf16"), _rows(2, 600, 512, "bf16"), _rows(3, 1, 512, "bf16")[0], _rows(4, 600, 512, "bf16")
    B.rms_norm(x, w, 1e-6, residual=res, quantized="both")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        (y, q), h = B.rms_norm(x, w, 1e-6, residual=res, quantized="both")
        dx, dw = B.rms_norm_backward(dy, h, w, 1e-6, dh=res)
    for i in range(4):
        x.copy_(_rows(10 + i, 600, 512, "bf16"))
        graph.replay()
        (y2, q2), h2 = B.rms_norm(x, w, 1e-6, residual=res, quantized="both")
        dx2, dw2 = B.rms_norm_backward(dy, h2, w, 1e-6, dh=res)
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(h, h2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)
        assert torch.equal(q.values.view(torch.uint8), q2.values.view(torch.uint8)) and torch.equal(q.scales[:, :600], q2.scales[:, :600])


def test_offsets_beyond_32_bits(B):
    """More than 2^31 elements: the last rows as they come out on their own."""
    import torch
    M, C = 66000, 32768
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, w = torch.randn((M, C), generator=gen, device="cuda", dtype=torch.bfloat16), torch.randn((C,), generator=gen, device="cuda", dtype=torch.bfloat16)
    (y, q), h = B.rms_norm(x, w, 1e-6, residual=x, quantized="both")
    (y1, q1), h1 = B.rms_norm(x[-32:], w, 1e-6, residual=x[-32:], quantized="both")
    assert torch.equal(y[-32:], y1) and torch.equal(h[-32:], h1)
    assert torch.equal(q.values[-32:].view(torch.uint8), q1.values.view(torch.uint8)) and torch.equal(q.scales[:, M - 32:M], q1.scales[:, :32])
    dx, _ = B.rms_norm_backward(y, h, w, 1e-6)
    assert torch.equal(dx[-32:], B.rms_norm_backward(y1, h1, w, 1e-6)[0])
