"""GPU parity of the products of 8-bit operands (quantisation, product, projection, its gradients) against 64-bit references."""
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


def _torch_dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def _data(seed, shape, dtype, spread=3.0):
    """(tensor on the GPU, the same in fp64): normal values in rows and columns of unlike size."""
    import torch
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp2(spread * rng.standard_normal((shape[0], 1))) * np.exp2(rng.standard_normal((1, shape[1])))
    t = torch.from_numpy(x.astype(np.float32)).to(_torch_dtype(dtype)).cuda()
    return t, t.double().cpu().numpy()


def _codes(m):
    import torch
    return ref.NUMBERS[m.values.cpu().view(torch.uint8).numpy()]


def _check_quantized(m, x, block_rows):
    """values, scales and what stands behind the last column and row."""
    values, exps = ref.quantize(x, block_rows)
    R, C = x.shape
    got, scales = _codes(m), m.scales.cpu().numpy()
    assert m.cols == C and got.shape == (R, -(-C // 128) * 128)
    np.testing.assert_array_equal(got[:, :C], values)
    assert np.all(got[:, C:] == 0)
    np.testing.assert_array_equal(scales[:, :R].astype(np.int64) - 127, exps)
    assert np.all(scales[:, R:] == 1)


SIZES = [(1, 1), (1, 128), (3, 129), (16, 127), (17, 256), (128, 128), (130, 300), (257, 77), (64, 1000)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("R,C", SIZES)
def test_quantize(B, R, C, block_rows, dtype):
    x, xe = _data(R * 1000 + C, (R, C), dtype)
    _check_quantized(B.quantize(x, block_rows), xe, block_rows)
    _check_quantized(B.quantize(x, block_rows, transpose=True), xe.T, block_rows)
    both = B.quantize(x, block_rows, transpose="both")
    _check_quantized(both[0], xe, block_rows)
    _check_quantized(both[1], xe.T, block_rows)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_quantize_row_pitch_and_alignment(B, dtype):
    """Rows of a wider matrix, started at an odd element: read one by one, the same values."""
    import torch
    wide, we = _data(5, (70, 413), dtype)
    for first, cols in ((0, 256), (1, 256), (3, 200)):
        _check_quantized(B.quantize(wide[:, first:first + cols], 1, transpose=True), we[:, first:first + cols].T, 1)
        _check_quantized(B.quantize(wide[:, first:first + cols]), we[:, first:first + cols], 1)
    assert wide.dtype == _torch_dtype(dtype) and torch.isfinite(wide).all()


def test_quantize_ties_borders_and_extremes(B):
    """Halfway values, the largest magnitude just below, at and above 448 * 2^e, subnormal e4m3 and fp32 values, zeros, infinities and NaN."""
    import torch
    inf, nan = np.inf, np.nan
    step = np.array([448, 432, 434, 416 + 8, 17, 19, 1.0625, 1.1875, 2 ** -9, 1.5 * 2 ** -9, 2.5 * 2 ** -9, 2 ** -10, 1.1 * 2 ** -10, -0.0, -17, -2.5 * 2 ** -9])
    rows = [np.resize(step, 128), np.resize(step, 128) * 2.0 ** 100, np.resize(step, 128) * 2.0 ** -110, np.zeros(128)]
    for top in (448.0, np.nextafter(np.float32(448), np.float32(500)), 447.99, 3.4028234e38, 1e-38, 1e-45, 2.0 ** -118, 448 * 2.0 ** -126):
        r = np.linspace(-1, 1, 128) * float(top)
        rows.append(r)
    weird = np.linspace(-3, 5, 128)
    weird[[0, 5, 9]] = inf, -inf, nan
    rows += [weird, np.full(128, nan), np.full(128, inf)]
    x = torch.from_numpy(np.array(rows, dtype=np.float32)).cuda()
    xe = x.double().cpu().numpy()
    _check_quantized(B.quantize(x), xe, 1)
    _check_quantized(B.quantize(x.t().contiguous(), transpose=True), xe, 1)
    _check_quantized(B.quantize(x, 128), xe, 128)
    xb = x.to(torch.bfloat16)
    _check_quantized(B.quantize(xb), xb.double().cpu().numpy(), 1)


# sizes at the edges of tiles, k-steps and their shares: one of everything, one k-step, odd counts, tiles of both sizes, long k on few tiles
PRODUCTS = [(1, 1, 1), (5, 3, 130), (128, 128, 128), (129, 127, 257), (64, 200, 1024), (300, 520, 384), (256, 256, 4096), (1000, 130, 640), (70, 70, 5000)]


@pytest.mark.parametrize("M,N,K", PRODUCTS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_product(B, M, N, K, dtype):
    a, _ = _data(M + 7 * N + K, (M, K), "bf16")
    b, _ = _data(M + 7 * N + K + 1, (N, K), "bf16", spread=1.0)
    qa, qb = B.quantize(a), B.quantize(b, 128)
    ae, be = ref.matrix(qa), ref.matrix(qb)
    y = B.quantized_product(qa, qb, _torch_dtype(dtype))
    want = ae @ be.T
    err, bar = np.abs(y.double().cpu().numpy() - want), ref.product_bar(ae, be, want, dtype)
    print(f"[product {M}x{N}x{K} {dtype}] worst err/bar {float((err / bar).max()):.3f}", flush=True)
    assert np.all(err <= bar)


def test_product_of_many_tiles(B):
    """Enough 256-row tiles to be chosen, ragged at both ends, on values whose sums are exact: every element is equal."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    M, N, K = 4096 + 17, 4096 - 55, 300
    a = torch.randint(-4, 5, (M, K), generator=gen, device="cuda").to(torch.bfloat16)
    b = torch.randint(-4, 5, (N, K), generator=gen, device="cuda").to(torch.bfloat16)
    y = B.quantized_product(B.quantize(a), B.quantize(b), torch.float32)
    assert torch.equal(y, a.float() @ b.float().t())


def test_product_selects_rows_and_columns(B):
    """One 1 per row: any wrong row, feature, k or scale in the tiling shows as a misplaced element."""
    import torch
    M, N, K = 300, 384, 384
    a, ae = _data(11, (M, K), "bf16", spread=6.0)
    perm = torch.randperm(K, generator=torch.Generator().manual_seed(5))
    eye = torch.eye(K, dtype=torch.bfloat16)[perm].cuda()
    y = B.quantized_product(B.quantize(a), B.quantize(eye), torch.float32)
    np.testing.assert_array_equal(y.double().cpu().numpy(), ref.held(ae)[:, perm.numpy()])
    y = B.quantized_product(B.quantize(eye), B.quantize(a), torch.float32)
    np.testing.assert_array_equal(y.double().cpu().numpy(), ref.held(ae)[:, perm.numpy()].T)


LINEARS = [(1, 64, 64), (1, 130, 1), (2, 1533, 1000), (16, 48, 4096), (17, 100, 129), (31, 257, 640), (33, 64, 2000), (64, 96, 768), (65, 96, 768), (333, 153, 1000),
           (9, 40, 8000), (16, 200, 600), (24, 33, 5000), (50, 64, 8192), (64, 1024, 6001)]


@pytest.mark.parametrize("M,N,K", LINEARS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_linear(B, M, N, K, dtype):
    x, xe = _data(M + N + K, (M, K), dtype)
    w, _ = _data(M + N + K + 1, (N, K), "bf16", spread=1.0)
    qw = B.quantize(w, 128)
    we, xh = ref.matrix(qw), ref.held(xe)
    want = xh @ we.T
    bar = ref.product_bar(xh, we, want, dtype)
    y = B.quantized_linear(x, qw)
    assert y.dtype == x.dtype and np.all(np.abs(y.double().cpu().numpy() - want) <= bar)
    # rows of wider matrices, results into a wider one, odd starts: the same bits
    import torch
    wide_x = torch.zeros((M, K + 3), dtype=x.dtype, device="cuda")
    wide_x[:, 1:K + 1] = x
    wide_y = torch.full((M, N + 5), 7.0, dtype=x.dtype, device="cuda")
    B.quantized_linear(wide_x[:, 1:K + 1], qw, out=wide_y[:, 3:N + 3])
    assert torch.equal(wide_y[:, 3:N + 3], y) and bool((wide_y[:, :3] == 7).all()) and bool((wide_y[:, N + 3:] == 7).all())


def test_linear_not_finite_stays_in_its_row(B):
    import torch
    for M in (5, 200):
        x, _ = _data(M, (M, 256), "bf16")
        w, _ = _data(M + 1, (96, 256), "bf16")
        qw = B.quantize(w, 128)
        clean = B.quantized_linear(x, qw)
        x2 = x.clone()
        x2[3, 17], x2[4, 200] = float("inf"), float("nan")
        y = B.quantized_linear(x2, qw)
        assert bool(torch.isnan(y[3:5]).all())
        rest = [r for r in range(M) if r not in (3, 4)]
        assert torch.equal(y[rest], clean[rest])


@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (50, 130, 70), (128, 256, 384), (1000, 384, 200), (2100, 100, 333)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_linear_backward(B, M, N, K, dtype):
    x, xe = _data(M + N, (M, K), dtype, spread=1.0)
    dy, dye = _data(M + N + 1, (M, N), dtype, spread=1.0)
    w, we = _data(M + N + 2, (N, K), "bf16", spread=1.0)
    w_t = B.quantize(w, 128, transpose=True)
    np.testing.assert_array_equal(ref.matrix(w_t), ref.matrix(B.quantize(w, 128)).T)
    wte = ref.matrix(w_t)
    dx, dw = B.quantized_linear_backward(dy, x, w_t)
    dyh = ref.held(dye)
    want = dyh @ wte.T
    assert dx.dtype == x.dtype and np.all(np.abs(dx.double().cpu().numpy() - want) <= ref.product_bar(dyh, wte, want, dtype))
    dyt, xt = ref.held(dye.T), ref.held(xe.T)
    want = dyt @ xt.T
    assert np.all(np.abs(dw.double().cpu().numpy() - want) <= ref.product_bar(dyt, xt, want, "fp32"))
    import torch
    only_dx, none = B.quantized_linear_backward(dy, x, w_t, want_dw=False)
    assert none is None and torch.equal(only_dx, dx)
    none, only_dw = B.quantized_linear_backward(dy, x, w_t, want_dx=False)
    assert none is None and torch.equal(only_dw, dw)


def test_linear_backward_against_differences(B):
    """On small whole numbers quantisation changes nothing and every sum is exact: the loss sum(dy * y) is linear in x and in w, so its
    differences are the gradients, element by element."""
    import torch
    rng = np.random.default_rng(9)
    M, N, K = 70, 24, 40
    ints = lambda *shape: torch.from_numpy(rng.integers(-3, 4, shape).astype(np.float32)).cuda()
    x, w, dy = ints(M, K), ints(N, K), ints(M, N)
    loss = lambda x, w: float((B.quantized_linear(x, B.quantize(w, 128)).double() * dy.double()).sum())
    dx, dw = B.quantized_linear_backward(dy, x, B.quantize(w, 128, transpose=True))
    base = loss(x, w)
    for i, j in ((0, 0), (69, 39), (33, 7)):
        x2 = x.clone()
        x2[i, j] += 1
        assert loss(x2, w) - base == float(dx[i, j])
    for i, j in ((0, 0), (23, 39), (11, 20)):
        w2 = w.clone()
        w2[i, j] += 1
        assert loss(x, w2) - base == float(dw[i, j])


def test_linear_repeats_captured_and_on_streams(B):
    """Equal calls give equal bits; a captured call replays on new inputs beside eager work; two streams with a workspace each."""
    import torch
    x, _ = _data(1, (300, 1024), "bf16")
    w, _ = _data(2, (200, 1024), "bf16")
    qw = B.quantize(w, 128)
    w_t = B.quantize(w, 128, transpose=True)
    few = x[:9].clone()
    dy = torch.randn((300, 200), device="cuda").to(torch.bfloat16)
    eager = lambda: (B.quantized_linear(x, qw), B.quantized_linear(few, qw), *B.quantized_linear_backward(dy, x, w_t))
    first = eager()
    assert all(torch.equal(a, b) for a, b in zip(first, eager()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = eager()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = eager()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    for trip in range(4):
        x.copy_(torch.randn((300, 1024), device="cuda"))
        few.copy_(x[:9])
        graph.replay()
        again = eager()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, again)), trip


def test_refusals(B):
    import torch
    x, _ = _data(1, (80, 256), "bf16")
    qw = B.quantize(torch.randn((64, 256), device="cuda"), 128)
    with pytest.raises(B.DfaError):
        B.quantized_linear(x[:, :128], qw)
    with pytest.raises(B.DfaError):
        B.quantized_linear(x.half(), qw)
    with pytest.raises(B.DfaError):
        B.quantized_linear(x, B.QuantizedMatrix(qw.values, qw.scales[:1], 256))
    with pytest.raises(TypeError):
        B.quantized_linear(x, B.QuantizedMatrix(qw.values.view(torch.uint8), qw.scales, 256))
    with pytest.raises(ValueError):
        B.quantized_linear(x.t()[:64], qw)
    with pytest.raises(B.DfaError):
        B.quantized_linear(x, qw, out=torch.empty((80, 63), dtype=x.dtype, device="cuda"))
    with pytest.raises(B.DfaError) as e:
        B.quantized_linear(x, qw, workspace=torch.empty((64,), dtype=torch.uint8, device="cuda"))
    assert e.value.code == B.DFA_ERR_WORKSPACE
    with pytest.raises(B.DfaError):
        B.quantized_linear(x[:0], qw)
    with pytest.raises(B.DfaError):
        B.quantize(x, 64)
    with pytest.raises(RuntimeError):
        B.quantize(x.cpu())
    with pytest.raises(B.DfaError):
        B.quantized_linear_backward(x, x, qw)
