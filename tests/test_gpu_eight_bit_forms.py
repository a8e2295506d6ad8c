"""Every form that the operators on 8-bit operands take, on ragged sizes (eight_bit_forms.py): each test names the form that it means and runs it."""
import numpy as np
import pytest

import cache_ref
import eight_bit_forms as forms
import quantized_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


def _type(dtype):
    import torch
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]


def _held(m):
    """What a QuantizedMatrix holds, fp64 on the GPU."""
    import torch
    unit = torch.exp2(m.scales[:, :m.values.shape[0]].double() - 127).t().repeat_interleave(128, 1)
    return (m.values.double() * unit[:, :m.values.shape[1]])[:, :m.cols]


def _whole(gen, rows, cols, by_row=5):
    """Whole numbers of -4 .. 4 times a power of two that changes from row to row and from block of 128 columns to the next: e4m3 blocks hold them exactly,
    and so do fp32 sums of products of them (each row's power is common to all terms of a sum)."""
    import torch
    x = torch.randint(-4, 5, (rows, cols), generator=gen, device="cuda").float()
    x *= torch.exp2((torch.arange(rows, device="cuda") * 7 // 3 % by_row).float())[:, None]
    return x * torch.exp2((torch.arange(cols, device="cuda") // 128 % 2).float())[None, :]


def _uneven(gen, rows, cols):
    import torch
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    x *= torch.exp2(2 * torch.randn((rows, 1), generator=gen, device="cuda"))
    return x * torch.exp2(torch.randn((1, cols), generator=gen, device="cuda"))


def _bar(a, b, y, dtype):
    """quantized_ref.product_bar, on the GPU."""
    import torch
    K = a.shape[1]
    mag = a.abs() @ b.abs().t()
    bar = K * 2.0 ** -24 * mag * 1.01 + 1e-45
    if dtype == "bf16":
        for k in range(0, K, 16):
            most = torch.zeros_like(bar)
            for i in range(k, min(k + 16, K)):
                torch.maximum(most, a[:, i, None].abs() * b[None, :, i].abs(), out=most)
            bar += 16 * 2.0 ** -13 * most
    return bar * 1.01 + ref.HALF_STEP[dtype] * y.abs()


def _rounded(y, dtype):
    return y.float().to(_type(dtype))                        # (whole sums below 2^24: fp32 holds them)


@pytest.mark.parametrize("dtype,M,N,K,tile,splits", forms.PRODUCTS)
def test_product(B, dtype, M, N, K, tile, splits):
    """Every element equal on whole numbers; random operands within the bar."""
    import torch
    assert forms.product(B, dtype, M, N, K) == (tile, splits)
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    for draw in (_whole, _uneven):
        qa, qb = B.quantize(draw(gen, M, K)), B.quantize(draw(gen, N, K))
        a, b = _held(qa), _held(qb)
        want = a @ b.t()
        got = B.quantized_product(qa, qb, _type(dtype))
        if draw is _whole:
            assert (want.abs() < 2.0 ** 30).all()            # 2^24 times the rows' powers
            assert torch.equal(got, _rounded(want, dtype))
        else:
            bar = _bar(a, b, want, dtype)
            worst = float(((got.double() - want).abs() / bar).max())
            print(f"[product {dtype} {M}x{N}x{K} {tile}/{splits}] worst err/bar {worst:.3f}", flush=True)
            assert worst <= 1


@pytest.mark.parametrize("dtype,M,N,K,blocks,tile", forms.LINEARS)
def test_linear(B, dtype, M, N, K, blocks, tile):
    """The same; a result in the middle of a wider matrix leaves what is around it."""
    import torch
    assert forms.linear(B, dtype, M, N, K) == (blocks, tile)
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    for draw in (_whole, _uneven):
        x = draw(gen, M, K).to(_type(dtype))
        qw = B.quantize(draw(gen, N, K), 1 if draw is _whole else 128)
        xh, w = _held(B.quantize(x)), _held(qw)
        want = xh @ w.t()
        wide = torch.full((M + 2, N + 3), 7.0, dtype=x.dtype, device="cuda")
        got = B.quantized_linear(x, qw, out=wide[1:M + 1, 1:N + 1])
        assert bool((wide[0] == 7).all()) and bool((wide[-1] == 7).all()) and bool((wide[:, 0] == 7).all()) and bool((wide[:, N + 1:] == 7).all())
        assert torch.equal(got, B.quantized_linear(x, qw))
        if draw is _whole:
            assert torch.equal(got, _rounded(want, dtype))
        else:
            worst = float(((got.double() - want).abs() / _bar(xh, w, want, dtype)).max())
            print(f"[linear {dtype} {M}x{N}x{K} {blocks} {tile}] worst err/bar {worst:.3f}", flush=True)
            assert worst <= 1


@pytest.mark.parametrize("dtype,M,N,K,dx_form,dw_form,paired", forms.GRADIENTS)
def test_gradients(B, dtype, M, N, K, dx_form, dw_form, paired):
    import torch
    assert forms.gradients(B, dtype, M, N, K) == (dx_form, dw_form, paired)
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    for draw in (_whole, _uneven):
        # (one power for all rows: rows are what dw sums over)
        dy, x = (_whole(gen, M, n, 1).to(_type(dtype)) if draw is _whole else draw(gen, M, n).to(_type(dtype)) for n in (N, K))
        qt = B.quantize(draw(gen, K, N))
        dyh, wt, dyt, xt = (_held(m) for m in (B.quantize(dy), qt, B.quantize(dy, transpose=True), B.quantize(x, transpose=True)))
        both = B.quantized_linear_backward(dy, x, qt)
        alone = B.quantized_linear_backward(dy, x, qt, want_dw=False)[0], B.quantized_linear_backward(dy, x, qt, want_dx=False)[1]
        for got, only, a, b, kind in ((both[0], alone[0], dyh, wt, dtype), (both[1], alone[1], dyt, xt, "fp32")):
            want = a @ b.t()
            assert got.dtype == _type(kind) and torch.equal(got, only)
            if draw is _whole:
                assert torch.equal(got, _rounded(want, kind))
            else:
                worst = float(((got.double() - want).abs() / _bar(a, b, want, kind)).max())
                print(f"[gradient {dtype} {M}x{N}x{K} {dx_form} {dw_form}] worst err/bar {worst:.3f}", flush=True)
                assert worst <= 1


def _filled(B, rng, Bsz, heads, page, D, tokens, std=1.0):
    """A cache whose sequences hold that many tokens in pages in no order, what else there is random bytes: (cache, model, table on the GPU, table)."""
    import torch
    width = -(-tokens // page) + 1
    pages = Bsz * width + 2
    byte = lambda *shape: torch.from_numpy(rng.integers(0, 256, shape).astype(np.uint8)).cuda()
    cache = B.KvCache(byte(pages, heads, page, D).view(torch.float8_e4m3fn), byte(pages, heads, D, page).view(torch.float8_e4m3fn), byte(pages, heads, 2))
    table = rng.permutation(pages)[:Bsz * width].reshape(Bsz, width).astype(np.int32)
    on_gpu = torch.from_numpy(table).cuda()
    k, v = (torch.from_numpy((s * rng.standard_normal((Bsz, tokens, heads, D))).astype(np.float32)).cuda() for s in (std, 1.0))
    B.cache_append(k, v, cache, on_gpu, torch.full((Bsz,), tokens, dtype=torch.int32, device="cuda"))
    return cache, cache_ref.Model(cache), on_gpu, table


@pytest.mark.parametrize("dtype,Bsz,M,H,heads,D,page,tokens,rows,tiles,splits", forms.ATTENTIONS)
def test_attention(B, dtype, Bsz, M, H, heads, D, page, tokens, rows, tiles, splits):
    """Causal and not, the sequences of unlike lengths, ragged counts."""
    import torch
    assert forms.attention(B, dtype, Bsz, M, H, heads, D, page, tokens) == (rows, tiles, splits)
    rng = np.random.default_rng(M + H + D + tokens)
    cache, model, on_gpu, table = _filled(B, rng, Bsz, heads, page, D, tokens)
    lengths = [max(tokens - 41 * b, 1) for b in range(Bsz)]
    counts = [M if b % 3 == 0 else max(M - 5 * b, 0) for b in range(Bsz)]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    q = torch.from_numpy(rng.standard_normal((Bsz, M, H, D)).astype(np.float32)).to(_type(dtype)).cuda()
    qe = q.double().cpu().numpy()
    for causal, n in ((True, counts), (False, None)):
        want = cache_ref.attention(model, qe, table, lengths, D ** -0.5, causal, n)
        args = (q, cache, on_gpu, ints(lengths), D ** -0.5)
        out, lse = B.cache_attention(*args, causal=causal, counts=None if n is None else ints(n))
        worst = cache_ref.check_attention(out, lse, want, dtype)
        print(f"[attention {dtype} {Bsz} {M} {H}/{heads} {D} {page} {tokens}: {rows} rows] worst err/bar {worst:.3f}", flush=True)
        again = B.cache_attention(*args, causal=causal, counts=None if n is None else ints(n))
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("M,tokens,splits", [(33, 3000, True), (47, 3000, True), (48, 200, False)])
def test_attention_48_rows_not_finite(B, M, tokens, splits):
    """NaN keys and values among the last tokens and a NaN in a query, in tiles of 48 rows: they reach the rows that attend to them and no others."""
    import torch
    rng = np.random.default_rng(M)
    Bsz, heads, page, D = (1, 12, 16, 64) if splits else (16, 12, 16, 64)
    assert forms.attention(B, "bf16", Bsz, M, heads, heads, D, page, tokens) == (48, False, splits)
    cache, _, on_gpu, table = _filled(B, rng, Bsz, heads, page, D, tokens, 8.0)
    place = lambda n: (int(table[0, n // page]), n % page)
    kb, vb = cache.k.view(torch.uint8), cache.v.view(torch.uint8)
    (p, s), (p2, s2) = place(tokens - 3), place(tokens - 20)
    kb[p, 3, s, 7] = 0x7f
    vb[p2, 5, 11, s2] = 0xff
    q = torch.from_numpy((8 * rng.standard_normal((Bsz, M, heads, D))).astype(np.float32)).to(torch.bfloat16).cuda()
    q[0, M - 2, 7, 3] = float("nan")
    qe = q.double().cpu().numpy()
    lengths = [tokens] * Bsz
    want = cache_ref.attention(cache_ref.Model(cache), qe, table, lengths, 1.0, True)
    assert np.isnan(want[0][0, -1, 3]).all() and np.isfinite(want[0][0, :M - 20]).all() and np.isnan(want[0][0, -1, 5]).sum() == 1
    out, lse = B.cache_attention(q, cache, on_gpu, torch.tensor(lengths, dtype=torch.int32, device="cuda"), 1.0)
    cache_ref.check_attention(out, lse, want, "bf16")
