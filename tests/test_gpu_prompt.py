"""Attention within packed sequences and its gradients against 64-bit references; bounds in packed_ref."""
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


def _make(seed, T, H, Hkv, D, dtype, std=1.0):
    """q, k, v as heads of one projection's result, and dout."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = (std * torch.randn((T, H + 2 * Hkv, D), generator=gen, device="cuda")).to(_type(dtype))
    dout = torch.randn((T, H, D), generator=gen, device="cuda").to(_type(dtype))
    return x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], dout


def _ints(values):
    import torch
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _within(got, want, tol, what):
    import torch
    got = got.double()
    fine = want.isfinite()
    assert torch.equal(got.isfinite(), fine), what
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or over.max().item() <= 0, f"{what}: {over.max().item():.3e} over its bound"


def _check(B, lengths, H, Hkv, D, dtype, causal, behind=0, seed=0, std=1.0, backward=True):
    import torch
    starts = ref.starts_of(lengths)
    T = starts[-1] + behind
    q, k, v, dout = _make(seed, T, H, Hkv, D, dtype, std)
    scale = D ** -0.5
    out, lse = B.prompt_attention(q, k, v, _ints(starts), scale, causal)
    o, l, o_tol, l_tol = ref.attention(q, k, v, starts, scale, causal)
    _within(out, o, o_tol, "out")
    _within(lse, l, l_tol, "lse")
    assert (out[starts[-1]:] == 0).all() and torch.isneginf(lse[:, starts[-1]:]).all()
    if not backward:
        return
    grads = B.prompt_attention_backward(q, k, v, out, lse, dout, _ints(starts), scale, causal)
    want, tols = ref.attention_backward(q, k, v, out, lse, dout, starts, scale, causal)
    for got, g, t, name in zip(grads, want, tols, ("dq", "dk", "dv")):
        _within(got, g, t, name)
        assert (got[starts[-1]:] == 0).all(), name


LENGTHS = [[1], [2], [31], [32, 33], [63, 64, 65], [127, 128, 129], [255, 0, 257], [0, 0, 5, 0], [1] * 70 + [40], [300, 1, 90]]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "-".join(map(str, x[:4])))
def test_lengths(B, lengths, causal, D, dtype):
    _check(B, lengths, 3, 3, D, dtype, causal, behind=len(lengths) % 3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (4, 1), (6, 2), (8, 8), (16, 8), (24, 8), (5, 1), (40, 5)])
def test_heads(B, H, Hkv, dtype):
    """Groups of query heads, numbers of heads that dies share evenly and not; dk and dv summed over a group."""
    _check(B, [70, 150], H, Hkv, 64 if H % 3 else 128, dtype, True, behind=3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_long(B, D, dtype):
    _check(B, [1500, 37], 2, 1, D, dtype, True, behind=200)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_many_tiles(B, D, causal, dtype):
    """Launches of many workgroups: larger tiles, dk and dv of a whole group in one workgroup."""
    _check(B, [40] * 60 + [200] + [7] * 10, 16, 8, D, dtype, causal, behind=70)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [384, 449, 640])
def test_one_prompt(B, n, D, causal, dtype):
    """Few tiles of a long walk: waves share it out."""
    _check(B, [n], 2, 1, D, dtype, causal, backward=n == 449)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lengths,H,Hkv", [([40] * 43 + [130, 7], 16, 8), ([500, 300, 200], 24, 24), ([500, 300, 200], 8, 4)], ids=["short", "long", "fewer"])
def test_some_tiles(B, lengths, H, Hkv, D, causal, dtype):
    """More tiles than the chip holds at once, but not many times as many."""
    _check(B, lengths, H, Hkv, D, dtype, causal, behind=3)


@pytest.mark.parametrize("causal,n", [(True, 2090), (False, 1500)])
@pytest.mark.parametrize("D", [64, 128])
def test_many_tiles_of_long_walks(B, D, causal, n):
    _check(B, [n], 96, 8, D, "bf16", causal, behind=10, backward=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_sequences(B, dtype):
    """More sequences than a wave has lanes, than are ranked, and than 64 times 64."""
    _check(B, [3] * 100 + [130] + [2] * 100, 1, 1, 64, dtype, True)
    _check(B, [3] * 300, 1, 1, 64, dtype, True, behind=40)
    _check(B, [1, 0] * 2500 + [90], 1, 1, 64, dtype, True, backward=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_large_scores(B, D, dtype):
    """Scores of hundreds: one key carries a row."""
    _check(B, [200, 100], 2, 2, D, dtype, True, std=8.0, backward=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_climbing_scores(B, D, dtype):
    """Every block's scores are far above those before it: the reference exponent moves each time."""
    import torch
    n = 200
    q, k, v, _ = _make(3, n, 1, 1, D, dtype)
    q = torch.ones_like(q)
    k = (torch.arange(n, device="cuda", dtype=torch.float32)[:, None, None] * 0.25 * torch.ones((1, 1, D), device="cuda")).to(q.dtype)
    out, lse = B.prompt_attention(q, k, v, _ints([0, n]), D ** -0.5, True)
    o, l, o_tol, l_tol = ref.attention(q, k, v, [0, n], D ** -0.5, True)
    _within(out, o, o_tol, "out")
    _within(lse, l, l_tol, "lse")


# two sequences of a few tiles; one whose walk waves share; many tiles; many tiles of long walks (the value lies in the second sequence, row 50 of it, or in the only one)
@pytest.mark.parametrize("lengths,H,at", [([150, 140], 4, 200), ([600], 4, 500), ([150] + [90] * 69, 16, 200), ([2090], 64, 1995)], ids=["few", "shared", "many", "long"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_values_behind_the_mask(B, value, D, dtype, lengths, H, at):
    """A value or key that is not finite reaches the rows that see it, in that head group, and no other."""
    import torch
    starts = ref.starts_of(lengths)
    T, end = starts[-1], next(s for s in starts if s > at)
    q, k, v, _ = _make(5, T, H, H // 2, D, dtype)
    clean = B.prompt_attention(q, k, v, _ints(starts), D ** -0.5, True)
    sees = torch.zeros((T,), dtype=torch.bool, device="cuda")
    sees[at:end] = True
    for tensor in ("v", "k"):
        k2, v2 = k.clone(), v.clone()
        (v2 if tensor == "v" else k2)[at, 1, 7] = value
        out, lse = B.prompt_attention(q, k2, v2, _ints(starts), D ** -0.5, True)
        hit = torch.zeros((T, H), dtype=torch.bool, device="cuda")
        hit[:, 2:4] = sees[:, None]
        # rows of another head, sequence, or before it: the same weights over the same values, each side within the bounds of n keys with |v| < 6
        off = 2 * 6 * ((7 * max(lengths) + 80) * ref.E + (ref.U[out.dtype] if dtype == "bf16" else 0.0))
        torch.testing.assert_close(out[~hit].float(), clean[0][~hit].float(), rtol=2 * ref.U[out.dtype], atol=off)
        torch.testing.assert_close(lse.t()[~hit], clean[1].t()[~hit], rtol=1e-6, atol=2 * (max(lengths) + 66) * ref.E)
        if tensor == "v":
            got = out[hit].float()
            assert (~got[:, 7].isfinite()).all() and got[:, :7].isfinite().all() and got[:, 8:].isfinite().all()
            if value == value and dtype == "bf16":        # (in parts an infinite number may come out as NaN)
                assert (got[:, 7] == value).all()


def test_rows_see_only_their_own(B):
    """Neighbouring sequences of huge values change nothing."""
    import torch
    starts = [0, 50, 130, 150]
    q, k, v, dout = _make(6, 150, 2, 1, 64, "bf16")
    x = [t.clone() for t in (q, k, v)]
    for t in x:
        t[:50] *= 1e4
        t[130:] = float("nan")
    a = B.prompt_attention(q, k, v, _ints(starts), 0.125)
    b = B.prompt_attention(*x, _ints(starts), 0.125)
    assert torch.equal(a[0][50:130], b[0][50:130]) and torch.equal(a[1][:, 50:130], b[1][:, 50:130])
    ga = B.prompt_attention_backward(q, k, v, *a, dout, _ints(starts), 0.125)
    gb = B.prompt_attention_backward(*x, *b, dout, _ints(starts), 0.125)
    assert all(torch.equal(m[50:130], n[50:130]) for m, n in zip(ga, gb))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_least_and_largest_scale(B, dtype):
    """Powers of two that leave every product as it was leave every result so, but for their own factor."""
    import torch
    starts = _ints([0, 70, 200])
    q, k, v, dout = _make(9, 200, 4, 2, 64, dtype)
    q = q * 0.25

    def run(by):
        a, b = q * by, k * by
        out, lse = B.prompt_attention(a, b, v, starts, 1.0 / (by * by))
        dq, dk, dv = B.prompt_attention_backward(a, b, v, out, lse, dout, starts, 1.0 / (by * by))
        return out, lse, dq * by, dk * by, dv

    plain = run(1.0)
    for by in (2.0 ** 50, 2.0 ** -50):
        for a, b in zip(run(by), plain):
            assert a.isfinite().all() and torch.equal(a, b)


def test_starts_out_of_range(B):
    """Starts outside the rows count as the nearest; the first is 0."""
    import torch
    q, k, v, _ = _make(7, 100, 2, 2, 64, "bf16")
    a = B.prompt_attention(q, k, v, _ints([0, 40, 100]), 0.125)
    b = B.prompt_attention(q, k, v, _ints([7, 40, 2 ** 30]), 0.125)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c = B.prompt_attention(q, k, v, _ints([0, -5, -3]), 0.125)
    assert (c[0] == 0).all() and torch.isneginf(c[1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_equal_calls_strides_and_given_results(B, dtype):
    """Equal calls give equal bits; heads may lie apart, heads before rows; results may be given."""
    import torch
    starts = _ints([0, 90, 210])
    q, k, v, dout = _make(8, 210, 8, 2, 64, dtype)
    out, lse = B.prompt_attention(q, k, v, starts, 0.125)
    grads = B.prompt_attention_backward(q, k, v, out, lse, dout, starts, 0.125)
    turned = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    given = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    for args, kw in (((q, k, v), {}), (turned, {}), ((q, k, v), dict(out=given[0], lse=given[1]))):
        o, l = B.prompt_attention(*args, starts, 0.125, **kw)
        assert torch.equal(o, out) and torch.equal(l, lse)
        again = B.prompt_attention_backward(*args, o, l, dout, starts, 0.125)
        assert all(torch.equal(a, b) for a, b in zip(again, grads))
    assert B.prompt_attention(q, k, v, starts, 0.125, want_lse=False)[1] is None


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_gradients_against_differences(B, dtype):
    """Directional derivatives of sum(out * dout), by central differences of the 64-bit forward."""
    import torch
    starts = [0, 40, 75]
    q, k, v, dout = _make(9, 75, 4, 2, 64, dtype)
    out, lse = B.prompt_attention(q, k, v, _ints(starts), 0.125)
    grads = B.prompt_attention_backward(q, k, v, out, lse, dout, _ints(starts), 0.125)
    _, tols = ref.attention_backward(q, k, v, out, lse, dout, starts, 0.125, True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i in range(3):
        way = torch.randn(grads[i].shape, generator=gen, device="cuda", dtype=torch.float64)

        def value(step):
            x = [t.double() for t in (q, k, v)]
            x[i] = x[i] + step * way
            total = 0.0
            for a, b in ref.sequences(starts):
                for h in range(4):
                    z = (x[0][a:b, h] @ x[1][a:b, h // 2].t()) * 0.125
                    z = z.masked_fill(torch.ones_like(z, dtype=torch.bool).triu(1), float("-inf"))
                    total = total + ((z.softmax(1) @ x[2][a:b, h // 2]) * dout[a:b, h].double()).sum()
            return total

        slope = (value(1e-5) - value(-1e-5)) / 2e-5
        got = (grads[i].double() * way).sum()
        # the gradient's own bound, and delta from the rounded out: dout . (its rounding) on every P, which the formula takes as given
        o_off = ref.U[out.dtype] * (out.double().abs() * dout.double().abs()).sum(2).amax() * way.abs().max() * out.numel() * 0.125 * max(t.double().abs().max() for t in (q, k))
        assert (got - slope).abs() <= (tols[i] * way.abs()).sum() + (o_off if i < 2 else 0.0) + 1e-6 * slope.abs() + 1e-6


def test_captured(B):
    """A captured forward and backward serve other lengths when they are replayed, beside eager work on another stream."""
    import torch
    T = 256
    q, k, v, dout = _make(10, T, 8, 2, 64, "bf16")
    starts = _ints([0, 100, 180, 250])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.prompt_attention(q, k, v, starts, 0.125)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = B.prompt_attention(q, k, v, starts, 0.125)
        grads = B.prompt_attention_backward(q, k, v, out, lse, dout, starts, 0.125)
    for lengths in ([100, 80, 70], [1, 0, 255], [0, 0, 0], [256, 0, 0], [100, 80, 70]):
        starts.copy_(_ints(ref.starts_of(lengths)))
        graph.replay()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            want = B.prompt_attention(q, k, v, starts, 0.125)
            want_grads = B.prompt_attention_backward(q, k, v, *want, dout, starts, 0.125)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and all(torch.equal(a, b) for a, b in zip(grads, want_grads)), lengths


@pytest.mark.parametrize("dtype,T", [("bf16", 140000), ("fp32", 70000)])
def test_offsets_beyond_32_bits(B, dtype, T):
    """Tensors of more than 2^31 elements (bf16) and bytes: the last sequences, and the rows behind them, against references and the same rows on their own."""
    import torch
    H, Hkv, D = 128, 2, 128
    lengths = [50] * (T // 50 - 1) + [33, 7]
    starts = ref.starts_of(lengths)
    gen = torch.Generator(device="cuda").manual_seed(12)
    rand = lambda heads: torch.randn((T, heads, D), generator=gen, device="cuda", dtype=_type(dtype))
    q, k, v, dout = rand(H), rand(Hkv), rand(Hkv), rand(H)
    out, lse = B.prompt_attention(q, k, v, _ints(starts), 0.1)
    grads = B.prompt_attention_backward(q, k, v, out, lse, dout, _ints(starts), 0.1)
    first, end = starts[-4], starts[-1]
    cut = [s - first for s in starts[-4:]]
    own = [t[first:end] for t in (q, k, v)]
    o, l, o_tol, l_tol = ref.attention(*own, cut, 0.1, True)
    _within(out[first:end], o, o_tol, "out")
    _within(lse[:, first:end], l, l_tol, "lse")
    want, tols = ref.attention_backward(*own, out[first:end], lse[:, first:end], dout[first:end], cut, 0.1, True)
    for got, g, t, name in zip(grads, want, tols, ("dq", "dk", "dv")):
        _within(got[first:end], g, t, name)
    assert end < T and not out[end:].any() and torch.isneginf(lse[:, end:]).all() and not any(g[end:].any() for g in grads)
