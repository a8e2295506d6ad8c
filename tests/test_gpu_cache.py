"""GPU parity of the cache of keys and values in e4m3 (appending, attention over it) against 64-bit references."""
import numpy as np
import pytest

import cache_ref
import quantized_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


def _tensor(rng, shape, dtype, std=1.0):
    import torch
    t = torch.from_numpy((std * rng.standard_normal(shape)).astype(np.float32)).to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]).cuda()
    return t, t.double().cpu().numpy()


def _garbage(B, rng, pages, heads, page, D, scale_bytes=(0, 256)):
    """A cache of random bytes, NaN among them: what memory may hold before anything is written."""
    import torch
    byte = lambda *shape: torch.from_numpy(rng.integers(0, 256, shape).astype(np.uint8)).cuda()
    return B.KvCache(byte(pages, heads, page, D).view(torch.float8_e4m3fn), byte(pages, heads, D, page).view(torch.float8_e4m3fn), torch.from_numpy(rng.integers(*scale_bytes, (pages, heads, 2)).astype(np.uint8)).cuda())


def _ints(values):
    import torch
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _table(rng, Bsz, width, pages):
    return rng.permutation(pages)[:Bsz * width].reshape(Bsz, width).astype(np.int32)


APPENDS = [  # heads, page, D, rows per step
    (1, 16, 64, [1, 1, 20, 1, 3, 40]), (3, 32, 64, [33, 1, 1, 64, 7]), (2, 64, 64, [1] * 5 + [130, 62, 1]), (2, 128, 64, [100, 30, 1, 128]),
    (2, 16, 128, [5, 16, 1, 1]), (1, 32, 128, [31, 1, 1, 70]), (4, 64, 128, [64, 1, 63, 1]), (1, 128, 128, [1, 127, 1, 200])]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,page,D,steps", APPENDS)
def test_append(B, heads, page, D, steps, dtype):
    """Step by step from garbage: scales that grow and do not, pages entered at any slot, ragged counts, no byte touched that is not written."""
    rng = np.random.default_rng(heads * 1000 + page + D)
    Bsz, width = 3, -(-sum(steps) // page) + 1
    cache = _garbage(B, rng, Bsz * width + 2, heads, page, D)
    model = cache_ref.Model(cache)
    table = _table(rng, Bsz, width, Bsz * width + 2)
    held = np.zeros(Bsz, dtype=np.int64)
    for step, T in enumerate(steps):
        counts = None if step % 2 == 0 else np.array([T, max(T - 2, 0), rng.integers(0, T + 1)])
        held += T if counts is None else counts
        size = 2.0 ** rng.integers(-6, 7)
        (k, ke), (v, ve) = _tensor(rng, (Bsz, T, heads, D), dtype, size), _tensor(rng, (Bsz, T, heads, D), dtype, 1.0 / size)
        B.cache_append(k, v, cache, _ints(table), _ints(held), counts=None if counts is None else _ints(counts))
        model.append(ke, ve, table, held, counts)
        model.check(cache)


def test_append_views_and_borders(B):
    """k and v read in place from a packed projection; tokens before the first and behind the table, pages that do not exist, values that are not
    finite, counts out of range."""
    import torch
    rng = np.random.default_rng(2)
    Bsz, T, heads, D, page, width = 4, 21, 2, 64, 16, 3
    packed, pe = _tensor(rng, (Bsz, T, 3, heads, D), "bf16")
    packed[0, 3, 1, 0, 5] = float("inf")
    packed[1, 20, 2, 1, 9] = float("nan")
    pe = packed.double().cpu().numpy()
    cache = _garbage(B, rng, 12, heads, page, D, (1, 248))     # pages are entered behind tokens that were never written
    model = cache_ref.Model(cache)
    table = _table(rng, Bsz, width, 12)
    table[2, 1], table[3, 0] = -1, 12
    for lengths, counts in (([21, 30, 48, 40], None), ([5, 50, 70, 21], None), ([21, 22, 23, 48], [-3, 400, 21, 1]), ([0, -5, 1000, 2 ** 31 - 1], [0, 3, 5, 21])):
        k, v = packed[:, :, 1], packed[:, :, 2]
        B.cache_append(k, v, cache, _ints(table), _ints(lengths), counts=None if counts is None else _ints(counts))
        model.append(pe[:, :, 1], pe[:, :, 2], table, lengths, counts)
        model.check(cache)
    assert packed.dtype == torch.bfloat16


ATTENDS = [  # B, M, H, heads, D, page, lengths, causal
    (1, 1, 1, 1, 64, 16, [1], True), (2, 1, 4, 4, 64, 64, [63, 64], False), (3, 1, 8, 2, 64, 32, [65, 0, 300], True),
    (2, 5, 6, 6, 64, 16, [5, 177], True), (2, 7, 6, 3, 64, 128, [3, 129], True), (1, 40, 2, 1, 64, 64, [513], True),
    (2, 33, 4, 1, 64, 32, [100, 1000], False), (1, 1, 16, 1, 128, 64, [2049], True), (2, 3, 8, 2, 128, 16, [31, 700], True),
    (1, 70, 4, 4, 128, 128, [385], True), (3, 17, 3, 3, 128, 32, [17, 1, 96], False), (1, 300, 2, 2, 64, 64, [1111], True),
    (1, 1, 2, 2, 64, 64, [9000], False), (5, 2, 4, 4, 64, 16, [1, 2, 3, 4, 5], True)]


def _filled(B, rng, Bsz, heads, page, D, lengths, extra=3, std=1.0):
    """A cache of garbage with that many tokens of every sequence appended: (cache, model, table)."""
    width = max(1, -(-max(lengths) // page)) + 1
    pages = Bsz * width + extra
    cache = _garbage(B, rng, pages, heads, page, D)
    table = _table(rng, Bsz, width, pages)
    T = max(max(lengths), 1)
    k, _ = _tensor(rng, (Bsz, T, heads, D), "bf16", std)
    v, _ = _tensor(rng, (Bsz, T, heads, D), "bf16")
    B.cache_append(k, v, cache, _ints(table), _ints(lengths), counts=_ints(lengths))
    return cache, cache_ref.Model(cache), table


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Bsz,M,H,heads,D,page,lengths,causal", ATTENDS)
def test_attention(B, Bsz, M, H, heads, D, page, lengths, causal, dtype):
    rng = np.random.default_rng(Bsz * 100 + M + D + page)
    cache, model, table = _filled(B, rng, Bsz, heads, page, D, lengths)
    q, qe = _tensor(rng, (Bsz, M, H, D), dtype)
    scale = D ** -0.5
    want = cache_ref.attention(model, qe, table, lengths, scale, causal)
    out, lse = B.cache_attention(q, cache, _ints(table), _ints(lengths), scale, causal=causal)
    worst = cache_ref.check_attention(out, lse, want, dtype)
    print(f"[cache attention {Bsz} {M} {H}/{heads} {D} {page} {lengths}] worst err/bar {worst:.3f}", flush=True)
    # however the walk is shared out
    for limit in (1, max(max(lengths) // 2, 1), 100000):
        o2, l2 = B.cache_attention(q, cache, _ints(table), _ints(lengths), scale, causal=causal, max_length=limit)
        cache_ref.check_attention(o2, l2, want, dtype)
    o3, l3 = B.cache_attention(q, cache, _ints(table), _ints(lengths), scale, causal=causal)
    import torch
    assert torch.equal(out, o3) and torch.equal(lse, l3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_counts_views_and_missing_pages(B, dtype):
    """A padded batch (rows behind a sequence's count are 0 and -inf), q as a view of a packed projection, a result of the caller's, no lse, a
    page that does not exist in the middle of a sequence, a sequence whose pages all do not."""
    import torch
    rng = np.random.default_rng(8)
    Bsz, M, H, heads, D, page, lengths, counts = 4, 9, 4, 2, 64, 32, [200, 131, 90, 64], [9, 4, 0, 1]
    cache, model, table = _filled(B, rng, Bsz, heads, page, D, lengths)
    table[1, 2], table[3, :] = 9999, -7
    packed, pe = _tensor(rng, (Bsz, M, 3, H, D), dtype)
    for causal in (True, False):
        want = cache_ref.attention(model, pe[:, :, 1], table, lengths, 0.3, causal, counts)
        out = torch.full((Bsz, M, H, D), 5.0, dtype=packed.dtype, device="cuda")
        o, lse = B.cache_attention(packed[:, :, 1], cache, _ints(table), _ints(lengths), 0.3, causal=causal, counts=_ints(counts), out=out)
        assert o is out
        cache_ref.check_attention(out, lse, want, dtype)
        assert bool((out[2] == 0).all()) and bool((out[3] == 0).all()) and bool((out[1, 4:] == 0).all())
        o2, none = B.cache_attention(packed[:, :, 1], cache, _ints(table), _ints(lengths), 0.3, causal=causal, counts=_ints(counts), want_lse=False)
        assert none is None and torch.equal(o2, out)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", [10, 40, 100])
@pytest.mark.parametrize("M,D", [(1, 64), (20, 64), (80, 64), (1, 128), (20, 128)])
def test_attention_large_scores(B, M, D, power, sign, dtype):
    """Scores of up to 2^112, of either sign or all of one.  q and k are integers times a power of two, so all scores are exact and two of them are equal or
    at least 128 exponents apart: the row is the mean of its best tokens' values.  Bars: the division (2^-20) and the rounding of the result; five
    roundings of lse."""
    import torch
    rng = np.random.default_rng(M + D + power)
    page, T = 32, 700
    cache = _garbage(B, rng, 24, 1, page, D)
    table = np.arange(24, dtype=np.int32)[None, :][:, ::-1].copy()
    k = torch.from_numpy(rng.integers(1 if sign < 0 else -8, 9, (1, T, 1, D)).astype(np.float32)).cuda()
    v, _ = _tensor(rng, (1, T, 1, D), "bf16")
    B.cache_append(k, v.float(), cache, _ints(table), _ints([T]))
    kk, vv, there = cache_ref.Model(cache).sequence(0, table, T)
    np.testing.assert_array_equal(kk[:, 0], k.double().cpu().numpy()[0, :, 0])
    assert there.all()
    qe = rng.integers(-8, 0 if sign < 0 else 9, (1, M, 1, D)) * 2.0 ** power
    q = torch.from_numpy(qe).to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]).cuda()
    scores = qe[0, :, 0] @ kk[:, 0].T                                          # exact
    scores[np.arange(T)[None, :] >= T - (M - 1 - np.arange(M))[:, None]] = -np.inf
    best = scores == scores.max(1, keepdims=True)
    want = best @ vv[:, 0] / best.sum(1, keepdims=True)
    want_lse = scores.max(1) * 0.125 + np.log(best.sum(1))
    bar = (2.0 ** -8 if dtype == "bf16" else 0.0) * np.abs(want) + 2.0 ** -20 * np.abs(vv).max()
    for limit in (1, 300, None):
        out, lse = B.cache_attention(q, cache, _ints(table), _ints([T]), 0.125, max_length=limit)
        assert (np.abs(out.double().cpu().numpy()[0, :, 0] - want) <= bar).all()
        assert (np.abs(lse.double().cpu().numpy()[0, 0] - want_lse) <= 2.0 ** -21 * np.abs(want_lse)).all()


def test_attention_lengths_out_of_range(B):
    rng = np.random.default_rng(9)
    cache, model, table = _filled(B, rng, 3, 1, 16, 64, [40, 48, 10])
    q, qe = _tensor(rng, (3, 2, 1, 64), "fp32")
    model_table = table[:, :3]
    lengths = [-4, 2 ** 31 - 1, 10]
    want = cache_ref.attention(model, qe, model_table, lengths, 0.125, True)
    out, lse = B.cache_attention(q, cache, _ints(model_table), _ints(lengths), 0.125)
    cache_ref.check_attention(out, lse, want, "fp32")
    assert bool((out[0] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,D", [(6, 64), (40, 64), (20, 128)])
def test_attention_not_finite(B, M, D, dtype):
    """NaN keys, values and queries reach the rows that attend to them and no others; large scores do not overflow."""
    import torch
    rng = np.random.default_rng(M + D)
    Bsz, H, heads, page, n = 2, 2, 1, 16, 150
    cache, model, table = _filled(B, rng, Bsz, heads, page, D, [n, n], std=8.0)
    q, qe = _tensor(rng, (Bsz, M, H, D), dtype, 8.0)
    q[1, 1, 0, 3] = float("nan")
    qe = q.double().cpu().numpy()
    kb, vb = cache.k.view(torch.uint8), cache.v.view(torch.uint8)
    late = n - 3                                             # the last two tokens: only the last rows attend to them
    kb[int(table[0, late // page]), 0, late % page, 7] = 0x7f
    vb[int(table[0, (n - 2) // page]), 0, 11, (n - 2) % page] = 0xff
    vb[int(table[1, (n - 1) // page]), 0, 2, (n - 1) % page] = 0x7f
    model = cache_ref.Model(cache)
    want = cache_ref.attention(model, qe, table, [n, n], 1.0, True)
    assert np.isnan(want[0]).any() and np.isfinite(want[0][0, :M - 3]).all()
    out, lse = B.cache_attention(q, cache, _ints(table), _ints([n, n]), 1.0)
    cache_ref.check_attention(out, lse, want, dtype)


def test_attention_shared_pages_and_whole_values(B):
    """Two sequences with the same first pages; values all alike come back as they are."""
    import torch
    rng = np.random.default_rng(12)
    cache, model, table = _filled(B, rng, 2, 2, 16, 64, [64, 64])
    table[1, :2] = table[0, :2]
    q, qe = _tensor(rng, (2, 1, 2, 64), "fp32")
    out, lse = B.cache_attention(q, cache, _ints(table), _ints([64, 50]), 0.125)
    cache_ref.check_attention(out, lse, cache_ref.attention(model, qe, table, [64, 50], 0.125, True), "fp32")
    alike = B.kv_cache(8, 1, 16, 64)
    ones = torch.full((1, 100, 1, 64), 0.6875, device="cuda")
    B.cache_append(ones, ones, alike, _ints([list(range(8))]), _ints([100]))
    out, lse = B.cache_attention(torch.zeros((1, 1, 1, 64), device="cuda"), alike, _ints([list(range(8))]), _ints([100]), 1.0)
    assert bool((out - 0.6875).abs().max() <= 0.6875 * 100 * 2.0 ** -23) and abs(float(lse) - np.log(100)) <= 1e-5


def test_offsets_beyond_32_bits(B):
    """A cache of more than 2^32 bytes of keys: its last pages."""
    import torch
    rng = np.random.default_rng(13)
    pages, heads, page, D = 66000, 8, 64, 128
    cache = B.KvCache(torch.empty((pages, heads, page, D), dtype=torch.float8_e4m3fn, device="cuda"),
                      torch.empty((pages, heads, D, page), dtype=torch.float8_e4m3fn, device="cuda"),
                      torch.empty((pages, heads, 2), dtype=torch.uint8, device="cuda"))
    assert cache.k.numel() > 2 ** 32
    small = B.kv_cache(3, heads, page, D)
    (k, _), (v, _) = _tensor(rng, (1, 150, heads, D), "bf16"), _tensor(rng, (1, 150, heads, D), "bf16")
    q, _ = _tensor(rng, (1, 2, heads, D), "bf16")
    far, near = _ints([[pages - 1, pages - 3, pages - 2]]), _ints([[2, 0, 1]])
    B.cache_append(k, v, cache, far, _ints([150]))
    B.cache_append(k, v, small, near, _ints([150]))
    for held, part in ((cache.k, small.k), (cache.v, small.v)):
        assert torch.equal(held[pages - 3:pages - 1].view(torch.uint8), part[:2].view(torch.uint8))
    a, b = B.cache_attention(q, cache, far, _ints([150]), 0.1), B.cache_attention(q, small, near, _ints([150]), 0.1)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_steps_captured_and_on_streams(B):
    """A step (projection, append, attention, projection) captured once and replayed while lengths grow, beside the same steps run eagerly; a
    second graph with buffers of its own on another stream."""
    import torch
    rng = np.random.default_rng(14)
    Bsz, H, heads, D, page, width = 2, 4, 2, 64, 16, 40
    E = H * D
    w_qkv = B.quantize(_tensor(rng, ((H + 2 * heads) * D, E), "bf16", E ** -0.5)[0], 128)
    w_o = B.quantize(_tensor(rng, (E, E), "bf16", E ** -0.5)[0], 128)
    table = _ints(np.arange(Bsz * width).reshape(Bsz, width))

    def step(x, cache, lengths):
        lengths.add_(1)
        qkv = B.quantized_linear(x, w_qkv).view(Bsz, 1, H + 2 * heads, D)
        B.cache_append(qkv[:, :, H:H + heads], qkv[:, :, H + heads:], cache, table, lengths)
        out, lse = B.cache_attention(qkv[:, :, :H], cache, table, lengths, D ** -0.5)
        return B.quantized_linear(out.view(Bsz, 1, E), w_o), lse

    runs = []
    for _ in range(3):
        runs.append(dict(x=torch.zeros((Bsz, 1, E), dtype=torch.bfloat16, device="cuda"), cache=B.kv_cache(Bsz * width, heads, page, D),
                         lengths=_ints([500, 3])))
    step(**runs[0])
    runs[0] = dict(x=runs[0]["x"], cache=B.kv_cache(Bsz * width, heads, page, D), lengths=_ints([500, 3]))
    graphs = []
    for r in runs[1:]:
        before = r["lengths"].clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r["y"], r["lse"] = step(r["x"], r["cache"], r["lengths"])
        r["lengths"].copy_(before)
        graphs.append(g)
    side = torch.cuda.Stream()
    for trip in range(20):
        x = _tensor(rng, (Bsz, 1, E), "bf16")[0]
        for r in runs:
            r["x"].copy_(x)
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        y, lse = step(**runs[0])
        torch.cuda.synchronize()
        for r in runs[1:]:
            assert torch.equal(r["y"], y) and torch.equal(r["lse"], lse), trip
            assert torch.equal(r["cache"].k.view(torch.uint8), runs[0]["cache"].k.view(torch.uint8))
            assert torch.equal(r["cache"].scales, runs[0]["cache"].scales)


def test_run_together_against_the_reference(B):
    """An image's tokens projected and cached, then prompt tokens in steps: every stage against its reference on what the stage before left."""
    import torch
    rng = np.random.default_rng(15)
    H, D, N, page = 6, 64, 300, 64
    E = H * D
    w, _ = _tensor(rng, (3 * E, E), "bf16", E ** -0.5)
    qw = B.quantize(w, 128)
    x, xe = _tensor(rng, (1, N, E), "bf16")
    qkv = B.quantized_linear(x, qw)
    xh, wh = ref.held(xe[0]), ref.matrix(qw)
    want = xh @ wh.T
    assert ref.far(qkv[0].double().cpu().numpy(), want) < 2.0 ** -8
    cache = B.kv_cache(8, H, page, D)
    model = cache_ref.Model(cache)
    table = rng.permutation(8)[None].astype(np.int32)
    parts = qkv.view(1, N, 3, H, D)
    B.cache_append(parts[:, :, 1], parts[:, :, 2], cache, _ints(table), _ints([N]))
    pe = parts.double().cpu().numpy()
    model.append(pe[:, :, 1], pe[:, :, 2], table, [N])
    model.check(cache)
    held = N
    for T in (5, 1, 9):
        held += T
        p, _ = _tensor(rng, (1, T, E), "bf16")
        new = B.quantized_linear(p, qw).view(1, T, 3, H, D)
        ne = new.double().cpu().numpy()
        B.cache_append(new[:, :, 1], new[:, :, 2], cache, _ints(table), _ints([held]))
        model.append(ne[:, :, 1], ne[:, :, 2], table, [held])
        model.check(cache)
        out, lse = B.cache_attention(new[:, :, 0], cache, _ints(table), _ints([held]), D ** -0.5)
        cache_ref.check_attention(out, lse, cache_ref.attention(model, ne[:, :, 0], table, [held], D ** -0.5, True), "bf16")
    assert out.dtype == torch.bfloat16


def test_refusals(B):
    import torch
    cache = B.kv_cache(4, 2, 16, 64)
    table, lengths = _ints([[0, 1], [2, 3]]), _ints([5, 6])
    k = torch.zeros((2, 3, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((2, 3, 4, 64), dtype=torch.bfloat16, device="cuda")
    B.cache_append(k, k, cache, table, lengths)
    B.cache_attention(q, cache, table, lengths, 0.125)
    wrong = [
        lambda: B.cache_append(k, k.float(), cache, table, lengths), lambda: B.cache_append(k.half(), k.half(), cache, table, lengths),
        lambda: B.cache_append(k, k[:, :2], cache, table, lengths), lambda: B.cache_append(k[:, :, :1], k[:, :, :1], cache, table, lengths),
        lambda: B.cache_append(k, k, cache, table[:1], lengths), lambda: B.cache_append(k, k, cache, table, lengths[:1]),
        lambda: B.cache_append(k, k, cache, table, lengths, counts=lengths[:1]), lambda: B.cache_append(k[:, :0], k[:, :0], cache, table, lengths),
        lambda: B.cache_append(k, k, B.KvCache(cache.k, cache.v, cache.scales[:2]), table, lengths),
        lambda: B.cache_append(k, k, B.kv_cache(4, 2, 24, 64), table, lengths),
        lambda: B.cache_attention(q[:, :, :3], cache, table, lengths, 0.125), lambda: B.cache_attention(q, cache, table, lengths, 0.0),
        lambda: B.cache_attention(q, cache, table, lengths, float("nan")), lambda: B.cache_attention(q.half(), cache, table, lengths, 0.125),
        lambda: B.cache_attention(q, cache, table, lengths, 0.125, max_length=-1),
        lambda: B.cache_attention(q, cache, table, lengths, 0.125, out=q[:, :2]),
        lambda: B.cache_attention(torch.zeros((2, 3, 4, 32), dtype=torch.bfloat16, device="cuda"), cache, table, lengths, 0.125)]
    for i, call in enumerate(wrong):
        with pytest.raises(B.DfaError):
            call()
            print("not refused:", i)
    for call in (lambda: B.cache_append(k, k, cache, table.long(), lengths), lambda: B.cache_attention(q, cache, table, lengths.long(), 0.125),
                 lambda: B.cache_attention(q, B.KvCache(cache.k.view(torch.uint8), cache.v, cache.scales), table, lengths, 0.125)):
        with pytest.raises(TypeError):
            call()
    long = B.kv_cache(400, 1, 16, 64)
    with pytest.raises(B.DfaError) as e:
        B.cache_attention(torch.zeros((1, 1, 1, 64), device="cuda"), long, _ints([list(range(400))]), _ints([6400]), 0.125, workspace=None)
    assert e.value.code == B.DFA_ERR_WORKSPACE
