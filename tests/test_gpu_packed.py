"""Pages and row maps of a step, appending packed rows, and a layer's operators on packed prompts one after the other."""
import random

import numpy as np
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


def _ints(values):
    import torch
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Step:
    """A cache's tables in use, here and in lists."""

    def __init__(self, seed, Bsz, width, page, spare=0):
        r = random.Random(seed)
        self.page, self.r = page, r
        self.free = list(range(Bsz * width + spare))
        r.shuffle(self.free)
        self.n_free, self.lengths = len(self.free), [0] * Bsz
        self.table = [[-7] * width for _ in range(Bsz)]
        self.dev = dict(free=_ints(self.free), n_free=_ints([self.n_free]), lengths=_ints(self.lengths), table=_ints(self.table))

    def reserve(self, B, counts, rows, in_place=False):
        d = self.dev
        got = B.cache_reserve(_ints(counts), d["lengths"], d["table"], d["free"], d["n_free"], self.page, rows, in_place=in_place)
        lengths, n_free, starts, slots, positions, refused = ref.reserve(counts, self.lengths, self.table, self.free, self.n_free, self.page, rows)
        want = dict(lengths=lengths, n_free=[n_free], starts=starts, slots=slots, positions=positions, refused=[refused])
        for name, values in want.items():
            assert getattr(got, name).tolist() == values, name
        assert d["table"].tolist() == self.table and d["free"].tolist() == self.free
        if in_place:
            assert got.lengths is d["lengths"] and got.n_free is d["n_free"]
        else:
            assert d["lengths"].tolist() == self.lengths and d["n_free"].tolist() == [self.n_free]
            d["lengths"], d["n_free"] = got.lengths, got.n_free
        self.lengths, self.n_free = lengths, n_free
        return got

    def release(self, B, done):
        d = self.dev
        refused = B.cache_release(_ints(done), d["lengths"], d["table"], d["free"], d["n_free"], self.page)
        for b, gone in enumerate(done):
            if gone:
                for at in range(-(-self.lengths[b] // self.page)):
                    self.free[self.n_free] = self.table[b][at]
                    self.n_free += 1
                self.lengths[b] = 0
        assert refused.tolist() == [0] and d["lengths"].tolist() == self.lengths and d["n_free"].tolist() == [self.n_free] and d["free"].tolist() == self.free


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("Bsz,most", [(1, 1), (1, 5000), (3, 40), (70, 200), (1023, 9), (1024, 3), (1025, 3), (2500, 12), (4500, 4)])
def test_steps(B, Bsz, most, page):
    """Prompts, single tokens, sequences that end and begin again; one launch and two."""
    width = 2 * most // page + 4
    s = Step(Bsz + page, Bsz, width, page)
    for step in range(6):
        counts = [1] * Bsz if step in (1, 4) else [s.r.choice([0, 1, s.r.randint(0, most)]) for _ in range(Bsz)]
        counts = [min(c, width * page - l) for c, l in zip(counts, s.lengths)]
        rows = max(1, sum(counts)) + (0 if step == 2 else s.r.randint(0, 70))
        assert s.reserve(B, counts, rows, in_place=step % 2 == 1).refused.item() == 0
        if step in (2, 3):
            s.release(B, [int(s.r.random() < 0.4) for _ in range(Bsz)])


@pytest.mark.parametrize("rows", [64, 6000])
def test_a_step_that_does_not_fit(B, rows):
    s = Step(1, 4, 8, 16)
    assert s.reserve(B, [40, 0, 17, 1], rows).refused.item() == 0
    assert s.reserve(B, [1, 100, 0, 0], rows).refused.item() == (4 if rows == 64 else 0)
    if rows == 64:
        s.reserve(B, [0, 64, 0, 0], rows)
    assert s.reserve(B, [89, 0, 0, 0], rows).refused.item() == (6 if rows == 64 else 2)
    assert s.reserve(B, [1, -1, 0, 0], rows).refused.item() == 8
    s.n_free = 3
    s.dev["n_free"] = _ints([3])
    assert s.reserve(B, [0, 0, 60, 0], rows).refused.item() == 0        # from 2 pages to 5: all that is left
    assert s.reserve(B, [0, 0, 30, 0], rows).refused.item() == 1
    assert s.reserve(B, [2 ** 31 - 1] * 4, rows).refused.item() == 7
    assert s.reserve(B, [0, 0, 0, 0], rows).refused.item() == 0


@pytest.mark.parametrize("rows", [64, 5000, 2 ** 20 + 1])
def test_reasons_add_up(B, rows):
    """A step of far more rows than there is room for: whether its pages are too many, too, is still told."""
    import torch
    table, free = torch.zeros((2, 500001), dtype=torch.int32, device="cuda"), torch.arange(10 ** 6, dtype=torch.int32, device="cuda")
    for counts, reasons in (([8 * 10 ** 6] * 2, 4), ([8 * 10 ** 6, 8 * 10 ** 6 + 1], 5), ([0, 16 * 10 ** 6], 6), ([0, 16 * 10 ** 6 + 1], 7)):
        r = B.cache_reserve(_ints(counts), _ints([0, 0]), table, free, _ints([10 ** 6]), 16, rows)
        assert r.refused.item() == reasons and r.lengths.tolist() == [0, 0] and r.n_free.item() == 10 ** 6 and r.starts.tolist() == [0, 0, 0]
        assert (r.slots == -1).all() and (r.positions == -1).all()
    assert not table.any()


def test_a_stack_without_room(B):
    lengths, table, free, n = _ints([30, 40]), _ints([[1, 2, 0], [3, 4, 5]]), _ints([9, 9, 9, 9]), _ints([0])
    before = free.clone()
    assert B.cache_release(_ints([1, 1]), lengths, table, free, n, 16).item() == 1
    assert lengths.tolist() == [30, 40] and n.tolist() == [0] and free.equal(before)
    assert B.cache_release(_ints([0, 5]), lengths, table, free, n, 16).item() == 0
    assert lengths.tolist() == [30, 0] and n.tolist() == [3] and free.tolist() == [3, 4, 5, 9]


def test_strided_table(B):
    """Rows of a wider table; entries outside are left alone."""
    import torch
    wide = torch.full((3, 10), -7, dtype=torch.int32, device="cuda")
    r = B.cache_reserve(_ints([17, 0, 33]), _ints([0, 0, 0]), wide[:, 2:6], _ints([5, 6, 7, 8, 9]), _ints([5]), 16, 50)
    assert wide.tolist() == [[-7, -7, 9, 8] + [-7] * 6, [-7] * 10, [-7, -7, 7, 6, 5] + [-7] * 5] and r.n_free.item() == 0


APPENDS = [(2, 16, 64, [40, 0, 1, 16, 17]), (3, 64, 128, [1, 1, 130, 63]), (1, 128, 64, [300, 2]), (2, 32, 128, [1] * 70), (12, 64, 64, [33, 64, 65])]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,page,D,counts", APPENDS)
def test_packed_append(B, heads, page, D, counts, dtype):
    """The same bytes as appending the rows padded, step after step, with rows of no sequence behind."""
    import torch
    Bsz, width = len(counts), 3 * max(counts) // page + 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = torch.randperm(Bsz * width, generator=gen, device="cuda").to(torch.int32).view(Bsz, width)
    caches = [B.kv_cache(Bsz * width, heads, page, D) for _ in range(2)]
    held = [0] * Bsz
    for step in range(3):
        now = [c if step != 1 else 1 for c in counts]
        held = [h + c for h, c in zip(held, now)]
        starts, most = ref.starts_of(now), max(now)
        packed = torch.randn((starts[-1] + 9, 2, heads, D), generator=gen, device="cuda").mul_(2.0 ** step).to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype])
        packed[starts[-1]:] = float("nan")
        padded = torch.zeros((Bsz, most, 2, heads, D), dtype=packed.dtype, device="cuda")
        for b in range(Bsz):
            padded[b, :now[b]] = packed[starts[b]:starts[b + 1]]
        B.cache_append(packed[:, 0], packed[:, 1], caches[0], table, _ints(held), starts=_ints(starts))
        B.cache_append(padded[:, :, 0], padded[:, :, 1], caches[1], table, _ints(held), counts=_ints(now))
        for a, b in zip(*caches):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def _layer(B, x, res, norm, weight, sizes, step):
    """norm -> 8-bit projection -> attention within the prompts, and their keys and values into the cache."""
    H, Hkv, D, page = sizes
    r = B.cache_reserve(step["counts"], step["lengths"], step["table"], step["free"], step["n_free"], page, x.shape[0], in_place=True)
    q8, h = B.rms_norm(x, norm, 1e-6, residual=res, quantized=True)
    import torch
    qkv = B.quantized_product(q8, weight, torch.bfloat16).view(x.shape[0], H + 2 * Hkv, D)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    out, lse = B.prompt_attention(q, k, v, r.starts, D ** -0.5)
    B.cache_append(k, v, step["cache"], step["table"], r.lengths, starts=r.starts)
    return r, h, q, k, v, out, lse


def _fresh(B, sizes, Bsz, width):
    H, Hkv, D, page = sizes
    return dict(counts=_ints([0] * Bsz), lengths=_ints([0] * Bsz), table=_ints([[0] * width for _ in range(Bsz)]), free=_ints(list(range(Bsz * width))),
                n_free=_ints([Bsz * width]), cache=B.kv_cache(Bsz * width, Hkv, page, D))


def test_a_layer_of_packed_prompts(B):
    """The operators one after the other, as a server runs them: prompts of unlike lengths, then a token of each against the cache."""
    import torch
    sizes = H, Hkv, D, page = 8, 2, 64, 16
    C, rows, lengths = 512, 192, [70, 1, 33, 80]
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, res = (torch.randn((rows, C), generator=gen, device="cuda").bfloat16() for _ in range(2))
    norm = (1 + 0.1 * torch.randn((C,), generator=gen, device="cuda")).bfloat16()
    weight = B.quantize(torch.randn(((H + 2 * Hkv) * D, C), generator=gen, device="cuda") * C ** -0.5, 128)
    step = _fresh(B, sizes, 4, 8)
    step["counts"].copy_(_ints(lengths))
    r, h, q, k, v, out, lse = _layer(B, x, res, norm, weight, sizes, step)
    starts = ref.starts_of(lengths)
    assert r.starts.tolist() == starts and step["lengths"].tolist() == lengths and r.refused.item() == 0
    want, want_lse, tol, tol_lse = ref.attention(q, k, v, starts, D ** -0.5, True)
    assert ((out.double() - want).abs() <= tol).all() and (out[starts[-1]:] == 0).all()
    # every row's slot holds its key: in e4m3, half a step of its own or of its page's smallest
    slots = r.slots[:starts[-1]]
    unit = torch.exp2(step["cache"].scales[..., 0].double() - 127)[slots // page]                   # [rows, Hkv]
    held = step["cache"].k.double()[slots // page, :, slots % page] * unit[:, :, None]
    kd = k[:starts[-1]].double()
    assert ((held - kd).abs() <= kd.abs() * 2.0 ** -4 + unit[:, :, None] * 2.0 ** -10).all()
    # a token each, against what the cache holds
    step["counts"].fill_(1)
    r2, _, q2, k2, v2, _, _ = _layer(B, x[:4].contiguous(), res[:4].contiguous(), norm, weight, sizes, step)
    assert step["lengths"].tolist() == [n + 1 for n in lengths] and r2.positions[:4].tolist() == lengths
    got, got_lse = B.cache_attention(q2[:4].view(4, 1, H, D), step["cache"], step["table"], step["lengths"], D ** -0.5)
    for b in range(4):
        n = lengths[b] + 1
        ids = step["table"][b].long()
        e = torch.exp2(step["cache"].scales[ids].double() - 127)
        kk = (step["cache"].k[ids].double() * e[..., 0, None, None]).permute(0, 2, 1, 3).reshape(-1, Hkv, D)[:n]
        vv = (step["cache"].v[ids].double() * e[..., 1, None, None]).permute(0, 3, 1, 2).reshape(-1, Hkv, D)[:n]
        for head in range(H):
            p = torch.softmax(kk[:, head // 4] @ q2[b, head].double() * D ** -0.5, 0)
            o, size = p @ vv[:, head // 4], p @ vv[:, head // 4].abs()
            assert ((got[b, 0, head].double() - o).abs() <= 2.0 ** -8 * (size + o.abs()) + 1e-4 * size).all()


def test_a_captured_layer(B):
    """One graph serves steps of any lengths; replays against eager calls on tables of their own."""
    import torch
    sizes = H, Hkv, D, page = 8, 2, 64, 16
    C, rows, Bsz = 256, 160, 3
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, res = (torch.randn((rows, C), generator=gen, device="cuda").bfloat16() for _ in range(2))
    norm = (1 + 0.1 * torch.randn((C,), generator=gen, device="cuda")).bfloat16()
    weight = B.quantize(torch.randn(((H + 2 * Hkv) * D, C), generator=gen, device="cuda") * C ** -0.5, 128)
    steps = [_fresh(B, sizes, Bsz, 40) for _ in range(2)]
    _layer(B, x, res, norm, weight, sizes, _fresh(B, sizes, Bsz, 40))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = _layer(B, x, res, norm, weight, sizes, steps[0])
    for counts in ([100, 30, 0], [1, 1, 1], [0, 60, 90], [1, 1, 1], [200, 0, 0], [1, 0, 1]):
        x.copy_(torch.randn((rows, C), generator=gen, device="cuda"))
        for s in steps:
            s["counts"].copy_(_ints(counts))
        graph.replay()
        eager = _layer(B, x, res, norm, weight, sizes, steps[1])
        torch.cuda.synchronize()
        for a, b in zip(captured[0], eager[0]):
            assert torch.equal(a, b)
        assert captured[0].refused.item() == (4 if sum(counts) > rows else 0)
        assert all(torch.equal(a, b) for a, b in zip(captured[1:], eager[1:]))
        for a, b in zip(steps[0]["cache"], steps[1]["cache"]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        for name in ("lengths", "table", "n_free"):
            assert torch.equal(steps[0][name], steps[1][name])


def test_native_calls(B, monkeypatch):
    """The ordinary calls in native code against the ones that Python marshals: the same bits."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *shape, dtype=torch.bfloat16: torch.randn(shape, generator=gen, device="cuda").to(dtype)
    for dtype in (torch.bfloat16, torch.float32):
        x, q, starts = rand(90, 200, dtype=dtype), rand(90, 8, 64, dtype=dtype), _ints([0, 30, 30, 85])
        w, r, dout = rand(200, dtype=dtype), rand(90, 200, dtype=dtype), rand(90, 4, 64, dtype=dtype)

        def calls():
            out, lse = B.prompt_attention(q[:, :4], q[:, 4:6], q[:, 6:], starts, 0.125)
            got = [out, lse, *B.prompt_attention_backward(q[:, :4], q[:, 4:6], q[:, 6:], out, lse, dout, starts, 0.125, False)]
            for residual in (None, r):
                for quantized in (False, True, "both"):
                    y, h = B.rms_norm(x, w, 1e-6, residual=residual, quantized=quantized)
                    y = y if quantized == "both" else (y,)
                    for part in y:
                        got += [part.values.view(torch.uint8), part.scales[:, :90]] if isinstance(part, B.QuantizedMatrix) else [part]
                    got += [h] if h is not None else []
            got += B.rms_norm_backward(x, r, w, 1e-6) + B.rms_norm_backward(x, r, None, 1e-6, dh=x)
            table = _ints([[0] * 4, [0] * 4])
            got += [*B.cache_reserve(_ints([20, 1]), _ints([0, 0]), table, _ints([5, 6, 7, 8]), _ints([4]), 16, 30), table]
            cache = B.kv_cache(9, 2, 16, 64)
            B.cache_append(q[:, 4:6], q[:, 6:], cache, table, _ints([20, 1]), starts=_ints([0, 20, 21]))
            return got + [t.view(torch.uint8) for t in cache]

        native = calls()
        with monkeypatch.context() as m:
            m.setattr(B, "_native_call", lambda *a: None)
            python = calls()
        assert len(native) == len(python)
        for a, b in zip(native, python):
            assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


def test_refusals(B):
    import torch
    q, starts = torch.zeros((10, 4, 64), dtype=torch.bfloat16, device="cuda"), _ints([0, 10])
    k = q[:, :2]
    out, lse = B.prompt_attention(q, k, k, starts, 0.125)
    for error, call in (
            (B.DfaError, lambda: B.prompt_attention(q, q[:, :3], q[:, :3], starts, 0.125)), (B.DfaError, lambda: B.prompt_attention(q, k, k[:5], starts, 0.125)),
            (B.DfaError, lambda: B.prompt_attention(q, k[:5], k[:5], starts, 0.125)), (B.DfaError, lambda: B.prompt_attention(q, k.float(), k, starts, 0.125)),
            (B.DfaError, lambda: B.prompt_attention(q.half(), k.half(), k.half(), starts, 0.125)), (B.DfaError, lambda: B.prompt_attention(q, k, k, starts, -1.0)),
            (B.DfaError, lambda: B.prompt_attention(q, k, k, starts[:1], 0.125)), (TypeError, lambda: B.prompt_attention(q, k, k, starts.long(), 0.125)),
            (RuntimeError, lambda: B.prompt_attention(q, k, k, starts.cpu(), 0.125)), (B.DfaError, lambda: B.prompt_attention(q[..., :32], k[..., :32], k[..., :32], starts, 0.125)),
            (B.DfaError, lambda: B.prompt_attention(q.transpose(1, 2), k, k, starts, 0.125)), (B.DfaError, lambda: B.prompt_attention(q, k, k, starts, 0.125, out=out[:5])),
            (B.DfaError, lambda: B.prompt_attention(q, k, k, starts, 0.125, lse=lse.double())),
            (B.DfaError, lambda: B.prompt_attention_backward(q, k, k, out, lse[:, :5], q, starts, 0.125)),
            (B.DfaError, lambda: B.prompt_attention_backward(q, k, k, out, lse, q, starts, 0.125, workspace=None)),
            (B.DfaError, lambda: B.prompt_attention_backward(q, k, k, out, lse, q, starts, 0.125, workspace=torch.zeros((16,), dtype=torch.uint8, device="cuda"))),
            (B.DfaError, lambda: B.cache_reserve(_ints([1]), _ints([0, 0]), _ints([[0]]), _ints([0]), _ints([1]), 16, 5)),
            (B.DfaError, lambda: B.cache_reserve(_ints([1]), _ints([0]), _ints([[0]]), _ints([0]), _ints([1]), 20, 5)),
            (B.DfaError, lambda: B.cache_reserve(_ints([1]), _ints([0]), _ints([[0]]), _ints([0]), _ints([1]), 16, 0)),
            (TypeError, lambda: B.cache_reserve(_ints([1]).long(), _ints([0]), _ints([[0]]), _ints([0]), _ints([1]), 16, 5)),
            (B.DfaError, lambda: B.cache_append(k, k, B.kv_cache(2, 3), _ints([[0, 1]]), _ints([10]), starts=starts)),
            (ValueError, lambda: B.cache_append(k, k, B.kv_cache(2, 2), _ints([[0, 1]]), _ints([10]), counts=_ints([1]), starts=starts))):
        with pytest.raises(error):
            call()


def test_two_streams(B):
    """Calls that overlap on two streams, each with tensors of its own, against the same calls one after the other."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(8)
    sets = []
    for dtype in (torch.bfloat16, torch.float32):
        qkv = torch.randn((2500, 16, 64), generator=gen, device="cuda").to(dtype)
        x, w = torch.randn((2500, 512), generator=gen, device="cuda").to(dtype), torch.randn((512,), generator=gen, device="cuda").to(dtype)
        sets.append((qkv, x, w, _ints([0, 1200, 1300, 2500]), [_ints([300] * 40), _ints([5] * 40), torch.zeros((40, 10), dtype=torch.int32, device="cuda"),
                                                              torch.arange(800, dtype=torch.int32, device="cuda"), _ints([800])]))

    def run(qkv, x, w, starts, pages):
        q, k, v = qkv[:, :8], qkv[:, 8:12], qkv[:, 12:]
        out, lse = B.prompt_attention(q, k, v, starts, 0.125)
        y, h = B.rms_norm(x, w, 1e-6, residual=x)
        return [out, lse, y, h, *B.prompt_attention_backward(q, k, v, out, lse, out, starts, 0.125), *B.rms_norm_backward(y, h, w, 1e-6),
                *B.cache_reserve(*pages, 64, 12000)]

    want = [run(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                got[i].append(run(*s))
    torch.cuda.synchronize()
    for mine, theirs in zip(got, want):
        for results in mine:
            assert all(torch.equal(a, b) for a, b in zip(results, theirs))
