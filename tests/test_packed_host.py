"""Host side of the operators on packed prompts: refusals of the C ABI (fake pointers, never dereferenced), workspace sizes, the references' own pins."""
import ctypes
import math

import pytest
import torch

import packed_ref as ref

OK = 0x10000


@pytest.fixture(scope="module")
def B():
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


BAD_PROMPTS = [(dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(starts=None), -1), (dict(out=None), -1), (dict(dt=2), -4), (dict(dt=-1), -4),
               (dict(T=0), -2), (dict(Bsz=0), -2), (dict(H=3), -2), (dict(H=1), -2), (dict(Hkv=0), -2), (dict(D=32), -2), (dict(D=96), -2), (dict(scale=0.0), -2),
               (dict(scale=-1.0), -2), (dict(scale=math.inf), -2), (dict(scale=math.nan), -2), (dict(scale=2.0 ** -101), -2), (dict(scale=1.5e30), -2), (dict(q=OK + 2), -5), (dict(s=(0, 1024, 60)), -5),
               (dict(s=(0, 1020, 64)), -5), (dict(starts=OK + 2), -5), (dict(out=OK + 8), -5), (dict(lse=OK + 2), -5), (dict(s=(0, 1 << 24, 64)), -7),
               (dict(s=(0, -1024, 64)), -7), (dict(T=2 ** 31 - 1), -7), (dict(Bsz=2 ** 31 - 1), -7), (dict(T=1 << 30, H=1 << 12, Hkv=1 << 12), -7)]


def test_refusals_of_attention(B):
    def rc(q=OK, k=OK, v=OK, s=(0, 1024, 64), dt=0, T=100, H=4, Hkv=2, D=64, starts=OK, Bsz=2, scale=0.125, out=OK, lse=OK):
        st = B.Strides(*s)
        return B.lib().dfa_prompt_attention(q, k, v, st, st, st, dt, T, H, Hkv, D, starts, Bsz, 1, ctypes.c_float(scale), out, lse, None)

    for bad, code in BAD_PROMPTS:
        assert rc(**bad) == code, bad


def test_refusals_of_its_backward(B):
    def rc(q=OK, k=OK, v=OK, s=(0, 1024, 64), dt=0, T=100, H=4, Hkv=2, D=64, starts=OK, Bsz=2, scale=0.125, out=OK, lse=OK, dout=OK, dq=OK, dk=OK, dv=OK, ws=OK,
           size=1 << 40):
        st = B.Strides(*s)
        return B.lib().dfa_prompt_attention_backward(q, k, v, st, st, st, out, lse, dout, dt, T, H, Hkv, D, starts, Bsz, 1, ctypes.c_float(scale), dq, dk, dv, ws,
                                                     size, None)

    for bad, code in BAD_PROMPTS + [(dict(lse=None), -1), (dict(dout=None), -1), (dict(dq=None), -1), (dict(dk=None), -1), (dict(dv=None), -1), (dict(dout=OK + 2), -5),
                                    (dict(dq=OK + 8), -5), (dict(dk=OK + 8), -5), (dict(dv=OK + 4), -5), (dict(ws=OK + 8), -5), (dict(H=1 << 18, Hkv=1 << 18), -7)]:
        assert rc(**bad) == code, bad


def test_workspaces(B):
    size = B.lib().dfa_prompt_attention_backward_workspace_bytes
    assert size(100, 4, 4, 64, 1) == 2 * 4 * 100 * 4 + (-3200) % 256                # -delta and lse of every row
    assert size(100, 8, 2, 64, 1) > 2 * 8 * 100 * 4 + 4 * 2 * 100 * 2 * 64 * 4 - 1   # and parts of dk and dv where a few workgroups share heads out
    assert size(10 ** 6, 8, 2, 64, 1) == 2 * 8 * 10 ** 6 * 4                        # not where there are enough
    assert size(0, 4, 4, 64, 1) == 0 and size(100, 4, 3, 64, 1) == 0 and size(100, 4, 4, 80, 1) == 0
    size = B.lib().dfa_rms_norm_backward_workspace_bytes
    assert size(1, 4096) == 0 and size(1000, 100) % 256 == 0 and size(1000, 100) > 0 and size(0, 5) == 0 and size(5, 32769) == 0


def test_refusals_of_the_norm(B):
    def rc(x=OK, ldx=64, res=OK, ldr=64, w=OK, w_dt=0, dt=0, eps=1e-6, h=OK, ldh=64, y=OK, ldy=64, q=None, M=4, C=64):
        m = None if q is None else ctypes.byref(B.Quantized(*q))
        return B.lib().dfa_rms_norm(x, ldx, res, ldr, w, w_dt, dt, ctypes.c_float(eps), h, ldh, y, ldy, m, M, C, None)

    good = (OK, OK, 128, 16)
    for bad, code in [(dict(x=None), -1), (dict(y=None), -1), (dict(q=(None, OK, 128, 16)), -1), (dict(q=(OK, None, 128, 16)), -1), (dict(dt=2), -4), (dict(w_dt=3), -4),
                      (dict(dt=1, w_dt=0), -4), (dict(M=0), -2), (dict(C=0), -2), (dict(eps=-1.0), -2), (dict(eps=math.nan), -2), (dict(eps=math.inf), -2),
                      (dict(ldx=63), -2), (dict(ldr=63), -2), (dict(ldh=63), -2), (dict(ldy=63), -2), (dict(q=(OK, OK, 64, 16)), -2), (dict(q=(OK, OK, 128, 3)), -2),
                      (dict(q=(OK, OK, 136, 16)), -5), (dict(q=(OK, OK, 128, 20)), -5), (dict(q=(OK + 8, OK, 128, 16)), -5), (dict(q=(OK, OK + 1, 128, 16)), -5),
                      (dict(x=OK + 1), -5), (dict(res=OK + 1), -5), (dict(h=OK + 1), -5), (dict(y=OK + 1), -5), (dict(w=OK + 1), -5),
                      (dict(C=32769, ldx=40000, ldr=40000, ldh=40000, ldy=40000), -7), (dict(M=1 << 40), -7)]:
        assert rc(**bad) == code, bad
    assert rc(y=None, q=good, C=0) == -2


def test_refusals_of_its_backward_too(B):
    def rc(dy=OK, lddy=64, h=OK, ldh=64, w=OK, w_dt=0, dt=0, eps=1e-6, dh=OK, lddh=64, dx=OK, lddx=64, dw=OK, M=4000, C=64, ws=OK, size=1 << 40):
        return B.lib().dfa_rms_norm_backward(dy, lddy, h, ldh, w, w_dt, dt, ctypes.c_float(eps), dh, lddh, dx, lddx, dw, M, C, ws, size, None)

    for bad, code in [(dict(dy=None), -1), (dict(h=None), -1), (dict(dx=None), -1), (dict(dt=2), -4), (dict(dt=1), -4), (dict(M=0), -2), (dict(C=0), -2), (dict(eps=-1.0), -2),
                      (dict(lddy=63), -2), (dict(ldh=63), -2), (dict(lddh=63), -2), (dict(lddx=63), -2), (dict(dy=OK + 1), -5), (dict(h=OK + 1), -5), (dict(dh=OK + 1), -5),
                      (dict(dx=OK + 1), -5), (dict(dw=OK + 2), -5), (dict(ws=OK + 8), -5), (dict(C=40000, lddy=40000, ldh=40000, lddh=40000, lddx=40000), -7)]:
        assert rc(**bad) == code, bad


def test_refusals_of_pages(B):
    names = ("counts", "lengths", "n_free", "new_lengths", "new_n_free", "starts", "slots", "positions", "refused", "table", "free")

    def rc(Bsz=2, page=16, width=4, ld=4, capacity=9, rows=10, **at):
        p = {n: at.get(n, OK) for n in names}
        return B.lib().dfa_cache_reserve(p["counts"], p["lengths"], Bsz, page, p["table"], width, ld, p["free"], capacity, p["n_free"], p["new_lengths"], p["new_n_free"],
                                         p["starts"], p["slots"], p["positions"], rows, p["refused"], None)

    for n in names:
        assert rc(**{n: None}) == -1 and rc(**{n: OK + 2}) == -5, n
    assert rc(slots=OK + 4) == -5
    for bad in (dict(Bsz=0), dict(page=8), dict(page=48), dict(page=256), dict(width=0), dict(ld=3), dict(capacity=0), dict(rows=0)):
        assert rc(**bad) == -2, bad
    for bad in (dict(width=1 << 28, ld=1 << 28), dict(rows=2 ** 31 - 1), dict(Bsz=2 ** 31 - 1)):
        assert rc(**bad) == -7, bad

    def release(Bsz=2, page=16, width=4, ld=4, capacity=9, done=OK, lengths=OK, table=OK, free=OK, n_free=OK, refused=OK):
        return B.lib().dfa_cache_release(done, lengths, Bsz, page, table, width, ld, free, capacity, n_free, refused, None)

    for n in ("done", "lengths", "table", "free", "n_free", "refused"):
        assert release(**{n: None}) == -1 and release(**{n: OK + 2}) == -5, n
    for bad in (dict(Bsz=0), dict(page=24), dict(width=0), dict(ld=1), dict(capacity=0)):
        assert release(**bad) == -2, bad


def test_refusals_of_packed_append(B):
    def rc(k=OK, v=OK, s=(0, 128, 64), dt=0, T=5, starts=OK, Bsz=2, cache={}, table=OK, width=2, ld=2, lengths=OK):
        a = dict(k=OK, v=OK, scales=OK, pages=4, heads=2, page=16, D=64)
        a.update(cache)
        st = B.Strides(*s)
        return B.lib().dfa_cache_append_packed(k, v, st, st, dt, T, starts, Bsz, B.Cache(*(a[n] for n in ("k", "v", "scales", "pages", "heads", "page", "D"))), table,
                                               width, ld, lengths, None)

    for bad in (dict(k=None), dict(v=None), dict(starts=None), dict(table=None), dict(lengths=None), dict(cache=dict(k=None)), dict(cache=dict(scales=None))):
        assert rc(**bad) == -1, bad
    for bad in (dict(T=0), dict(Bsz=0), dict(width=0), dict(ld=1), dict(cache=dict(page=8)), dict(cache=dict(D=32)), dict(cache=dict(heads=0)), dict(cache=dict(pages=0))):
        assert rc(**bad) == -2, bad
    for bad in (dict(k=OK + 8), dict(s=(0, 128, 60)), dict(starts=OK + 2), dict(lengths=OK + 2), dict(table=OK + 2), dict(cache=dict(v=OK + 8))):
        assert rc(**bad) == -5, bad
    assert rc(dt=7) == -4 and rc(T=2 ** 31 - 1) == -7 and rc(Bsz=2 ** 30) == -7 and rc(width=1 << 28, ld=1 << 28) == -7


def test_the_attention_reference():
    """By hand: equal keys are a mean; a sequence of one row is its value; gradients are those of autograd."""
    g = torch.Generator().manual_seed(0)
    q, v = torch.randn((6, 2, 4), generator=g), torch.randn((6, 1, 4), generator=g)
    out, lse, _, _ = ref.attention(q, torch.zeros_like(v), v, [0, 1, 5], 0.5, True)
    assert torch.equal(out[0, 1], v[0, 0].double()) and lse[0, 0] == 0
    torch.testing.assert_close(out[3, 0], v[1:4, 0].double().mean(0))
    assert abs(lse[1, 4] - math.log(4)) < 1e-12 and (out[5] == 0).all() and torch.isneginf(lse[:, 5]).all()
    x = [t.double().requires_grad_() for t in (q, torch.randn((6, 1, 4), generator=g), v)]
    dout = torch.randn((6, 2, 4), generator=g).double()
    total = 0.0
    for a, b in ((0, 1), (1, 5)):
        for h in range(2):
            z = (x[0][a:b, h] @ x[1][a:b, 0].t() * 0.5).masked_fill(torch.ones(b - a, b - a, dtype=torch.bool).triu(1), -math.inf)
            total = total + ((z.softmax(1) @ x[2][a:b, 0]) * dout[a:b, h]).sum()
    want = torch.autograd.grad(total, x)
    y = [t.detach() for t in x]
    ref.U[torch.float64] = 0.0
    out, lse, _, _ = ref.attention(*y, [0, 1, 5], 0.5, True)
    grads, _ = ref.attention_backward(*y, out, lse, dout, [0, 1, 5], 0.5, True)
    del ref.U[torch.float64]
    for a, b in zip(grads, want):
        torch.testing.assert_close(a, b)


def test_the_norm_reference():
    h = torch.tensor([[3.0, 4.0]])
    y, _ = ref.norm(h, torch.tensor([1.0, 2.0]), 0.0)
    torch.testing.assert_close(y, torch.tensor([[3.0, 8.0]], dtype=torch.float64) / math.sqrt(12.5))
    x, w = torch.randn((4, 9), dtype=torch.float64, requires_grad=True), torch.randn((9,), dtype=torch.float64, requires_grad=True)
    dy, dh = torch.randn((4, 9), dtype=torch.float64), torch.randn((4, 9), dtype=torch.float64)
    y, _ = ref.norm(x, w, 0.1)
    want = torch.autograd.grad((y * dy).sum() + (x * dh).sum(), (x, w))
    got, _ = ref.norm_backward(dy, x.detach(), w.detach(), 0.1, dh)
    for a, b in zip(got, want):
        torch.testing.assert_close(a, b)


def test_the_reserve_reference():
    table = [[0, 0, 0], [9, 0, 0], [0, 0, 0]]
    got = ref.reserve([20, 1, 0], [0, 16, 0], table, [3, 4, 5, 6], 4, 16, 24)
    assert got == ([20, 17, 0], 1, [0, 20, 21, 21], [6 * 16 + i for i in range(16)] + [5 * 16 + i for i in range(4)] + [4 * 16] + [-1] * 3,
                   list(range(20)) + [16] + [-1] * 3, 0)
    assert table == [[6, 5, 0], [9, 4, 0], [0, 0, 0]]
    assert ref.reserve([33], [16], [[0, 0, 0]], [1, 2], 2, 16, 8)[-1] == 7
