"""Ordinary calls of the operators on packed prompts are made in native code: each of them, with tensors as a user has them, is answered there."""
import pytest

pytestmark = pytest.mark.gpu

NAMES = ("prompt_attention", "prompt_attention_backward", "rms_norm", "rms_norm_backward", "cache_reserve", "cache_append_packed")


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


@pytest.fixture
def answers(B, monkeypatch):
    """(name, whether native code took it) of every call there is from here on."""
    seen, native = [], B._native_call

    def recorded(name, *args):
        res = native(name, *args)
        seen.append((name, res is not None))
        return res

    monkeypatch.setattr(B, "_native_call", recorded)
    return seen


def _ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention(B, answers, dtype, D):
    import torch
    qkv, starts = torch.randn((90, 8, D), device="cuda").to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]), _ints([0, 30, 30, 85])
    for q, k, v in ((qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]), tuple(t.contiguous() for t in (qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]))):
        for causal in (True, False):
            out, lse = B.prompt_attention(q, k, v, starts, 0.125, causal)
            B.prompt_attention_backward(q, k, v, out, lse, torch.ones_like(out), starts, 0.125, causal)
    assert answers == [(name, True) for _ in range(4) for name in NAMES[:2]]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_norm(B, answers, dtype):
    import torch
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    x, res = (torch.randn((9, 200), device="cuda").to(dt) for _ in range(2))
    calls = 0
    for weight in (None, torch.ones((200,), dtype=dt, device="cuda"), torch.ones((200,), device="cuda")):
        for residual in (None, res):
            for quantized in (False, True, "both"):
                B.rms_norm(x, weight, 1e-6, residual=residual, quantized=quantized)
                calls += 1
    assert answers == [("rms_norm", True)] * calls
    del answers[:]
    for weight in (None, torch.ones((200,), dtype=dt, device="cuda"), torch.ones((200,), device="cuda")):
        for dh in (None, res):
            B.rms_norm_backward(x, res, weight, 1e-6, dh=dh)
    assert answers == [("rms_norm_backward", True)] * 6


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pages(B, answers, dtype):
    import torch
    kv = torch.randn((30, 4, 64), device="cuda").to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype])
    table, cache = _ints([[0] * 4, [0] * 4]), B.kv_cache(9, 2, 16, 64)
    step = B.cache_reserve(_ints([20, 1]), _ints([0, 0]), table, _ints([5, 6, 7, 8]), _ints([4]), 16, 30)
    B.cache_append(kv[:, :2], kv[:, 2:], cache, table, step.lengths, starts=step.starts)
    assert answers == [("cache_reserve", True), ("cache_append_packed", True)]
    assert step.refused.item() == 0 and step.lengths.tolist() == [20, 1]


def test_what_python_marshals(B, answers):
    """Refusals, and results that the caller gives, are Python's: native code leaves them alone."""
    import torch
    q, starts, x = torch.randn((10, 2, 64), device="cuda"), _ints([0, 10]), torch.randn((4, 64), device="cuda")
    with pytest.raises(TypeError):
        B.prompt_attention(q, q, q, starts.long(), 0.125)
    with pytest.raises(B.DfaError):
        B.rms_norm(x, x[0, :-1], 1e-6)
    B.rms_norm(x.t()[:, :3].t(), None, 1e-6, h=torch.empty((3, 64), device="cuda"))
    assert answers == [("prompt_attention", False), ("rms_norm", False)]
