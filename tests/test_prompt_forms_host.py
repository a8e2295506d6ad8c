"""Which form of prompt attention's forward a call takes: of sizes that were timed both ways, the faster one."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2403_09195_amd import binding
    binding.lib()
    return binding


# dtype, T, H, D, B -> (rows of a tile, groups of waves) causal, not causal
FORMS = [
    # one round of workgroups of half the rows, or less: two groups
    ("bf16", 1000, 16, 128, 1, (64, 2), (64, 2)), ("bf16", 2000, 8, 128, 1, (64, 2), (64, 2)), ("bf16", 2000, 12, 64, 1, (64, 2), (64, 2)),
    # two rounds of heads of 128, one and a half of 64, where the walks of the second are short: causal
    ("bf16", 2000, 16, 128, 1, (64, 2), (128, 1)), ("bf16", 4000, 8, 128, 1, (64, 2), (128, 1)), ("bf16", 2000, 12, 128, 1, (64, 2), (128, 1)),
    ("bf16", 3000, 8, 128, 1, (64, 2), (128, 1)), ("bf16", 4000, 8, 128, 2, (64, 2), (128, 1)), ("bf16", 8000, 4, 128, 1, (64, 2), (128, 1)),
    ("bf16", 3000, 12, 64, 1, (64, 2), (128, 1)), ("bf16", 4000, 12, 64, 1, (64, 2), (128, 1)), ("bf16", 4000, 12, 64, 2, (64, 2), (128, 1)),
    ("bf16", 2000, 24, 64, 1, (64, 2), (128, 1)), ("bf16", 3000, 16, 64, 1, (64, 2), (128, 1)),
    # more: one group
    ("bf16", 2500, 16, 128, 1, (128, 1), (128, 1)), ("bf16", 5000, 8, 128, 1, (128, 1), (128, 1)), ("bf16", 4000, 16, 128, 1, (128, 1), (128, 1)),
    ("bf16", 4000, 16, 128, 2, (128, 1), (128, 1)), ("bf16", 2000, 32, 64, 1, (128, 1), (128, 1)),
    # short walks, and many: one group of 32 rows a wave, or of 64
    ("bf16", 1000, 32, 128, 1, (128, 1), (128, 1)), ("bf16", 300, 16, 128, 1, (128, 1), (128, 1)), ("bf16", 4096, 12, 64, 8, (128, 1), (128, 1)),
    ("bf16", 16384, 32, 64, 1, (256, 1), (256, 1)), ("bf16", 8 * 4096, 12, 64, 8, (256, 1), (256, 1)), ("bf16", 8 * 1024, 24, 64, 8, (128, 1), (256, 1)),
    # fp32
    ("fp32", 1000, 12, 64, 1, (64, 4), (64, 4)), ("fp32", 4096, 12, 64, 8, (64, 2), (64, 2)), ("fp32", 65536, 12, 64, 32, (128, 1), (128, 1)),
    ("fp32", 1000, 12, 128, 1, (64, 2), (64, 2)), ("fp32", 65536, 12, 128, 32, (128, 1), (128, 1))]


def test_sizes_take_the_faster_form(B):
    for dtype, T, H, D, Bsz, *forms in FORMS:
        for causal, form in zip((True, False), forms):
            f = B.describe_prompt_attention(T, H, H, D, {"bf16": 0, "fp32": 1}[dtype], Bsz, causal)
            assert (f.rows, f.groups) == form, (dtype, T, H, D, Bsz, causal)


def test_every_form_has_a_size(B):
    assert {(d, D, f) for d, _, _, D, _, *forms in FORMS for f in forms} == {
        ("bf16", 64, (64, 2)), ("bf16", 64, (128, 1)), ("bf16", 64, (256, 1)), ("bf16", 128, (64, 2)), ("bf16", 128, (128, 1)),
        ("fp32", 64, (64, 4)), ("fp32", 64, (64, 2)), ("fp32", 64, (128, 1)), ("fp32", 128, (64, 2)), ("fp32", 128, (128, 1))}


def test_refusals(B):
    L, f = B.lib(), B.PromptAttentionForm()
    for size, code in (((0, 4, 2, 64, 0, 1), -2), ((10, 3, 2, 64, 0, 1), -2), ((10, 4, 2, 32, 0, 1), -2), ((10, 4, 2, 64, 2, 1), -4), ((10, 4, 2, 64, 0, 0), -2),
                       ((1 << 30, 1 << 12, 1 << 12, 64, 0, 1), -7)):
        assert L.dfa_prompt_attention_describe(*size, 1, ctypes.byref(f)) == code
    assert L.dfa_prompt_attention_describe(10, 4, 2, 64, 0, 1, 1, None) == -1
