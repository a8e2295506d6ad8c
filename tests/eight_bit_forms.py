"""A size for every form that the operators on 8-bit operands take, with the form: a host test holds the sizes to them, GPU tests run them."""

# dtype of the result, M, N, K -> rows of a tile, shares of the k-steps
PRODUCTS = [
    ("bf16", 4113, 4041, 300, 128, 1), ("bf16", 700, 2000, 1100, 128, 1), ("bf16", 1025, 1030, 20000, 128, 3), ("bf16", 200, 255, 3000, 128, 12),
    ("bf16", 3801, 3801, 300, 256, 1), ("bf16", 4252, 645, 33223, 256, 5),
    ("fp32", 4113, 4041, 300, 128, 1), ("fp32", 1025, 1030, 20000, 128, 7), ("fp32", 300, 500, 20000, 128, 20), ("fp32", 3801, 3801, 300, 256, 1),
    ("fp32", 5209, 917, 5667, 256, 3)]

# dtype, M, N, K -> 16-row blocks of the launch that quantises x itself (0: two launches), rows of a tile
LINEARS = [(dtype, *size) for dtype in ("bf16", "fp32") for size in (
    (1, 64, 4096, 1, 0), (3, 33, 1500, 2, 0), (9, 40, 2000, 2, 0), (17, 100, 2048, 2, 0), (24, 768, 4096, 2, 0), (32, 1000, 2048, 2, 0), (18, 64, 4100, 4, 0),
    (64, 96, 768, 4, 0), (60, 4096, 4096, 0, 128), (65, 97, 768, 0, 128), (3801, 3801, 300, 0, 256))]

# dtype, M, N, K -> tile and shares of dx, of dw, whether one launch multiplies for both
GRADIENTS = [
    ("bf16", 1000, 384, 200, (128, 1), (128, 4), True), ("fp32", 2100, 100, 333, (128, 1), (128, 6), True), ("bf16", 8200, 384, 768, (128, 1), (128, 11), False),
    ("fp32", 8200, 384, 768, (128, 1), (128, 11), False), ("bf16", 5000, 130, 1101, (128, 1), (128, 10), False), ("bf16", 3801, 300, 3801, (256, 1), (128, 2), False),
    ("fp32", 300, 3801, 3801, (128, 2), (256, 1), False)]

# dtype, B, M, H, heads of the cache, D, page, tokens -> query rows of a tile, several tiles, several shares of the walk
ATTENTIONS = [
    ("bf16", 1, 7, 2, 2, 64, 16, 60, 16, False, False), ("bf16", 1, 7, 2, 1, 64, 32, 700, 16, False, True), ("bf16", 1, 20, 1, 1, 64, 64, 60, 32, False, False),
    ("bf16", 1, 33, 2, 2, 64, 128, 60, 32, True, False), ("bf16", 1, 17, 2, 2, 64, 16, 3000, 32, False, True), ("bf16", 1, 33, 4, 1, 64, 64, 3000, 32, True, True),
    ("bf16", 16, 33, 12, 12, 64, 32, 60, 48, False, False), ("bf16", 8, 33, 24, 12, 64, 64, 200, 48, True, False), ("bf16", 1, 47, 12, 12, 64, 64, 3000, 48, False, True),
    ("bf16", 3, 36, 4, 4, 64, 16, 3000, 48, False, True), ("bf16", 3, 33, 12, 3, 64, 128, 3000, 48, True, True),
    ("bf16", 1, 7, 2, 2, 128, 16, 60, 16, False, False), ("bf16", 1, 7, 4, 2, 128, 32, 700, 16, False, True), ("bf16", 1, 17, 1, 1, 128, 64, 60, 32, False, False),
    ("bf16", 1, 33, 2, 1, 128, 128, 60, 32, True, False), ("bf16", 1, 20, 1, 1, 128, 16, 3000, 32, False, True), ("bf16", 1, 33, 4, 1, 128, 64, 3000, 32, True, True),
    ("fp32", 1, 7, 2, 2, 64, 16, 60, 16, False, False), ("fp32", 1, 7, 2, 1, 64, 32, 700, 16, False, True), ("fp32", 1, 20, 1, 1, 64, 64, 60, 32, False, False),
    ("fp32", 1, 33, 2, 2, 64, 128, 60, 32, True, False), ("fp32", 1, 17, 2, 2, 64, 16, 3000, 32, False, True), ("fp32", 1, 33, 4, 1, 64, 64, 3000, 32, True, True),
    ("fp32", 1, 7, 2, 2, 128, 16, 60, 16, False, False), ("fp32", 1, 17, 1, 1, 128, 32, 60, 16, True, False), ("fp32", 1, 7, 4, 2, 128, 64, 700, 16, False, True),
    ("fp32", 1, 17, 2, 1, 128, 128, 700, 16, True, True)]

CODES = {"bf16": 0, "fp32": 1}


def product(B, dtype, M, N, K):
    f = B.describe_quantized(B.CALL_PRODUCT, CODES[dtype], M, N, K)
    return f.tile, f.splits


def linear(B, dtype, M, N, K):
    f = B.describe_quantized(B.CALL_LINEAR, CODES[dtype], M, N, K)
    return f.few_rows, f.tile


def gradients(B, dtype, M, N, K):
    dx, dw = (B.describe_quantized(call, CODES[dtype], M, N, K) for call in (B.CALL_DX, B.CALL_DW))
    assert dx.paired == dw.paired
    return (dx.tile, dx.splits), (dw.tile, dw.splits), bool(dx.paired)


def attention(B, dtype, Bsz, M, H, heads, D, page, tokens):
    """(The binding's default: room for a page more than the tokens need.)"""
    f = B.describe_cache_attention(Bsz, M, H, heads, D, CODES[dtype], (-(-tokens // page) + 1) * page)
    return f.tile_rows, f.row_tiles > 1, f.splits > 1
