"""Plain 64-bit references of the operators on 8-bit operands, in numpy, written from the format's definition: a block's scale is the
smallest 2^e, e >= -126, with max|finite x| <= 448 * 2^e; a value is the e4m3 number nearest to x / 2^e, ties to even; NaN for what is not finite."""
import numpy as np


def e4m3_numbers():
    """The value of every e4m3 code (sign, 4 exponent bits with bias 7, 3 fraction bits; all ones is NaN)."""
    code = np.arange(256)
    exp, frac = (code >> 3) & 15, code & 7
    mag = np.where(exp == 0, frac * 2.0 ** -9, (8 + frac) * 2.0 ** (exp - 10.0))
    mag = np.where((code & 127) == 127, np.nan, mag)
    return np.where(code & 128, -mag, mag)


NUMBERS = e4m3_numbers()


def scale_exponents(amax):
    """The smallest e >= -126 with amax <= 448 * 2^e, by trying."""
    amax = np.asarray(amax, dtype=np.float64)
    e = np.full(amax.shape, -126)
    for _ in range(260):
        short = amax > 448.0 * np.exp2(e.astype(np.float64))
        if not short.any():
            break
        e = e + short
    return e


def to_e4m3(y):
    """The nearest e4m3 number to every y (|y| <= 448), ties to the one whose last fraction bit is 0; NaN for what is not finite."""
    y = np.asarray(y, dtype=np.float64)
    grid = NUMBERS[:127]                                     # ascending magnitudes; the code's last bit is the fraction's
    a = np.where(np.isfinite(y), np.abs(y), 0.0)
    hi = np.clip(np.searchsorted(grid, a, side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = a - grid[lo], grid[hi] - a
    pick = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isfinite(y), np.copysign(grid[pick], y), np.nan)


def finite_max(x, axis):
    return np.where(np.isfinite(x), np.abs(x), 0.0).max(axis=axis)


def quantize(x, block_rows):
    """x [R, C] fp64 -> (values [R, C] of x / 2^e in e4m3, exponents [ceil(C / 128), R])."""
    R, C = x.shape
    values, exps = np.zeros((R, C)), np.zeros((-(-C // 128), R), dtype=np.int64)
    for c in range(0, C, 128):
        for r in range(0, R, 128 if block_rows == 128 else R):
            part = x[r:r + 128, c:c + 128] if block_rows == 128 else x[:, c:c + 128]
            e = scale_exponents(finite_max(part, None if block_rows == 128 else 1))
            e = np.broadcast_to(e, (part.shape[0],))
            values[r:r + part.shape[0], c:c + 128] = to_e4m3(part / np.exp2(e.astype(np.float64))[:, None])
            exps[c // 128, r:r + part.shape[0]] = e
    return values, exps


def held(x, block_rows=1):
    """x as its blocks hold it."""
    values, exps = quantize(x, block_rows)
    return values * np.exp2(exps.astype(np.float64)).repeat(128, 0)[:x.shape[1]].T


def matrix(m):
    """What a binding.QuantizedMatrix holds, fp64 [rows, cols]."""
    import torch
    codes = m.values.detach().cpu().view(torch.uint8).numpy()
    e = m.scales.detach().cpu().numpy()[:, :codes.shape[0]].astype(np.float64) - 127.0
    return (NUMBERS[codes] * np.exp2(e).repeat(128, 0).T[:, :codes.shape[1]])[:, :m.cols]


HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def product_bar(a, b, y, dtype):
    """How far a product may be from the sum in 64 bits.  Any result: each of the K additions in fp32 is off by at most 2^-24 of what has been
    added up in magnitude, and the result is rounded once.  bf16 results come from e4m3 products: of 16 neighbouring k the matrix
    instruction cuts what lies below 2^-13 of the largest product's power of two, at most that much of each of 16."""
    mag = np.abs(a) @ np.abs(b).T
    bar = a.shape[1] * 2.0 ** -24 * mag * 1.01 + 1e-45
    if dtype == "bf16":
        for k in range(0, a.shape[1], 16):
            bar += 16 * 2.0 ** -13 * (np.abs(a[:, None, k:k + 16]) * np.abs(b[None, :, k:k + 16])).max(2)
    return bar * 1.01 + HALF_STEP[dtype] * np.abs(y)


def far(got, want):
    """The 2-norm of the difference over that of the result."""
    return float(np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-300))
