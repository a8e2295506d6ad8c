"""Plain 64-bit reference of the cache of keys and values in e4m3 and of attention over it, in numpy, sequence by sequence."""
import numpy as np

import quantized_ref as ref


class Model:
    """What a binding.KvCache holds: numbers of the e4m3 codes (kept as fp64) and exponents."""

    def __init__(self, cache):
        import torch
        codes = lambda t: ref.NUMBERS[t.cpu().view(torch.uint8).numpy()]
        self.k, self.v = codes(cache.k).copy(), codes(cache.v).transpose(0, 1, 3, 2).copy()      # [pages, heads, P, D]
        self.e = cache.scales.cpu().numpy().astype(np.int64) - 127                               # [pages, heads, 2]
        self.P = self.k.shape[2]

    def append(self, k, v, table, lengths, counts=None):
        """k, v [B, T, heads, D] fp64."""
        B, T, heads, _ = k.shape
        for b in range(B):
            n = T if counts is None else min(max(int(counts[b]), 0), T)
            start = int(lengths[b]) - n
            slots = {}
            for t in range(n):
                pos = start + t
                if 0 <= pos < table.shape[1] * self.P:
                    slots.setdefault(pos // self.P, []).append((pos % self.P, t))
            for at, new in slots.items():
                page = int(table[b, at])
                if not 0 <= page < self.k.shape[0]:
                    continue
                where, rows, first = [s for s, _ in new], [t for _, t in new], new[0][0]
                for i, (x, held) in enumerate(((k, self.k), (v, self.v))):
                    for h in range(heads):
                        fresh = x[b, rows, h]
                        e = int(ref.scale_exponents(ref.finite_max(fresh, None)))
                        if first > 0:
                            old = self.e[page, h, i]
                            e = max(e, int(old))
                            if e > old:
                                held[page, h, :first] = ref.to_e4m3(held[page, h, :first] * 2.0 ** float(old - e))
                        held[page, h, where] = ref.to_e4m3(fresh / 2.0 ** float(e))
                        self.e[page, h, i] = e

    def check(self, cache):
        """The cache holds exactly this."""
        got = Model(cache)
        np.testing.assert_array_equal(got.e, self.e)
        np.testing.assert_array_equal(got.k, self.k)
        np.testing.assert_array_equal(got.v, self.v)

    def sequence(self, b, table, length):
        """(k, v [tokens, heads, D], which of the tokens are on a page)."""
        P, pages = self.P, self.k.shape[0]
        length = min(max(int(length), 0), table.shape[1] * P)
        ids = np.array([int(table[b, n // P]) for n in range(length)], dtype=np.int64)
        there = (ids >= 0) & (ids < pages)
        ids, slot = np.where(there, ids, 0), np.arange(length) % P
        unit = np.exp2(self.e[ids].astype(np.float64))                                           # [tokens, heads, 2]
        return self.k[ids, :, slot] * unit[:, :, :1], self.v[ids, :, slot] * unit[:, :, 1:], there


def attention(model, q, table, lengths, scale, causal, counts=None):
    """(out [B, M, H, D], lse [B, H, M], and their bars without the roundings to the call's type) in fp64.  The bars: scores are fp32 sums of D
    products, so is everything behind them; exponentials and logarithms are good to 2^-21; p_half is the half step that each probability is
    rounded by."""
    B, M, H, D = q.shape
    group = H // model.k.shape[1]
    out, lse = np.zeros((B, M, H, D)), np.full((B, H, M), -np.inf)
    weight, lse_bar = np.zeros((B, M, H, D)), np.zeros((B, H, M))
    loose = np.zeros((B, M, H, 1))
    for b in range(B):
        k, v, there = model.sequence(b, table, lengths[b])
        n = M if counts is None else min(max(int(counts[b]), 0), M)
        for i in range(n):
            end = len(there) - (n - 1 - i) if causal else len(there)
            seen = np.arange(len(there)) < end
            seen &= there
            if not seen.any():
                continue
            for h in range(H):
                kh, vh = k[seen, h // group], v[seen, h // group]
                z = scale * (kh @ q[b, i, h])
                size = scale * (np.abs(kh) @ np.abs(q[b, i, h]))
                top = z.max()
                p = np.exp(z - top)
                out[b, i, h] = p @ vh / p.sum()
                lse[b, h, i] = top + np.log(p.sum())
                delta = (D + 8) * 2.0 ** -24 * size.max() + 2.0 ** -21 * (1 + np.abs(z - top).max() * 2.0 ** -3)
                weight[b, i, h] = p @ np.abs(vh) / p.sum()
                loose[b, i, h] = 2 * delta + 2 * len(p) * 2.0 ** -24
                lse_bar[b, h, i] = delta + len(p) * 2.0 ** -24 + 2.0 ** -21 * max(1.0, abs(lse[b, h, i]))
    return out, lse, weight, loose, lse_bar


def check_attention(got_out, got_lse, want, dtype):
    """Results of cache_attention (torch) against attention() of the same call."""
    out, lse, weight, loose, lse_bar = want
    got, got_l = got_out.double().cpu().numpy(), got_lse.double().cpu().numpy()
    half = ref.HALF_STEP[dtype]
    bar = (half + loose) * weight * 1.01 + half * np.abs(out) + 1e-44
    np.testing.assert_array_equal(np.isnan(got), np.isnan(out))
    fine = ~np.isnan(out)
    err = np.abs(got - out)[fine]
    worst = float((err / bar[fine]).max()) if err.size else 0.0
    assert np.all(err <= bar[fine]), worst
    np.testing.assert_array_equal(np.isneginf(got_l), np.isneginf(lse))
    np.testing.assert_array_equal(np.isnan(got_l), np.isnan(lse))
    fin = np.isfinite(lse)
    off = np.abs(got_l[fin] - lse[fin])
    assert np.all(off <= lse_bar[fin]), float((off / lse_bar[fin]).max())
    return worst
