"""Plain 64-bit references of the operators on packed prompts, with how far a right result may be from them.

A rounding to bf16 is off by at most U = 2^-8 of the value (half a step), one to fp32 by E = 2^-24.  An fp32 sum of n terms (products included) is off by at
most (n + 2) E of the sum of magnitudes, in any order.  An exponential of a base-2 exponent x in fp32 is off by at most 2^-23 and what x is
off by, which is its own rounding and those of the two factors it is made of: 4 E |x| in all."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
E = 2.0 ** -24


def starts_of(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return s


def sequences(starts):
    return [(a, b) for a, b in zip(starts[:-1], starts[1:]) if b > a]


def _score_error(q, k, scale, z):
    """How far fp32 scores of one head may be off: the sum over d, in bf16 products or in parts (six terms of a product, 3 * 2^-23 left out), then the exponent."""
    D = q.shape[1]
    return scale * ((6 * D + 8) * E) * (q.abs() @ k.abs().t()) + 8 * E * z.abs() + 2.0 ** -22


def _hidden(n, causal, device):
    return torch.ones((n, n), dtype=torch.bool, device=device).triu(1) if causal else torch.zeros((n, n), dtype=torch.bool, device=device)


def attention(q, k, v, starts, scale, causal):
    """(out, lse, bound of out, bound of lse) in 64 bits; rows of no sequence 0 and -inf."""
    T, H, D = q.shape
    group, dt = H // k.shape[1], q.dtype
    f = dict(dtype=torch.float64, device=q.device)
    out, lse, tol, tol_lse = torch.zeros((T, H, D), **f), torch.full((H, T), -math.inf, **f), torch.zeros((T, H, D), **f), torch.zeros((H, T), **f)
    for a, b in sequences(starts):
        n = b - a
        for h in range(H):
            qh, kh, vh = q[a:b, h].double(), k[a:b, h // group].double(), v[a:b, h // group].double()
            z = (qh @ kh.t()) * scale
            err = _score_error(qh, kh, scale, z)
            hide = _hidden(n, causal, q.device)
            z = z.masked_fill(hide, -math.inf)
            worst = err.masked_fill(hide, 0.0).amax(1)                                          # of a row's scores
            lse[h, a:b] = torch.logsumexp(z, 1)
            p = torch.exp(z - lse[h, a:b, None])
            out[a:b, h] = p @ vh
            size = p @ vh.abs()
            # every weight off by its score's error (numerator and denominator), by the sums over n keys (six terms a product in parts), in bf16 by its rounding; then out's own
            tol[a:b, h] = (2 * worst + (7 * n + 80) * E + (U[dt] if dt == torch.bfloat16 else 0.0))[:, None] * size + (U[dt] + 4 * E) * out[a:b, h].abs()
            tol_lse[h, a:b] = worst + (n + 66) * E + 8 * E * lse[h, a:b].abs()
    return out, lse, 1.001 * tol, 1.001 * tol_lse


def attention_backward(q, k, v, out, lse, dout, starts, scale, causal):
    """((dq, dk, dv), (their bounds)) in 64 bits of the formula on these out and lse."""
    T, H, D = q.shape
    group, dt = H // k.shape[1], q.dtype
    f = dict(dtype=torch.float64, device=q.device)
    grads = [torch.zeros((T, n, D), **f) for n in (H, k.shape[1], k.shape[1])]
    tols = [torch.zeros_like(g) for g in grads]
    u = U[dt] if dt == torch.bfloat16 else 0.0
    for a, b in sequences(starts):
        n = b - a
        for h in range(H):
            kv = h // group
            qh, kh, vh, go, o = q[a:b, h].double(), k[a:b, kv].double(), v[a:b, kv].double(), dout[a:b, h].double(), out[a:b, h].double()
            z = (qh @ kh.t()) * scale
            hide = _hidden(n, causal, q.device)
            l = lse[h, a:b].double()
            p = torch.exp(z - l[:, None]).masked_fill(hide, 0.0)
            p_off = _score_error(qh, kh, scale, z) + 8 * E * l.abs()[:, None]                   # relative
            diff = go @ vh.t() - (go * o).sum(1, keepdim=True)
            diff_off = (6 * D + 8) * E * (go.abs() @ vh.abs().t() + (go * o).abs().sum(1, keepdim=True))
            ds = p * diff
            ds_off = ds.abs() * (p_off + u + 4 * E) + p * diff_off * (1 + u)
            sums = (6 * n + 8 * (H // k.shape[1]) + 66) * E
            for i, (g, t, x, rows) in enumerate(((scale * ds @ kh, scale * (ds_off + sums * ds.abs()) @ kh.abs(), None, h),
                                                 (scale * ds.t() @ qh, scale * (ds_off + sums * ds.abs()).t() @ qh.abs(), None, kv),
                                                 (p.t() @ go, (p * (p_off + u + sums)).t() @ go.abs(), None, kv))):
                grads[i][a:b, rows] += g
                tols[i][a:b, rows] += t
    return grads, [1.001 * (t + (U[dt] + 4 * E) * g.abs()) for g, t in zip(grads, tols)]


def norm(x, weight, eps, residual=None):
    """(y, h) in 64 bits."""
    h = x.double() + (residual.double() if residual is not None else 0.0)
    y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + eps)
    return (y * weight.double() if weight is not None else y), h


# fp32 work of the norm beside the roundings of results: at most 32 terms a thread and 16 sums of sums, half of it through the root, and a few roundings
NORM_OFF = 64 * E


def norm_backward(dy, h, weight, eps, dh=None):
    """((dx, dw), (their bounds)) in 64 bits."""
    M, C = h.shape
    h, dy = h.double(), dy.double()
    r = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    u, g = h * r, dy * weight.double() if weight is not None else dy
    mean = (g * u).mean(1, keepdim=True)
    dx = r * (g - u * mean)
    off = NORM_OFF * r * (g.abs() + 3 * u.abs() * (g * u).abs().mean(1, keepdim=True))
    if dh is not None:
        dx = dx + dh.double()
        off = off + 4 * E * dh.double().abs()
    return (dx, (dy * u).sum(0)), (off, ((M + 2) * E + NORM_OFF) * (dy * u).abs().sum(0))


def reserve(counts, lengths, table, free, n_free, page, rows):
    """What dfa_cache_reserve does, in lists: (lengths, n_free, starts, slots, positions, refused), the table changed in place."""
    up = lambda n: -(-n // page)
    bad = 8 if min(counts) < 0 or min(lengths) < 0 else 0
    if not bad:
        taken = sum(up(l + c) - up(l) for l, c in zip(lengths, counts))
        bad = (1 if taken > n_free else 0) | (2 if any(up(l + c) > len(table[0]) for l, c in zip(lengths, counts)) else 0) | (4 if sum(counts) > rows else 0)
    if bad:
        return list(lengths), n_free, [0] * (len(counts) + 1), [-1] * rows, [-1] * rows, bad
    slots, positions = [], []
    for b, (l, c) in enumerate(zip(lengths, counts)):
        for at in range(up(l), up(l + c)):
            n_free -= 1
            table[b][at] = free[n_free]
        for pos in range(l, l + c):
            slots.append(table[b][pos // page] * page + pos % page)
            positions.append(pos)
    fill = [-1] * (rows - len(slots))
    return [l + c for l, c in zip(lengths, counts)], n_free, starts_of(counts), slots + fill, positions + fill, 0
