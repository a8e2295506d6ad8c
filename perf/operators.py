"""The 8-bit operators as measured cases: products with e4m3 operands and their gradients, the cache of keys and
values in e4m3, and attention over it.

Format of everything held in 8 bits: e4m3 values in blocks that share a power of two, the smallest 2^e (e >= -126) with
max|finite x| <= 448 * 2^e.  A block's byte is e + 127; a value is the nearest e4m3 number to x / 2^e, ties to even, NaN for
what is not finite.  Blocks: 1 x 128 of a matrix's rows (activations, gradients), 128 x 128 (weights), the tokens of one page
and head (cache).

Where `own` is false the operators are computed in elementary torch operations; where it is true, by the entry points of
`paper_2403_09195_amd.binding`.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128


# ---- cases -------------------------------------------------------------------------------------------------------------------

def _linear(name, M, K, N, dtype="bf16"):
    return {"name": name, "op": "linear", "M": M, "K": K, "N": N, "dtype": dtype}


def _train(name, M, K, N, dtype="bf16"):
    return {"name": name, "op": "train", "M": M, "K": K, "N": N, "dtype": dtype}


def _append(name, B, T, Hkv, D, page, held, dtype="bf16", ragged=False):
    return {"name": name, "op": "append", "B": B, "T": T, "Hkv": Hkv, "D": D, "page": page, "held": held, "dtype": dtype, "ragged": ragged}


def _attend(name, B, M, H, Hkv, D, page, L, causal, dtype="bf16", ragged=False):
    return {"name": name, "op": "attend", "B": B, "M": M, "H": H, "Hkv": Hkv, "D": D, "page": page, "L": L, "causal": causal,
            "dtype": dtype, "ragged": ragged}


def listed():
    return [
        # a projection of one token's activations: the weight is read once, nothing else counts
        _linear("linear_token", 1, 4096, 4096),
        # the fused QKV projection (12 heads of 64) of the prompt tokens of a few sessions, fp32 activations
        _linear("linear_prompts_fp32", 23, 768, 2304, "fp32"),
        # sizes that suit nothing: a row count between the small and the large, features that no tile divides
        _linear("linear_odd", 333, 1000, 1533),
        # a large batch through a wide layer
        _linear("linear_batch", 16384, 4096, 4096),
        # a training step's gradients of the student model's QKV projection (6 heads of 64) on one 512^2 image
        _train("train_512px", 1024, 384, 1152),
        # the same of 12 heads on eight 1024^2 images
        _train("train_batch", 32768, 768, 2304),
        # the step that every generated token takes: one new row per sequence into pages that are partly filled
        _append("append_token", 32, 1, 8, 128, 64, 700, "bf16", True),
        # keys and values of eight encoded 1024^2 images
        _append("append_images", 8, 4096, 12, 64, 64, 0),
        # one prompt token against one encoded image
        _attend("attend_image", 1, 1, 12, 12, 64, 64, 4096, False),
        # a batch of token steps over long caches of unlike lengths, query heads in groups of four
        _attend("attend_batch", 64, 1, 32, 8, 128, 64, 8192, True, "bf16", True),
        # a handful of prompt tokens per image, fp32, small pages, odd lengths
        _attend("attend_prompts_fp32", 5, 9, 12, 6, 64, 16, 4001, False, "fp32", True),
        # a chunk of a long prompt against what is cached, itself included
        _attend("attend_chunk", 2, 1024, 12, 12, 64, 64, 5000, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "train", "append", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op in ("linear", "train"):
        M, K, N = _log_int(rng, 1, 8192), _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)
        if rng.random() < 0.5:
            K, N = -(-K // 64) * 64, -(-N // 64) * 64
        limit = 16384 * 4096 * 4096 if op == "linear" else 32768 * 768 * 2304
        M = max(1, min(M, limit // (K * N)))
        if op == "train":
            return {"op": op, "M": max(M, 16), "K": min(K, 4096), "N": min(N, 4096), "dtype": dtype}
        return {"op": op, "M": M, "K": K, "N": N, "dtype": dtype}
    Hkv, D, page = rng.choice([1, 2, 3, 4, 6, 8, 12, 16]), rng.choice([64, 64, 128]), rng.choice([16, 32, 64, 64, 128])
    if op == "append":
        T = _log_int(rng, 1, 4096) if rng.random() < 0.6 else 1
        B = max(1, min(_log_int(rng, 1, 64), 32768 // T))
        return {"op": op, "B": B, "T": T, "Hkv": Hkv, "D": D, "page": page, "held": rng.choice([0, _log_int(rng, 1, 2000)]), "dtype": dtype,
                "ragged": rng.random() < 0.5}
    B, L = _log_int(rng, 1, 64), _log_int(rng, 1, 16384)
    M = 1 if rng.random() < 0.5 else min(_log_int(rng, 1, 512), L)
    H = Hkv * rng.choice([1, 1, 2, 4, 8])
    B = max(1, min(B, 64 * 8192 * 8 * 128 // (L * Hkv * D), 2 * 1024 * 12 * 5000 * 64 // (M * H * L * D)))
    return {"op": op, "B": B, "M": M, "H": H, "Hkv": Hkv, "D": D, "page": page, "L": L, "causal": rng.random() < 0.6, "dtype": dtype,
            "ragged": rng.random() < 0.5}


# ---- what a user's program has in hand ---------------------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _spread(n, lo, hi, ragged):
    """n whole numbers in [lo, hi]: all hi, or spread over the range in no order, the same for every seed."""
    return [hi if not ragged or b == 0 else lo + (b * 2654435761 % 1000003) * (hi - lo + 1) // 1000003 for b in range(n)]


def _held(case):
    """Tokens that each sequence holds before an append, and new ones."""
    return _spread(case["B"], case["held"] // 2, case["held"], case["ragged"]), _spread(case["B"], 1, case["T"], case["ragged"])


def _lengths(case):
    return _spread(case["B"], min(case["M"], case["L"]), case["L"], case["ragged"])


def _whole(n, of):
    return -(-n // of) * of


def _exponents(amax):
    """The smallest e >= -126 with amax <= 448 * 2^e (448 = 0.875 * 2^9)."""
    f, k = torch.frexp(amax)
    return torch.where(amax > 0, k - 9 + (f > 0.875).int(), -126).clamp(min=-126)


def _finite_max(x, dim):
    return torch.where(x.isfinite(), x.abs(), 0.0).amax(dim)


def _quantize(x, square):
    """x [R, C] -> (values [R, C'] e4m3, bytes [C' / 128, R'] uint8): C' = C rounded up to 128, zeros behind C; R' = R rounded up to 16."""
    R, C = x.shape
    side = BLOCK if square else 1
    Rp, Cp = _whole(R, side), _whole(C, BLOCK)
    full = torch.zeros((Rp, Cp), dtype=torch.float32, device=x.device)
    full[:R, :C] = x
    tiles = full.view(Rp // side, side, Cp // BLOCK, BLOCK)
    e = _exponents(_finite_max(tiles, (1, 3)))
    values = torch.ldexp(tiles, -e[:, None, :, None]).view(Rp, Cp)[:R].to(torch.float8_e4m3fn)
    scales = torch.full((Cp // BLOCK, _whole(R, 16)), 1, dtype=torch.uint8, device=x.device)
    scales[:, :R] = (e + 127).to(torch.uint8).repeat_interleave(side, 0)[:R].t()
    return values, scales


def _normal(gen, shape, dtype, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _activations(gen, shape, dtype):
    """Rows of unlike size with a few large channels, as between layers of a network."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    x.mul_(torch.exp2(torch.randn((shape[0], 1), generator=gen, device="cuda")))
    x.mul_(torch.exp2(torch.randn((1, shape[1]), generator=gen, device="cuda").clamp(min=0.0)))
    return x.to(dtype)


def _cache(gen, pages, Hkv, D, page):
    """Pages full of normal keys and values: k [pages, Hkv, page, D], v [pages, Hkv, D, page] in e4m3, bytes [pages, Hkv, 2] (k, v)."""
    held, scales = [], torch.empty((pages, Hkv, 2), dtype=torch.uint8, device="cuda")
    for i, shape in enumerate(((pages, Hkv, page, D), (pages, Hkv, D, page))):
        x = _normal(gen, shape, torch.float32)
        e = _exponents(x.abs().amax((2, 3)))
        held.append(torch.ldexp(x, -e[:, :, None, None]).to(torch.float8_e4m3fn))
        scales[:, :, i] = (e + 127).to(torch.uint8)
    return held[0], held[1], scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s, dt = dict(case), _dtype(case)
    if case["op"] in ("linear", "train"):
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = _activations(gen, (M, K), dt)
        w = _normal(gen, (N, K), torch.float32, K ** -0.5)
        if case["op"] == "linear":
            s["w"] = _quantize(w, True)
        else:
            s["dy"] = _activations(gen, (M, N), dt)
            s["wt"] = _quantize(w.t(), True)
        return s
    page, D, Hkv, B = case["page"], case["D"], case["Hkv"], case["B"]
    if case["op"] == "append":
        held, new = _held(case)
        width = max(h // page for h in held) + (case["T"] + page - 2) // page + 1
        s["lengths"] = torch.tensor([h + n for h, n in zip(held, new)], dtype=torch.int32, device="cuda")
        s["counts"] = torch.tensor(new, dtype=torch.int32, device="cuda") if case["ragged"] else None
        s["kn"], s["vn"] = (_normal(gen, (B, case["T"], Hkv, D), dt) for _ in range(2))
    else:
        width = -(-case["L"] // page)
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        s["q"] = _normal(gen, (B, case["M"], case["H"], D), dt)
    s["k"], s["v"], s["scales"] = _cache(gen, B * width, Hkv, D, page)
    s["table"] = torch.randperm(B * width, generator=gen, device="cuda").to(torch.int32).view(B, width)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------------

def _values(values, scales, cols):
    """A quantised matrix [R, C'] in 32 bits, without the columns behind `cols`."""
    R, Cp = values.shape
    e = scales[:, :R].t().int() - 127
    return torch.ldexp(values.float().view(R, Cp // BLOCK, BLOCK), e[:, :, None]).view(R, Cp)[:, :cols]


def _rounded(x):
    """x [R, C] as its 1 x 128 blocks hold it, in 32 bits."""
    return _values(*_quantize(x, False), x.shape[1])


def _append_plain(s):
    page, Hkv, D, T = s["page"], s["Hkv"], s["D"], s["T"]
    lengths, B = s["lengths"].long(), s["B"]
    n = s["counts"].long() if s["counts"] is not None else torch.full_like(lengths, T)
    start = lengths - n
    J = (T + page - 2) // page + 1                                                # pages that T tokens can touch
    at = start[:, None] // page + torch.arange(J, device=lengths.device)          # [B, J] places in the table
    ids = torch.gather(s["table"].long(), 1, at).view(-1)
    pos = at[:, :, None] * page + torch.arange(page, device=lengths.device)       # [B, J, page] token numbers
    t = pos - start[:, None, None]
    new = (t >= 0) & (t < n[:, None, None])
    old = (t < 0).view(-1, 1, page, 1)
    touched, kept = new.any(2).view(-1, 1), (t < 0).any(2).view(-1, 1)
    new = new.view(-1, 1, page, 1)
    rows = (torch.arange(B, device=t.device)[:, None, None] * T + t.clamp(0, T - 1)).view(-1)
    for i, (x, held) in enumerate(((s["kn"], s["k"]), (s["vn"], s["v"].transpose(2, 3)))):
        fresh = x.reshape(B * T, Hkv, D)[rows].view(B * J, page, Hkv, D).transpose(1, 2).float()
        before = s["scales"][ids, :, i]
        e = _exponents(_finite_max(torch.where(new, fresh, 0.0), (2, 3)))
        old_e = before.int() - 127
        e = torch.where(kept, torch.maximum(e, old_e), e)
        codes = held[ids]
        moved = torch.ldexp(codes.float(), (old_e - e)[:, :, None, None]).to(torch.float8_e4m3fn)
        put = torch.ldexp(fresh, -e[:, :, None, None]).to(torch.float8_e4m3fn)
        bits = torch.where(new, put.view(torch.uint8), torch.where(old & touched[:, :, None, None], moved.view(torch.uint8), codes.view(torch.uint8)))
        held.view(torch.uint8)[ids] = bits
        s["scales"][ids, :, i] = torch.where(touched, (e + 127).to(torch.uint8), before)
    return s["k"], s["v"], s["scales"]


def _attend_plain(s):
    B, M, H, Hkv, D, page = (s[n] for n in ("B", "M", "H", "Hkv", "D", "page"))
    L, table = s["table"].shape[1] * page, s["table"].long()
    e = s["scales"][table].int() - 127                                            # [B, width, Hkv, 2]
    k = torch.ldexp(s["k"][table].float(), e[..., 0, None, None]).transpose(1, 2).reshape(B, Hkv, L, D)
    v = torch.ldexp(s["v"][table].float(), e[..., 1, None, None]).permute(0, 2, 1, 4, 3).reshape(B, Hkv, L, D)
    q = s["q"].float().view(B, M, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    scores = (torch.matmul(q, k.transpose(2, 3)) * D ** -0.5).view(B, H, M, L)
    ends = s["lengths"].long()[:, None].expand(B, M)
    if s["causal"]:
        ends = ends - (M - 1) + torch.arange(M, device=ends.device)
    seen = torch.arange(L, device=ends.device) < ends[:, :, None]                 # [B, M, L]
    scores = torch.where(seen[:, None], scores, -math.inf)
    top = scores.amax(3, keepdim=True)
    p = torch.exp(scores - torch.where(top.isfinite(), top, 0.0))
    total = p.sum(3, keepdim=True)
    out = torch.matmul((p / torch.where(total > 0, total, 1.0)).view(B, Hkv, -1, L), v).view(B, H, M, D).transpose(1, 2)
    return out.to(s["q"].dtype).contiguous(), (top + torch.log(total)).view(B, H, M)


def run(s):
    if own:
        from paper_2403_09195_amd import binding
        if s["op"] == "linear":
            return binding.quantized_linear(s["x"], binding.QuantizedMatrix(*s["w"], s["K"]))
        if s["op"] == "train":
            return binding.quantized_linear_backward(s["dy"], s["x"], binding.QuantizedMatrix(*s["wt"], s["N"]))
        cache = binding.KvCache(s["k"], s["v"], s["scales"])
        if s["op"] == "append":
            binding.cache_append(s["kn"], s["vn"], cache, s["table"], s["lengths"], counts=s["counts"])
            return cache.k, cache.v, cache.scales
        return binding.cache_attention(s["q"], cache, s["table"], s["lengths"], s["D"] ** -0.5, causal=s["causal"])
    if s["op"] == "linear":
        return torch.matmul(_rounded(s["x"]), _values(*s["w"], s["K"]).t()).to(s["x"].dtype)
    if s["op"] == "train":
        dx = torch.matmul(_rounded(s["dy"]), _values(*s["wt"], s["N"]).t())
        return dx.to(s["dy"].dtype), torch.matmul(_rounded(s["dy"].t()), _rounded(s["x"].t()).t())
    return _append_plain(s) if s["op"] == "append" else _attend_plain(s)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("linear", "train"):
        M, K, N = case["M"], case["K"], case["N"]
        weight = N * K + N * K // BLOCK
        if case["op"] == "linear":
            return {"bytes": (M * K + M * N) * size + weight, "flops": 2 * M * K * N}
        return {"bytes": (2 * M * K + M * N) * size + weight + 4 * N * K, "flops": 4 * M * K * N}
    Hkv, D, B = case["Hkv"], case["D"], case["B"]
    if case["op"] == "append":
        return {"bytes": sum(_held(case)[1]) * Hkv * D * 2 * (size + 1), "flops": 0}
    lengths, M, H = _lengths(case), case["M"], case["H"]
    pairs = sum(sum(max(0, n - M + 1 + i) for i in range(M)) if case["causal"] else n * M for n in lengths)
    return {"bytes": sum(lengths) * Hkv * D * 2 + B * M * H * (D * 2 * size + 4), "flops": 4 * D * H * pairs}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------------

def _e4m3(y):
    """The nearest e4m3 numbers to y, |y| <= 448: steps of an eighth of the power of two below, 2^-9 at least; ties to even."""
    size = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -60)))
    size = torch.where(torch.exp2(size) > y.abs(), size - 1, torch.where(torch.exp2(size + 1) <= y.abs(), size + 1, size))
    step = torch.exp2(size.clamp(min=-6.0) - 3)
    return torch.round(y / step) * step


def _smallest(amax):
    """2^e of a block with this maximum."""
    e = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -130) / 448))
    e = torch.where(448 * torch.exp2(e - 1) >= amax, e - 1, torch.where(448 * torch.exp2(e) < amax, e + 1, e))
    return torch.exp2(e.clamp(min=-126))


def _held_exactly(x):
    """x as its 1 x 128 blocks hold it."""
    parts = []
    for c in range(0, x.shape[1], BLOCK):
        part = x[:, c:c + BLOCK].double()
        unit = _smallest(part.abs().amax(1, keepdim=True))
        parts.append(_e4m3(part / unit) * unit)
    return torch.cat(parts, 1)


def _units(scales):
    return torch.exp2(scales.double() - 127)


def _matrix_exactly(values, scales, cols):
    unit = _units(scales[:, :values.shape[0]]).t()
    return torch.cat([values[:, c * BLOCK:(c + 1) * BLOCK].double() * unit[:, c:c + 1] for c in range(unit.shape[1])], 1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        return _held_exactly(s["x"]) @ _matrix_exactly(*s["w"], s["K"]).t()
    if case["op"] == "train":
        dx = _held_exactly(s["dy"]) @ _matrix_exactly(*s["wt"], s["N"]).t()
        return dx, _held_exactly(s["dy"].t().contiguous()) @ _held_exactly(s["x"].t().contiguous()).t()
    page, D, Hkv, B = case["page"], case["D"], case["Hkv"], case["B"]
    lengths, table = s["lengths"].tolist(), s["table"].tolist()
    if case["op"] == "append":
        held, new = _held(case)
        k, v, scales = s["k"].double(), s["v"].double(), s["scales"].clone()
        for b in range(B):
            done = 0
            while done < new[b]:
                pos = held[b] + done
                first, p = pos % page, table[b][pos // page]
                n = min(page - first, new[b] - done)
                for i, (x, pool) in enumerate(((s["kn"], k), (s["vn"], v.transpose(2, 3)))):
                    rows = x[b, done:done + n].double().transpose(0, 1)           # [Hkv, n, D]
                    unit = _smallest(rows.abs().amax((1, 2)))
                    if first:
                        before = _units(scales[p, :, i])
                        unit = torch.maximum(unit, before)
                        pool[p, :, :first] = _e4m3(pool[p, :, :first] * (before / unit)[:, None, None])
                    pool[p, :, first:first + n] = _e4m3(rows / unit[:, None, None])
                    scales[p, :, i] = (torch.log2(unit) + 127).to(torch.uint8)
                done += n
        return k, v, scales
    M, H = case["M"], case["H"]
    out = torch.zeros((B, M, H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, M), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, ids = lengths[b], s["table"][b].long()
        unit = _units(s["scales"][ids])                                           # [width, Hkv, 2]
        k = (s["k"][ids].double() * unit[:, :, 0, None, None]).permute(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :n]
        v = (s["v"][ids].double() * unit[:, :, 1, None, None]).permute(1, 0, 3, 2).reshape(Hkv, -1, D)[:, :n]
        k, v = (x.repeat_interleave(H // Hkv, 0) for x in (k, v))                 # [H, n, D]
        z = torch.bmm(s["q"][b].double().transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) / math.sqrt(D)
        if case["causal"]:
            hidden = torch.ones((M, n), dtype=torch.bool, device="cuda").triu(n - M + 1)
            z = z.masked_fill(hidden, -math.inf)
        lse[b] = torch.logsumexp(z, 2)
        out[b] = torch.bmm(torch.exp(z - lse[b][:, :, None]), v).transpose(0, 1)
    return out, lse
