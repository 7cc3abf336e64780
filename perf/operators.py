"""Decoding with the KV cache and the weights held in 4 bits: what is measured of these operators.

listed() gives fixed cases, draw(rng) further ones of the same ranges, prepare(case, seed) what a program has in hand before
the call, run(state) one pass, work(case) the bytes and operations a pass cannot do without, exact(case, seed) the results
in 64 bits. With ``own`` the passes are calls of the framework, without it elementary torch operations.

The format: groups of 32 neighbouring values share an exponent byte s and stand for code * 2^(s - 127); a code is four bits,
a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, two codes to a byte, the lower index in the lower half. The exponent is the
least one that leaves no magnitude above 7 steps, the code the nearest, ties to the even code.

Operators:
  write    K and V rows into a cache held in 4 bits, at every sample's own next row, and those rows read back
  attn     one new token per sample attending over such a cache
  project  few rows times a matrix held in 4 bits
  pack     a matrix of weights to 4 bits and back
"""
import math

import torch

own = False

GROUP = 32
# (query heads, KV heads, head dimension)
HEADS = {"mha7b": (32, 32, 128), "gqa7b": (28, 4, 128), "small": (16, 16, 128), "small64": (16, 4, 64)}
# (model width, MLP width)
WIDTHS = {"mha7b": (4096, 11008), "gqa7b": (3584, 14336), "small": (2048, 5632), "small64": (1024, 2816)}


# ------------------------------------------------------------------------------------------------------------- cases


def listed():
    return [
        # the new token of 64 conversations appended to caches of different lengths, one layer: a latency
        {"name": "write_token", "op": "write", "model": "mha7b", "B": 64, "T": 1, "capacity": 640, "ragged": False},
        # the caches of four unpruned high-resolution prompts of different lengths, K and V inside fused QKV rows
        {"name": "write_prompts", "op": "write", "model": "mha7b", "B": 4, "T": 2944, "capacity": 4096, "ragged": True},
        # the output projection of one conversation's token: the smallest product
        {"name": "project_token", "op": "project", "M": 1, "N": 4096, "K": 4096, "residual": True},
        # the up projection of seven conversations
        {"name": "project_some", "op": "project", "M": 7, "N": 11008, "K": 4096, "residual": False},
        # the down projection of 64 conversations
        {"name": "project_batch", "op": "project", "M": 64, "N": 4096, "K": 11008, "residual": True},
        # the down projection of a pruned prompt's rows
        {"name": "project_prompt", "op": "project", "M": 317, "N": 3584, "K": 14336, "residual": True},
        # one conversation after a pruned prefill
        {"name": "attn_prompt", "op": "attn", "model": "mha7b", "B": 1, "N": 317, "ragged": False},
        # small grouped heads, 24 short conversations of different lengths, one of them empty: the smallest attention
        {"name": "attn_small", "op": "attn", "model": "small64", "B": 24, "N": 60, "ragged": True},
        # 64 conversations of up to 1536 tokens
        {"name": "attn_batch", "op": "attn", "model": "mha7b", "B": 64, "N": 1536, "ragged": True},
        # four long video conversations, grouped heads
        {"name": "attn_long", "op": "attn", "model": "gqa7b", "B": 4, "N": 65536, "ragged": False},
        # one layer's key projection of a small model, and the up projection of a 7B one
        {"name": "pack_small", "op": "pack", "N": 256, "K": 1024},
        {"name": "pack_up", "op": "pack", "N": 11008, "K": 4096},
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["write", "attn", "attn", "project", "project", "pack"])
    model = rng.choice(list(HEADS))
    if op == "write":
        _, Hkv, d = HEADS[model]
        T = rng.choice([1, _log(rng, 1, 3000)])
        B = _log(rng, 1, max(1, min(64, 11000 * 4096 // (T * Hkv * d))))
        return {"op": op, "model": model, "B": B, "T": T, "capacity": T + _log(rng, 1, 1500), "ragged": rng.random() < 0.5}
    if op == "attn":
        _, Hkv, d = HEADS[model]
        N = _log(rng, 1, 131072)
        most = 180_000_000 // (N * Hkv * d)
        return {"op": op, "model": model, "B": _log(rng, 1, max(1, min(128, most))), "N": min(N, 180_000_000 // (Hkv * d)),
                "ragged": rng.random() < 0.5}
    D, F = WIDTHS[model]
    if op == "project":
        N, K = rng.choice([(D, D), (F, D), (D, F), (256, D), (rng.randrange(16, 6000, 16), rng.randrange(32, 6000, 32))])
        return {"op": op, "M": rng.choice([_log(rng, 1, 16), _log(rng, 1, 64), _log(rng, 1, 317)]), "N": N, "K": K,
                "residual": rng.random() < 0.5}
    N, K = rng.choice([(D, D), (F, D), (_log(rng, 1, 8000), GROUP * _log(rng, 1, 170))])
    return {"op": op, "N": min(N, 45_000_000 // K), "K": K}


def _lengths(case, longest):
    """Rows per sample: the longest one first and, of three samples and more, one that has none."""
    B = case["B"]
    if not case["ragged"]:
        return [longest] * B
    lens = [max(1, int(longest * (1.0 - 0.9 * ((b * 0.6180339887) % 1.0)))) for b in range(B)]
    if B >= 3:
        lens[B // 2] = 0
    return lens


# ------------------------------------------------------------------------------------------ the format, elementary torch


def _power(e):
    """2^e for whole e in [-126, 127], in 32 bits."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _quantise(x):
    """x [..., n], n a multiple of 32 -> (codes [..., n / 2], exponent bytes [..., n / 32])."""
    g = x.float().unflatten(-1, (-1, GROUP))
    mant, exp = torch.frexp(g.abs().amax(-1))
    e = torch.where(mant <= 0.875, exp - 3, exp - 2).clamp(-125, 125)
    e = torch.where(mant == 0, -125, e)
    t = g * _power(-e)[..., None]                    # (a power of two: exact)
    a = t.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
            + 8 * torch.signbit(t)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What codes [..., n / 2] and exponent bytes [..., n / 32] stand for, in 32 bits [..., n]."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                         device=codes.device)
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    v = table[both.int()].unflatten(-1, (-1, GROUP))
    return (v * _power(scales.int() - 127)[..., None]).flatten(-2)


# ------------------------------------------------------------------------------------------------------------ inputs


def _normal(g, shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)


def _rows(g, shape):
    """K or V rows: channels of different gains, a few of them large, as trained projections leave them."""
    gain = torch.exp(0.4 * _normal(g, shape[-2:]))
    return _normal(g, shape) * gain


def _cache(g, B, capacity, Hkv, d):
    """Four tensors of a cache that holds rows already: K and V codes [B,Hkv,capacity,d/2], exponents [.., d/32]."""
    out = {}
    for name in ("k", "v"):
        codes, scales = [], []
        for _ in range(B):                           # (a sample at a time: 32-bit values of a whole batch are large)
            c, s = _quantise(_rows(g, (capacity, Hkv, d)).bfloat16())
            codes.append(c.transpose(0, 1))
            scales.append(s.transpose(0, 1))
        out[name + "_codes"] = torch.stack(codes).contiguous()
        out[name + "_scales"] = torch.stack(scales).contiguous()
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    st = {"op": op}
    if op in ("write", "attn"):
        Hq, Hkv, d = HEADS[case["model"]]
        B = case["B"]
    if op == "write":
        T, capacity = case["T"], case["capacity"]
        st |= _cache(g, B, capacity, Hkv, d)
        rows = torch.empty((B, T, (Hq + 2 * Hkv) * d), dtype=torch.bfloat16, device="cuda")
        for b in range(B):
            rows[b] = _rows(g, (T, Hq + 2 * Hkv, d)).flatten(1)
        st["k"] = rows[:, :, Hq * d:(Hq + Hkv) * d].unflatten(-1, (Hkv, d))
        st["v"] = rows[:, :, (Hq + Hkv) * d:].unflatten(-1, (Hkv, d))
        room = capacity - T
        st["start"] = torch.tensor([(b * 97 + 13) % (room + 1) for b in range(B)], dtype=torch.int32, device="cuda")
        st["count"] = torch.tensor(_lengths(case, T), dtype=torch.int32, device="cuda") if case["ragged"] else None
        st["out"] = [torch.empty((B, T, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    elif op == "attn":
        st |= _cache(g, B, case["N"], Hkv, d)
        st["q"] = _normal(g, (B, Hq, d), 1.5).bfloat16()
        st["N"] = case["N"]
        st["lens"] = torch.tensor(_lengths(case, case["N"]), dtype=torch.int32, device="cuda") if case["ragged"] else None
        st["out"] = (torch.empty((B, Hq, d), dtype=torch.bfloat16, device="cuda"),
                     torch.empty((B, Hq), dtype=torch.float32, device="cuda"))
    elif op == "project":
        M, N, K = case["M"], case["N"], case["K"]
        st["codes"], st["scales"] = _quantise(_normal(g, (N, K), 1.28 / math.sqrt(K)).bfloat16())
        st["x"] = _normal(g, (M, K)).bfloat16()
        st["residual"] = _normal(g, (M, N)).bfloat16() if case["residual"] else None
        st["out"] = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    else:
        st["w"] = _normal(g, (case["N"], case["K"]), 1.28 / math.sqrt(case["K"])).bfloat16()
        st["out"] = torch.empty_like(st["w"])
    return st


# ------------------------------------------------------------------------------------------------------------ passes


def _run_write(st):
    k, v, start, count = st["k"], st["v"], st["start"], st["count"]
    B, T = k.shape[:2]
    row = torch.arange(T, device="cuda")
    at = start[:, None].long() + row                                       # [B,T]
    sample = torch.arange(B, device="cuda")[:, None].expand(B, T)
    live = row < (count[:, None] if count is not None else T)              # rows behind a sample's count stay as they were
    live = live.expand(B, T)
    got = {}
    for name, x in (("k", k), ("v", v)):
        codes, scales = _quantise(x)
        c, s = st[name + "_codes"], st[name + "_scales"]
        c.transpose(1, 2)[sample[live], at[live]] = codes[live]
        s.transpose(1, 2)[sample[live], at[live]] = scales[live]
        got[name] = _values(c.transpose(1, 2)[sample, at], s.transpose(1, 2)[sample, at]).bfloat16()
    return got


def _run_attn(st):
    q, N = st["q"].float(), st["N"]
    B, Hq, d = q.shape
    k = _values(st["k_codes"], st["k_scales"])                             # [B,Hkv,N,d]
    Hkv = k.shape[1]
    s = torch.matmul(q.view(B, Hkv, Hq // Hkv, d), k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    del k
    if st["lens"] is not None:
        live = torch.arange(N, device="cuda") < st["lens"][:, None]
        s = torch.where(live[:, None, None, :], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    base = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(s - base)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, _values(st["v_codes"], st["v_scales"]))
    o = torch.where(total > 0, o / total, 0.0)                             # a sample without rows: zeros
    lse = torch.log(total) + base
    return {"out": o.reshape(B, Hq, d).bfloat16(), "lse": lse.reshape(B, Hq)}


def _run_project(st):
    y = torch.matmul(st["x"].float(), _values(st["codes"], st["scales"]).t())
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return y.bfloat16()


def run(st):
    op = st["op"]
    if own:
        from paper_2601_17818_amd import binding as vc
        if op == "project":
            return vc.vitcop_project_mx4(st["x"], st["codes"], st["scales"], residual=st["residual"], out=st["out"])
        if op == "pack":
            return vc.vitcop_mx4_dequantize(*vc.vitcop_mx4_quantize(st["w"]), out=st["out"])
        cache = vc.CacheMx4(st["k_codes"], st["k_scales"], st["v_codes"], st["v_scales"])
        if op == "attn":
            out, lse = vc.vitcop_decode_attn_mx4(st["q"], cache, st["N"], n_samples=st["lens"], out=st["out"])
            return {"out": out, "lse": lse}
        vc.vitcop_cache_mx4_write(cache, st["k"], st["v"], start_samples=st["start"], n_samples=st["count"])
        k, v = vc.vitcop_cache_mx4_read(cache, st["k"].shape[1], start_samples=st["start"], out=st["out"])
        return {"k": k, "v": v}
    if op == "project":
        return _run_project(st)
    if op == "pack":
        return _values(*_quantise(st["w"])).bfloat16()
    return _run_attn(st) if op == "attn" else _run_write(st)


# -------------------------------------------------------------------------------------------------- what a pass costs


def work(case):
    op = case["op"]
    held = 0.5 + 1.0 / GROUP                                               # bytes a value takes in the format
    if op == "project":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": held * N * K + 2 * M * K + (4 if case["residual"] else 2) * M * N, "flops": 2 * M * N * K}
    if op == "pack":                                                       # to 4 bits, and back
        n = case["N"] * case["K"]
        return {"bytes": 2 * (2 + held) * n, "flops": 4 * n}
    Hq, Hkv, d = HEADS[case["model"]]
    if op == "attn":
        rows = sum(_lengths(case, case["N"]))
        return {"bytes": 2 * held * rows * Hkv * d + 4 * case["B"] * Hq * (d + 1), "flops": 4 * rows * Hq * d}
    written, back = sum(_lengths(case, case["T"])), case["B"] * case["T"]
    return {"bytes": 2 * (2 + held) * Hkv * d * (written + back), "flops": 4 * Hkv * d * (written + back)}


# ---------------------------------------------------------------------------------------------------- in 64 bits


def _power64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _held64(codes, scales):
    """The values of a packed tensor, from a code's bits: exponent in bits 1 and 2, fraction in bit 0, sign in bit 3."""
    n = codes.shape[-1] * 2
    code = torch.empty(codes.shape[:-1] + (n,), dtype=torch.long, device=codes.device)
    code[..., 0::2] = codes.long() % 16
    code[..., 1::2] = codes.long() // 16
    exp, frac = (code // 2) % 4, (code % 2).double()
    size = torch.where(exp == 0, frac * 0.5, (1.0 + 0.5 * frac) * _power64(exp - 1))
    size = torch.where(code >= 8, -size, size)
    return size * _power64(scales.long() - 127).repeat_interleave(GROUP, -1)


def _rounded64(x):
    """x [..., n] as the format holds it: the least exponent that leaves no magnitude above 7, each value to the nearest of
    the sixteen, which are whole multiples of 0.5 up to 2, of 1 up to 4 and of 2 up to 6 (round: ties to even multiples)."""
    g = x.double().reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    top = g.abs().max(-1, keepdim=True).values
    e = torch.full_like(top, -125.0).long()
    guess = torch.floor(torch.log2(top.clamp(min=2.0 ** -120))).long() - 4          # at least one too low
    for _ in range(3):
        guess = torch.where(top > 7.0 * _power64(guess), guess + 1, guess)
    e = torch.maximum(e, guess).clamp(max=125)
    t = g / _power64(e)
    a = t.abs()
    r = torch.where(a < 2.0, torch.round(a * 2.0) / 2.0, torch.where(a < 4.0, torch.round(a), 2.0 * torch.round(a / 2.0)))
    return (torch.copysign(r.clamp(max=6.0), t) * _power64(e)).reshape(x.shape)


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "project":
        y = st["x"].double() @ _held64(st["codes"], st["scales"]).T
        return y if st["residual"] is None else y + st["residual"].double()
    if op == "pack":
        return _rounded64(st["w"])
    B = case["B"]
    Hq, Hkv, d = HEADS[case["model"]]
    if op == "write":
        lens, start, out = _lengths(case, case["T"]), st["start"].tolist(), {}
        for name in ("k", "v"):
            got = []
            for b in range(B):
                at = slice(start[b], start[b] + case["T"])
                x = _held64(st[name + "_codes"][b, :, at], st[name + "_scales"][b, :, at]).transpose(0, 1).clone()
                if lens[b]:
                    x[:lens[b]] = _rounded64(st[name][b, :lens[b]])
                got.append(x)
            out[name] = torch.stack(got)
        return out
    out = torch.zeros((B, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(case, case["N"])):
        for h in range(Hkv if n else 0):
            k = _held64(st["k_codes"][b, h, :n], st["k_scales"][b, h, :n])
            v = _held64(st["v_codes"][b, h, :n], st["v_scales"][b, h, :n])
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            s = st["q"][b, heads].double() @ k.T / math.sqrt(d)
            lse[b, heads] = torch.logsumexp(s, -1)
            out[b, heads] = torch.softmax(s, -1) @ v
    return {"out": out, "lse": lse}
