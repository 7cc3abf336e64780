"""Prompts and drafts of an image or video conversation over a bf16 KV cache: what is measured of these operators.

listed() gives fixed cases, draw(rng) further ones of the same ranges, prepare(case, seed) what a program has in hand before
the call, run(state) one pass, work(case) the bytes and operations a pass cannot do without, exact(case, seed) the results
in 64 bits. With ``own`` the passes are calls of the framework, without it elementary torch operations.

Operators:
  rope    rotary embedding with one position for each of several axes (time, height, width): the queries turned into a buffer
          of their own, the keys turned and the values copied into the rows of a cache. Channel pair (i, i + d/2) turns by
          position * theta^(-2i/d) of the axis that the pair belongs to
  window  attention of T tokens at the end of a cache, each over the last `window` rows up to its own (0: all of them) and
          the first `sinks` rows
  tree    attention of up to 64 drafted tokens over a cache and over those of the drafts that a bit mask names
  append  rows chosen from the drafts' keys and values (the accepted path of a tree) to the end of the caches of all layers
"""
import math

import torch

own = False

# (query heads, KV heads, head dimension)
HEADS = {"mha7b": (32, 32, 128), "gqa7b": (28, 4, 128), "small": (16, 16, 128), "small64": (16, 4, 64)}
# pairs of channels that turn with time, height and width
SECTIONS = {128: (16, 24, 24), 64: (8, 12, 12)}


# ------------------------------------------------------------------------------------------------------------- cases


def listed():
    return [
        # the new token of one conversation, its key and value appended: a latency
        {"name": "rope_token", "op": "rope", "model": "gqa7b", "B": 1, "T": 1, "ragged": False, "interleaved": False},
        # four image prompts, right-padded
        {"name": "rope_images", "op": "rope", "model": "mha7b", "B": 4, "T": 640, "ragged": True, "interleaved": False},
        # two long video prompts, pairs dealt to the axes in turn
        {"name": "rope_videos", "op": "rope", "model": "gqa7b", "B": 2, "T": 6400, "ragged": False, "interleaved": True},
        # one conversation's next token, four first tokens and a window: a latency
        {"name": "window_token", "op": "window", "model": "mha7b", "B": 1, "T": 1, "start": 2944, "window": 1024, "sinks": 4,
         "ragged": False},
        # the next token of 64 conversations of different lengths, grouped heads
        {"name": "window_tokens", "op": "window", "model": "gqa7b", "B": 64, "T": 1, "start": 8192, "window": 4096, "sinks": 4,
         "ragged": True},
        # another question of 317 tokens at the end of one long video conversation
        {"name": "window_question", "op": "window", "model": "gqa7b", "B": 1, "T": 317, "start": 16384, "window": 0, "sinks": 0,
         "ragged": False},
        # two long video prompts
        {"name": "window_prompts", "op": "window", "model": "gqa7b", "B": 2, "T": 8192, "start": 0, "window": 2048, "sinks": 16,
         "ragged": True},
        # eight drafted tokens after one pruned prompt
        {"name": "tree_small", "op": "tree", "model": "mha7b", "B": 1, "T": 8, "start": 384, "ragged": False},
        # 16 conversations, 25 drafted tokens each, one of them without any
        {"name": "tree_batch", "op": "tree", "model": "mha7b", "B": 16, "T": 25, "start": 2000, "ragged": True},
        # 64 drafted tokens of eight conversations, grouped heads: 448 query rows share a row of the cache
        {"name": "tree_wide", "op": "tree", "model": "gqa7b", "B": 8, "T": 64, "start": 4096, "ragged": False},
        # the accepted path of one conversation's eight drafts, all layers
        {"name": "append_path", "op": "append", "model": "mha7b", "layers": 32, "B": 1, "T": 8, "rows": 4},
        # the accepted paths of 32 conversations, all layers
        {"name": "append_paths", "op": "append", "model": "gqa7b", "layers": 28, "B": 32, "T": 64, "rows": 12},
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "window", "window", "window", "tree", "tree", "append"])
    model = rng.choice(list(HEADS))
    Hq, Hkv, d = HEADS[model]
    if op == "rope":
        T = rng.choice([1, _log(rng, 1, 6400)])
        B = _log(rng, 1, max(1, min(64, 11000 * 4096 // (T * (Hq + 2 * Hkv) * d))))
        return {"op": op, "model": model, "B": B, "T": T, "ragged": rng.random() < 0.5, "interleaved": rng.random() < 0.5}
    if op == "window":
        T = rng.choice([1, 1, _log(rng, 1, 64), _log(rng, 1, 8192)])
        start = rng.choice([0, _log(rng, 1, 32768 if T <= 64 else 8192)])
        window = rng.choice([0, _log(rng, 1, 8192), _log(rng, 256, 4096)])
        sinks = rng.choice([0, rng.randrange(1, 8), _log(rng, 1, 300)])
        T = min(T, 280_000_000_000 // (4 * Hq * d * min(start + T, window + sinks if window else start + T)))
        most = min(280_000_000_000 // (4 * Hq * d * T * min(start + T, window + sinks if window else start + T)),
                   2 * 28 * 8192 ** 2 // (Hq * T * (start + T)), 105_000_000 // ((start + T) * Hkv * d + T * Hq * d))
        return {"op": op, "model": model, "B": _log(rng, 1, max(1, min(64, most))), "T": T, "start": start, "window": window,
                "sinks": sinks, "ragged": rng.random() < 0.5}
    if op == "tree":
        T, start = _log(rng, 1, 64), rng.choice([0, _log(rng, 1, 16384), _log(rng, 1, 16384), _log(rng, 1, 16384)])
        most = min(105_000_000 // ((start + T) * Hkv * d + T * Hq * d), 280_000_000_000 // (4 * Hq * d * T * (start + T)))
        return {"op": op, "model": model, "B": _log(rng, 1, max(1, min(64, most))), "T": T, "start": start,
                "ragged": rng.random() < 0.5}
    layers, T = _log(rng, 1, 32), _log(rng, 1, 64)
    B = _log(rng, 1, max(1, min(64, 4_000_000 // (layers * T * Hkv * d // 16))))
    return {"op": op, "model": model, "layers": layers, "B": B, "T": T, "rows": rng.randint(1, min(T, 16))}


def _lengths(case, longest, least=1):
    """A count per sample: the longest first and, of three samples and more, one that has none."""
    B = case["B"]
    if not case["ragged"]:
        return [longest] * B
    lens = [max(min(least, longest), int(longest * (1.0 - 0.9 * ((b * 0.6180339887) % 1.0)))) for b in range(B)]
    if B >= 3:
        lens[B // 2] = 0
    return lens


def _starts(case):
    """Rows in the cache before the call: the longest first, one of five samples and more without any."""
    B, start = case["B"], case["start"]
    if not case["ragged"]:
        return [start] * B
    lens = [int(start * (1.0 - 0.9 * ((b * 0.7548776662) % 1.0))) for b in range(B)]
    if B >= 5:
        lens[B - 2] = 0
    return lens


def _accepted(case):
    """Drafts that a sample accepts, at least one."""
    return [1 + (b * 7 + case["rows"] - 1) % case["rows"] for b in range(case["B"])]


# ------------------------------------------------------------------------------------------------------------ inputs


def _normal(g, shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)


def _rows(g, shape):
    """K or V rows [..., heads, d]: channels of different gains, a few of them large, as trained projections leave them."""
    gain = torch.exp(0.4 * _normal(g, shape[-2:]))
    return (_normal(g, shape) * gain).bfloat16()


def _cache(g, B, capacity, Hkv, d):
    gain = torch.exp(0.4 * _normal(g, (Hkv, d)))     # (a sample at a time: 32-bit values of a whole batch are large)
    return torch.stack([(_normal(g, (capacity, Hkv, d)) * gain).bfloat16() for _ in range(B)])


def _ints(values, shape=None):
    t = torch.tensor(values, dtype=torch.int32, device="cuda")
    return t if shape is None else t.view(shape)


def _positions(g, B, T):
    """[3,B,T]: some text, frames of 14 x 14 patches of which pruning left two in three, each sample's at a place of its own."""
    t = torch.arange(T, device="cuda")
    patch = (t * 3) // 2
    text = min(35, T)
    first = torch.randint(0, 30000, (B, 1), device="cuda", generator=g)
    grid = torch.stack([patch // 196, patch % 196 // 14, patch % 14])[:, None] + text
    axes = torch.where(t < text, t, grid)
    return (axes + first).to(torch.int32).contiguous()


def _trees(g, B, T):
    """[B,T] bit masks: a drafted token sees itself and its ancestors, which have lower numbers."""
    t = torch.arange(T, device="cuda")
    parent = t - 1 - (torch.rand((B, T), device="cuda", generator=g) * (t.clamp(max=6) + 1)).long()    # one of the last six
    parent = torch.where(torch.rand((B, T), device="cuda", generator=g) < 0.1, -1, parent)             # or none
    step = (parent[:, :, None] == t) | (t[:, None] == t)
    sees = torch.linalg.matrix_power(step.double(), T) > 0
    return (sees.long() << t).sum(-1)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    Hq, Hkv, d = HEADS[case["model"]]
    B, T = case["B"], case["T"]
    st = {"op": op}
    if op == "append":
        L, R = case["layers"], case["rows"]
        capacity = 4 * R + 32
        st["k_cache"], st["v_cache"] = (_rows(g, (L, B, capacity, Hkv, d)) for _ in range(2))
        st["k"], st["v"] = (_rows(g, (L, B, T, Hkv, d)) for _ in range(2))
        # a path goes down the tree: drafts of rising numbers; each layer's caches have lengths of their own
        path = torch.rand((B, T), device="cuda", generator=g).argsort(1)[:, :R].sort(1).values
        st["path"] = path.to(torch.int32).contiguous()
        st["count"] = _ints(_accepted(case))
        st["starts"] = torch.randint(0, capacity - R + 1, (L, B), device="cuda", generator=g).to(torch.int32)
        return st
    if op == "rope":
        capacity = T + 300
        rows = torch.empty((B, T, (Hq + 2 * Hkv) * d), dtype=torch.bfloat16, device="cuda")
        for b in range(B):
            rows[b] = _rows(g, (T, Hq + 2 * Hkv, d)).flatten(1)
        st["q"] = rows[:, :, :Hq * d].unflatten(-1, (Hq, d))               # side by side in fused QKV rows
        st["k"] = rows[:, :, Hq * d:(Hq + Hkv) * d].unflatten(-1, (Hkv, d))
        st["v"] = rows[:, :, (Hq + Hkv) * d:].unflatten(-1, (Hkv, d))
        st["positions"] = _positions(g, B, T)
        st["sections"], st["theta"], st["interleaved"] = SECTIONS[d], 1000000.0, case["interleaved"]
        st["start"] = _ints([(b * 97 + 13) % 301 for b in range(B)])
        st["count"] = _ints(_lengths(case, T)) if case["ragged"] else None
        st["k_cache"], st["v_cache"] = (torch.zeros((B, capacity, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        st["out"] = torch.zeros((B, T, Hq, d), dtype=torch.bfloat16, device="cuda")
    else:
        start = case["start"]
        rows = start + T if op == "window" else max(start, 1)
        st["k_cache"], st["v_cache"] = (_cache(g, B, rows, Hkv, d) for _ in range(2))
        st["q"] = _normal(g, (B, T, Hq, d), 1.5).bfloat16()
        st["start"] = start
        st["starts"] = _ints(_starts(case)) if case["ragged"] else None
        st["count"] = _ints(_lengths(case, T)) if case["ragged"] else None
        st["out"] = (torch.zeros((B, T, Hq, d), dtype=torch.bfloat16, device="cuda"),
                     torch.zeros((B, Hq, T), dtype=torch.float32, device="cuda"))
        if op == "window":
            st["window"], st["sinks"] = case["window"], case["sinks"]
        else:
            st["k"], st["v"] = (_rows(g, (B, T, Hkv, d)) for _ in range(2))
            st["tree"] = _trees(g, B, T)
    return st


# ------------------------------------------------------------------------------------------------------------ passes


def _axis_of_pairs(sections, interleaved):
    """The axis of each pair of channels: section after section, or one pair to each axis in turn while it has some left."""
    if not interleaved:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    return [a for i in range(max(sections)) for a, n in enumerate(sections) if i < n]


def _run_rope(st):
    q, k, v = st["q"], st["k"], st["v"]
    B, T, _, d = q.shape
    axis = torch.tensor(_axis_of_pairs(st["sections"], st["interleaved"]), device="cuda")
    pair = torch.arange(d // 2, dtype=torch.float64, device="cuda")
    angle = st["positions"][axis].permute(1, 2, 0).double() * torch.pow(st["theta"], -2.0 * pair / d)      # [B,T,d/2]
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]

    def turned(x):
        lo, hi = x[..., :d // 2].float(), x[..., d // 2:].float()
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).bfloat16()

    row = torch.arange(T, device="cuda")
    live = (row < (st["count"][:, None] if st["count"] is not None else T)).expand(B, T)   # rows behind a sample's: as they were
    at = st["start"][:, None].long() + row
    sample = torch.arange(B, device="cuda")[:, None].expand(B, T)
    st["k_cache"][sample[live], at[live]] = turned(k)[live]
    st["v_cache"][sample[live], at[live]] = v[live]
    return {"q": torch.where(live[:, :, None, None], turned(q), st["out"]), "k": st["k_cache"], "v": st["v_cache"]}


def _attend(q, k, v, seen):
    """q [B,T,Hq,d], k, v [B,N,Hkv,d], seen [B,T,N] -> out [B,T,Hq,d] and lse [B,Hq,T] in 32 bits; nothing seen: 0 and -inf."""
    B, T, Hq, d = q.shape
    N, Hkv = k.shape[1:3]
    qg = q.float().view(B, T, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    s = torch.matmul(qg, k.float().permute(0, 2, 3, 1).contiguous()).view(B, Hkv, -1, T, N) * (1.0 / math.sqrt(d))
    s = torch.where(seen[:, None, None], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    base = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(s - base)
    del s
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, -1, N), v.float().transpose(1, 2).contiguous()).view(B, Hkv, -1, T, d)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (torch.log(total) + base).view(B, Hq, T)
    return o.permute(0, 3, 1, 2, 4).reshape(B, T, Hq, d), lse


def _stored(st, o, lse):
    """The results where a sample has tokens; rows behind them as they were."""
    if st["count"] is not None:
        live = torch.arange(o.shape[1], device="cuda") < st["count"][:, None]
        o = torch.where(live[:, :, None, None], o.bfloat16(), st["out"][0])
        lse = torch.where(live[:, None], lse, st["out"][1])
    return {"out": o.bfloat16(), "lse": lse}


def _run_window(st):
    B, T = st["q"].shape[:2]
    starts = st["starts"] if st["starts"] is not None else torch.full((B,), st["start"], device="cuda")
    at = (starts[:, None] + torch.arange(T, device="cuda"))[:, :, None]                     # the row of each token
    key = torch.arange(st["k_cache"].shape[1], device="cuda")
    seen = key <= at
    if st["window"]:
        seen = seen & ((key > at - st["window"]) | (key < st["sinks"]))
    return _stored(st, *_attend(st["q"], st["k_cache"], st["v_cache"], seen))


def _run_tree(st):
    B, T = st["q"].shape[:2]
    n = st["start"]
    starts = st["starts"] if st["starts"] is not None else torch.full((B,), n, device="cuda")
    in_cache = (torch.arange(n, device="cuda") < starts[:, None])[:, None].expand(B, T, n)
    drafted = (st["tree"][:, :, None] >> torch.arange(T, device="cuda")) & 1 == 1           # [B,T,T]
    if st["count"] is not None:
        drafted = drafted & (torch.arange(T, device="cuda") < st["count"][:, None])[:, None]
    k = torch.cat([st["k_cache"][:, :n], st["k"]], 1)
    v = torch.cat([st["v_cache"][:, :n], st["v"]], 1)
    return _stored(st, *_attend(st["q"], k, v, torch.cat([in_cache, drafted], -1)))


def _run_append(st):
    L, B, _, Hkv, d = st["k"].shape
    R = st["path"].shape[1]
    i = torch.arange(R, device="cuda")
    live = (i < st["count"][:, None]).expand(L, B, R)
    layer = torch.arange(L, device="cuda")[:, None, None].expand(L, B, R)[live]
    sample = torch.arange(B, device="cuda")[:, None].expand(L, B, R)[live]
    at = (st["starts"][:, :, None].long() + i)[live]
    src = st["path"].long().expand(L, B, R)[live]
    st["k_cache"][layer, sample, at] = st["k"][layer, sample, src]
    st["v_cache"][layer, sample, at] = st["v"][layer, sample, src]
    return {"k": st["k_cache"], "v": st["v_cache"]}


def run(st):
    op = st["op"]
    if own:
        from paper_2601_17818_amd import binding as vc
        if op == "append":
            vc.vitcop_cache_append(st["k_cache"], st["v_cache"], st["k"], st["v"], start_samples=st["starts"],
                                   idx=st["path"], n_samples=st["count"])
            return {"k": st["k_cache"], "v": st["v_cache"]}
        cache = vc.Cache(st["k_cache"], st["v_cache"])
        if op == "rope":
            q, _ = vc.vitcop_rope_axes(st["q"], st["k"], st["positions"], st["sections"], st["theta"], v=st["v"],
                                       interleaved=st["interleaved"], cache=cache, start_samples=st["start"],
                                       n_samples=st["count"], out=st["out"])
            return {"q": q, "k": st["k_cache"], "v": st["v_cache"]}
        if op == "window":
            out, lse = vc.vitcop_window_attn(st["q"], cache, st["start"], window=st["window"], sinks=st["sinks"],
                                             start_samples=st["starts"], n_samples=st["count"], out=st["out"])
        else:
            out, lse = vc.vitcop_tree_attn(st["q"], st["k"], st["v"], st["tree"], cache, st["start"],
                                           start_samples=st["starts"], n_samples=st["count"], out=st["out"])
        return {"out": out, "lse": lse}
    if op == "rope":
        return _run_rope(st)
    if op == "append":
        return _run_append(st)
    return _run_window(st) if op == "window" else _run_tree(st)


# -------------------------------------------------------------------------------------------------- what a pass costs


def _pairs_seen(start, n, window, sinks):
    """(keys that n tokens at rows start.. see, together; rows that at least one of them sees)."""
    if n == 0:
        return 0, 0
    if not window:
        return n * start + n * (n + 1) // 2, start + n
    first = max(0, start + 1 - window)
    pairs = sum(min(p + 1, window) + min(sinks, max(0, p + 1 - window)) for p in range(start, start + n))
    return pairs, start + n - first + min(sinks, first)


def work(case):
    op = case["op"]
    Hq, Hkv, d = HEADS[case["model"]]
    B, T = case["B"], case["T"]
    if op == "rope":
        tokens = sum(_lengths(case, T))
        return {"bytes": tokens * (4 * (Hq + 2 * Hkv) * d + 12), "flops": 3 * tokens * (Hq + Hkv) * d}
    if op == "append":
        rows = case["layers"] * sum(_accepted(case))
        return {"bytes": 8 * rows * Hkv * d, "flops": 0}
    pairs = rows = 0
    for start, n in zip(_starts(case), _lengths(case, T)):
        if op == "window":
            p, r = _pairs_seen(start, n, case["window"], case["sinks"])
        else:
            p, r = n * (start + min(n, 5)), (start + n if n else 0)
        pairs, rows = pairs + p, rows + r
    tokens = sum(_lengths(case, T))
    return {"bytes": 4 * rows * Hkv * d + 4 * tokens * Hq * (d + 1), "flops": 4 * pairs * Hq * d}


# ---------------------------------------------------------------------------------------------------- in 64 bits


def _head64(q, k, v, seen):
    """q [G,n,d], k, v [N,d], seen [n,N] -> out [n,G,d], lse [G,n]."""
    s = torch.einsum("gnd,kd->gnk", q.double(), k.double()) / math.sqrt(q.shape[-1])
    s.masked_fill_(~seen, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[..., None])
    return torch.einsum("gnk,kd->ngd", p, v.double()), lse


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    B, T = case["B"], case["T"]
    Hq, Hkv, d = HEADS[case["model"]]
    if op == "append":
        out = {"k": st["k_cache"].double(), "v": st["v_cache"].double()}
        count, path, starts = st["count"].tolist(), st["path"].tolist(), st["starts"].tolist()
        for layer in range(case["layers"]):
            for b in range(B):
                to, src = slice(starts[layer][b], starts[layer][b] + count[b]), path[b][:count[b]]
                out["k"][layer, b, to] = st["k"][layer, b, src].double()
                out["v"][layer, b, to] = st["v"][layer, b, src].double()
        return out
    lens = _lengths(case, T)
    if op == "rope":
        pairs = SECTIONS[d]
        if case["interleaved"]:                      # sorted by the turn in which an axis gives its j-th pair
            axis = [a for _, a in sorted((j, a) for a, n in enumerate(pairs) for j in range(n))]
        else:
            axis = sorted(a for a, n in enumerate(pairs) for _ in range(n))
        speed = torch.tensor([math.exp(-math.log(st["theta"]) * 2 * i / d) for i in range(d // 2)], dtype=torch.float64,
                             device="cuda")
        out = {"q": st["out"].double(), "k": st["k_cache"].double(), "v": st["v_cache"].double()}
        for b in range(B):
            n, first = lens[b], int(st["start"][b])
            turn = st["positions"][axis, b, :n].double().T * speed
            unit = torch.polar(torch.ones_like(turn), turn)[:, None]
            for name, to in (("q", out["q"][b, :n]), ("k", out["k"][b, first:first + n])):
                x = st[name][b, :n].double()
                z = torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * unit
                to[:] = torch.cat([z.real, z.imag], -1)
            out["v"][b, first:first + n] = st["v"][b, :n].double()
        return out
    out, lse = st["out"][0].double(), st["out"][1].double()
    for b, (n, start) in enumerate(zip(lens, _starts(case))):
        if n == 0:
            continue
        row = torch.arange(start, start + n, device="cuda")[:, None]
        if op == "window":
            k, v = st["k_cache"][b, :start + n], st["v_cache"][b, :start + n]
            key = torch.arange(start + n, device="cuda")
            back = row - key
            near = back < (case["window"] or start + n + 1)
            seen = (back >= 0) & (near | (key < case["sinks"]))
        else:
            k = torch.cat([st["k_cache"][b, :start], st["k"][b, :n]])
            v = torch.cat([st["v_cache"][b, :start], st["v"][b, :n]])
            seen = torch.ones((n, start + n), dtype=torch.bool)
            for t, mask in enumerate(st["tree"][b, :n].tolist()):
                for j in range(n):
                    seen[t, start + j] = bool((mask >> j) & 1)
            seen = seen.to("cuda")
        for h in range(Hkv):
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            o, e = _head64(st["q"][b, :n, heads].transpose(0, 1), k[:, h], v[:, h], seen)
            out[b, :n, heads] = o
            lse[b, heads, :n] = e
    return {"out": out, "lse": lse}
