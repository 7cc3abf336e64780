"""vitcop_window_attn and vitcop_tree_attn against float64 over explicit masks.

Bounds. A score's fp32 sum of d products and its scaling are off by at most e = (d + 4) 2^-24 of the sum of |q k| scale; a
probability then by e twice over (its own and its sum's) and by 2^-21 of the exponential and its argument; the sums over n keys
by n 2^-24. A probability goes into the product with V in 24 bits (half a step of the third eight: 2^-24), in calls of more than
16 query rows to a KV head in 16 (2^-16), of more than 32 in eight (2^-8). The output is rounded to bf16: 2^-8 of it. lse: e, the sum's n 2^-24, 2^-21 and 2^-22 of its own size.
"""
import math

import numpy as np
import pytest
import torch

import vitcop_inputs as I
from gpu_util import dev, host_f64
from oracle import span_oracle as S
from oracle import vitcop_oracle as O

pytestmark = pytest.mark.gpu



@pytest.fixture(scope="module")
def vc():
    from paper_2601_17818_amd import binding
    return binding


def bits(rng, shape, std=1.0):
    return I.f32_to_bf16_bits((rng.standard_normal(shape) * std).astype(np.float32))


def check(got, lse, want, rows, where):
    """got [n,Hq,d], lse [Hq,n] of one sample's tokens."""
    d = got.shape[-1]
    keys = want["keys"]
    e = (d + 4) * 2.0 ** -24 * want["reach"]
    p = 2.0 ** -24 if rows <= 16 else 2.0 ** -16 if rows <= 32 else 2.0 ** -8
    bound = 2.0 ** -8 * np.abs(want["out"]) + (p + 2 * e[..., None] + 2.0 ** -21 + keys * 2.0 ** -24) * want["mass"] * 1.01
    err = np.abs(got - want["out"])
    assert (err <= bound).all(), f"{where}: {np.max(err - bound)} over the bound {bound.flat[np.argmax(err - bound)]}"
    if lse is None:
        return
    empty = np.isneginf(want["lse"])
    assert np.array_equal(np.isneginf(lse), empty), where
    assert (got[empty.T] == 0).all(), where
    tol = (1.01 * e.T + 2.0 ** -21 + keys * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(empty, 0, want["lse"])))[~empty]
    assert (np.abs(lse[~empty] - want["lse"][~empty]) <= tol).all(), where


class Case:
    """One layer's cache and the tokens of a call; what no token sees is NaN, outputs hold a mark before the call."""

    def __init__(self, vc, seed, B, T, start, Hq, Hkv, d, starts=None, counts=None, spare=3, q_std=1.5, fused=False):
        rng = self.rng = np.random.default_rng(seed)
        self.vc, self.B, self.T, self.start, self.Hq, self.Hkv, self.d = vc, B, T, start, Hq, Hkv, d
        self.capacity = start + T + spare
        self.k, self.v = bits(rng, (B, self.capacity, Hkv, d)), bits(rng, (B, self.capacity, Hkv, d))
        self.qd = dev(bits(rng, (B, T, Hq, d), q_std))
        if fused:                                        # in fused QKV rows, samples further apart than their tokens
            wide = torch.full((B, T + 2, (Hq + 2 * Hkv) * d), float("nan"), dtype=torch.bfloat16, device="cuda")
            view = wide[:, :T, :Hq * d].unflatten(-1, (Hq, d))
            view.copy_(self.qd)
            self.qd = view
        self.q = host_f64(self.qd)
        self.starts = list(starts) if starts is not None else [start] * B
        self.counts = list(counts) if counts is not None else [T] * B
        as_ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda") if x is not None else None  # noqa: E731
        self.starts_d, self.counts_d = as_ints(starts), as_ints(counts)
        self.out = (torch.full((B, T, Hq, d), 7.5, dtype=torch.bfloat16, device="cuda"),
                    torch.full((B, Hq, T), 7.5, device="cuda"))

    def cache(self, seen):
        """seen: per sample, the rows that a token sees."""
        k, v = self.k.copy(), self.v.copy()
        for b in range(self.B):
            hidden = np.setdiff1d(np.arange(self.capacity), seen[b])
            k[b, hidden], v[b, hidden] = 0x7FC0, 0x7F80      # NaN and infinity
        return self.vc.Cache(dev(k), dev(v))

    def n(self, b):
        return min(max(self.counts[b], 0), self.T)

    def held(self, b):
        return min(max(self.starts[b], 0), self.start)

    def compare(self, out, lse, sample):
        got, glse = host_f64(out), host_f64(lse)
        for b in range(self.B):
            n = self.n(b)
            assert (got[b, n:] == 7.5).all() and (glse[b, :, n:] == 7.5).all(), f"sample {b}: rows behind its tokens"
            if n:
                k, v, sees, scale = sample(b, n)
                want = S.attend(self.q[b, :n], k, v, sees, scale)
                want["keys"] = sees.shape[1]
                check(got[b, :n], glse[b, :, :n], want, self.T * self.Hq // self.Hkv, f"sample {b}")

    def window(self, window, sinks, scale=0.0, **kw):
        rows = [self.held(b) + self.n(b) for b in range(self.B)]
        sees = [S.window_sees(self.held(b), self.n(b), rows[b], window, sinks) for b in range(self.B)]
        seen = [np.flatnonzero(s.any(0)) if len(s) else [] for s in sees]
        out, lse = self.vc.vitcop_window_attn(self.qd, self.cache(seen), self.start, window, sinks, self.starts_d, self.counts_d,
                                              scale, out=self.out, **kw)
        f64 = O.bf16_to_f64
        self.compare(out, lse, lambda b, n: (f64(self.k[b, :rows[b]]), f64(self.v[b, :rows[b]]), sees[b], scale))
        return out, lse

    def tree(self, masks, scale=0.0, fused=False, **kw):
        """masks: [B][T] whole numbers, or [T] for all samples."""
        shared = not isinstance(masks[0], (list, tuple, np.ndarray))
        per_sample = [masks] * self.B if shared else masks
        signed = [[m - 2 ** 64 if m >= 2 ** 63 else m for m in row] for row in per_sample]
        k2, v2 = bits(self.rng, (self.B, self.T, self.Hkv, self.d)), bits(self.rng, (self.B, self.T, self.Hkv, self.d))
        kd, vd = k2.copy(), v2.copy()
        sees = []
        for b in range(self.B):
            n = self.n(b)
            s = S.tree_sees(self.held(b), n, [m & (2 ** 64 - 1) for m in per_sample[b]])
            sees.append(s)
            hidden = np.setdiff1d(np.arange(self.T), np.flatnonzero(s[:, self.held(b):].any(0)))
            kd[b, hidden], vd[b, hidden] = 0xFF80, 0x7FC0
        kd, vd = dev(kd), dev(vd)
        if fused:                                        # v in fused rows, k dense, as the rotary embedding leaves them
            wide = torch.full((self.B, self.T, 3 * self.Hkv * self.d), float("nan"), dtype=torch.bfloat16, device="cuda")
            view = wide[:, :, self.Hkv * self.d:2 * self.Hkv * self.d].unflatten(-1, (self.Hkv, self.d))
            view.copy_(vd)
            vd = view
        tree = torch.tensor(signed[0] if shared else signed, dtype=torch.int64, device="cuda")
        seen = [np.arange(self.held(b) if self.n(b) else 0) for b in range(self.B)]
        out, lse = self.vc.vitcop_tree_attn(self.qd, kd, vd, tree, self.cache(seen), self.start, self.starts_d, self.counts_d,
                                            scale, out=self.out, **kw)
        f64 = O.bf16_to_f64

        def sample(b, n):
            at = self.held(b)
            return (np.concatenate([f64(self.k[b, :at]), f64(k2[b, :n])]), np.concatenate([f64(self.v[b, :at]), f64(v2[b, :n])]),
                    sees[b], scale)

        self.compare(out, lse, sample)
        return out, lse


def trees(rng, B, T):
    """Random trees: a token sees itself and its ancestors."""
    out = []
    for _ in range(B):
        masks = []
        for t in range(T):
            parent = int(rng.integers(-1, t)) if t else -1
            masks.append((1 << t) | (masks[parent] if parent >= 0 else 0))
        out.append(masks)
    return out


WINDOWS = [
    # B, T, start, Hq, Hkv, d, window, sinks
    (1, 1, 0, 1, 1, 128, 0, 0), (1, 1, 0, 4, 4, 64, 1, 1), (2, 1, 31, 4, 2, 128, 0, 0), (1, 1, 32, 28, 4, 128, 33, 1),
    (3, 1, 100, 16, 4, 64, 32, 5), (1, 1, 500, 17, 1, 128, 64, 33), (1, 1, 700, 24, 1, 64, 0, 0), (2, 1, 2500, 8, 8, 128, 0, 0),
    (2, 1, 2500, 8, 2, 64, 1000, 4), (1, 2, 3, 2, 1, 128, 1, 0), (2, 5, 40, 28, 4, 128, 31, 0), (1, 15, 17, 1, 1, 64, 8, 2),
    (1, 16, 0, 2, 2, 128, 0, 0), (1, 17, 250, 14, 2, 128, 100, 300), (1, 33, 1, 4, 1, 64, 33, 32), (2, 63, 65, 3, 3, 128, 0, 7),
    (1, 64, 64, 4, 4, 128, 64, 64), (1, 65, 1200, 4, 1, 128, 500, 3), (1, 127, 0, 2, 1, 128, 0, 0), (2, 128, 0, 2, 2, 64, 32, 0),
    (1, 129, 33, 4, 2, 128, 65, 1), (1, 200, 0, 3, 1, 128, 1, 0), (1, 257, 100, 2, 2, 128, 64, 16), (1, 300, 700, 2, 1, 64, 0, 0),
    # (two blocks of 128 query rows a workgroup)
    (2, 700, 0, 28, 4, 128, 100, 5), (3, 700, 130, 16, 8, 128, 0, 0), (2, 600, 0, 32, 16, 128, 64, 16), (5, 500, 60, 16, 8, 128, 90, 3),
    (2, 700, 33, 28, 4, 128, 60, 200), (2, 650, 0, 28, 4, 128, 1, 0),
    (1, 513, 0, 2, 1, 128, 130, 65), (1, 600, 50, 1, 1, 64, 200, 40), (1, 640, 0, 2, 2, 128, 0, 0), (2, 384, 0, 7, 1, 128, 100, 129),
]


@pytest.mark.parametrize("B,T,start,Hq,Hkv,d,window,sinks", WINDOWS)
def test_window(vc, B, T, start, Hq, Hkv, d, window, sinks):
    Case(vc, 1, B, T, start, Hq, Hkv, d).window(window, sinks)


@pytest.mark.parametrize("B,T,start,Hq,Hkv,d,window,sinks", [
    (5, 1, 300, 8, 2, 128, 64, 4), (5, 1, 300, 2, 2, 64, 0, 0), (6, 9, 130, 28, 4, 128, 33, 2), (4, 70, 50, 4, 1, 64, 0, 0),
    (4, 150, 0, 4, 2, 128, 40, 3), (4, 300, 20, 2, 2, 128, 0, 0), (4, 300, 20, 2, 1, 64, 100, 70), (3, 530, 0, 2, 1, 128, 70, 1), (5, 500, 60, 16, 8, 128, 90, 3), (4, 900, 100, 28, 4, 128, 0, 0),
    (70, 1, 40, 2, 2, 64, 0, 0), (130, 3, 20, 4, 2, 128, 7, 1), (67, 20, 9, 4, 2, 64, 0, 0)])
def test_samples_of_their_own_lengths(vc, B, T, start, Hq, Hkv, d, window, sinks):
    rng = np.random.default_rng(5)
    starts = rng.integers(0, start + 1, B).tolist()
    counts = rng.integers(1, T + 1, B).tolist()
    starts[0], counts[0], starts[1], counts[2] = start, T, 0, 0
    Case(vc, 2, B, T, start, Hq, Hkv, d, starts, counts).window(window, sinks)


def test_lengths_past_the_ends_are_clamped(vc):
    Case(vc, 3, 4, 6, 40, 4, 2, 128, starts=[41, -5, 2 ** 31 - 1, 40], counts=[7, 2 ** 31 - 1, -1, -2 ** 31]).window(16, 2)
    Case(vc, 3, 3, 6, 40, 4, 2, 64, starts=[99, -1, -2 ** 31], counts=[99, -9, 3]).tree(trees(np.random.default_rng(1), 3, 6))


@pytest.mark.parametrize("T,start", [(1, 90), (7, 90), (300, 90)])
def test_queries_in_fused_rows(vc, T, start):
    Case(vc, 4, 2, T, start, 4, 2, 128, fused=True).window(50, 2)


@pytest.mark.parametrize("T", [1, 200])
@pytest.mark.parametrize("scale,std", [(0.02, 1.0), (1.0, 3.0)])
def test_scales(vc, T, scale, std):
    Case(vc, 5, 1, T, 200, 2, 1, 128, q_std=std).window(90, 3, scale)


def test_windows_and_sinks_past_the_cache(vc):
    for window, sinks in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (5, 2 ** 31 - 1)):
        Case(vc, 6, 1, 9, 70, 2, 2, 128).window(window, sinks)
        Case(vc, 6, 1, 300, 0, 2, 2, 128).window(window, sinks)


TREES = [                                                # (of more than 64 query rows, too)
    (1, 9, 200, 8, 1, 128), (2, 20, 63, 14, 2, 64), (2, 20, 63, 2, 2, 64), (2, 5, 300, 16, 4, 64), (1, 64, 1000, 4, 2, 128), (2, 33, 0, 4, 1, 128), (1, 40, 2100, 28, 4, 64),
    # B, T, start, Hq, Hkv, d
    (1, 1, 0, 1, 1, 128), (1, 1, 33, 4, 4, 64), (2, 8, 384, 4, 4, 128), (1, 16, 31, 28, 4, 128), (1, 17, 32, 16, 4, 64),
    (2, 25, 500, 3, 3, 128), (1, 31, 2000, 2, 2, 128), (1, 32, 64, 4, 1, 128), (1, 33, 1000, 8, 1, 64), (1, 63, 5, 2, 1, 128),
    (2, 64, 300, 7, 1, 128), (1, 64, 0, 16, 4, 64)]


@pytest.mark.parametrize("B,T,start,Hq,Hkv,d", TREES)
def test_tree(vc, B, T, start, Hq, Hkv, d):
    Case(vc, 7, B, T, start, Hq, Hkv, d).tree(trees(np.random.default_rng(T), B, T))


def test_trees_of_their_own_lengths(vc):
    for d in (64, 128):
        for Hq in (2, 6, 16):
            c = Case(vc, 8, 5, 40, 130, Hq, 2, d, starts=[130, 0, 77, 1, 129], counts=[40, 39, 0, 1, 33])
            c.tree(trees(np.random.default_rng(9), 5, 40), fused=True)


def test_any_masks(vc):
    rng = np.random.default_rng(10)
    every = [2 ** 64 - 1] * 48                                       # bits past the drafts are not looked at
    Case(vc, 9, 2, 48, 0, 2, 1, 128).tree(every)
    some = [[int(x) for x in rng.integers(0, 2 ** 48, 48, dtype=np.uint64)] for _ in range(2)]
    some[0][:3], some[1][47] = [0, 1 << 47, 0], 0                    # nothing, one later draft alone
    Case(vc, 9, 2, 48, 0, 2, 1, 128).tree(some)
    Case(vc, 9, 2, 48, 37, 2, 1, 64).tree(some)
    Case(vc, 9, 2, 48, 1500, 4, 1, 128).tree(some)
    Case(vc, 9, 1, 64, 0, 2, 2, 64).tree([0] * 63 + [1 << 63])
    Case(vc, 9, 2, 64, 0, 4, 2, 64).tree([0] * 63 + [1 << 63])       # all but one see nothing


def test_a_tree_for_all_samples(vc):
    Case(vc, 10, 3, 12, 50, 4, 2, 128).tree(trees(np.random.default_rng(2), 1, 12)[0])


def test_a_chain_of_drafts_is_a_question(vc):
    """Drafts that see all drafts before them are tokens behind the cache: both calls, and each token by itself."""
    B, T, n, Hq, Hkv, d = 2, 9, 140, 8, 2, 128
    rng = np.random.default_rng(3)
    k, v, q = (dev(bits(rng, (B, n + T, h, d))) for h in (Hkv, Hkv, Hq))
    cache, q = vc.Cache(k, v), q[:, :T].contiguous()
    tree = torch.tensor([2 ** (t + 1) - 1 for t in range(T)], device="cuda")
    a, la = vc.vitcop_tree_attn(q, k[:, n:], v[:, n:], tree, cache, n)
    b, lb = vc.vitcop_window_attn(q, cache, n)
    # two results of half a bf16 step each, of sums in another order
    assert (a.float() - b.float()).abs().max() <= 2.0 ** -7 * a.float().abs().max() and (la - lb).abs().max() < 1e-5
    for t in range(T):
        c, lc = vc.vitcop_window_attn(q[:, t:t + 1], cache, n + t)
        assert (c[:, 0].float() - b[:, t].float()).abs().max() <= 2.0 ** -7 * b.float().abs().max()
        assert (lc[..., 0] - lb[..., t]).abs().max() < 1e-5


def test_the_same_as_the_framework_s_other_attentions(vc):
    rng = np.random.default_rng(4)
    q, k, v = (dev(bits(rng, (2, 300, h, 128))) for h in (8, 2, 2))
    cache = vc.Cache(k, v)
    out, lse = vc.vitcop_window_attn(q, cache, 0)
    ref, rlse = vc.vitcop_prefill_attn(q, k, v, want_lse=True)
    assert (out.float() - ref.float()).abs().max() <= 2e-2 and (lse - rlse).abs().max() < 1e-4
    out, lse = vc.vitcop_window_attn(q[:, 299:], cache, 299)
    ref, rlse = vc.vitcop_decode_attn(q[:, 299].contiguous(), k, v)[:2]
    assert (out[:, 0].float() - ref.float()).abs().max() <= 2.0 ** -7 * ref.float().abs().max()
    assert (lse[..., 0] - rlse).abs().max() < 1e-5


def test_rows_past_32_bits_of_a_cache(vc):
    """One sample's rows span more than 2^32 bytes: 40000 of 128 KB."""
    Hkv, d, n = 512, 128, 40000
    k = torch.zeros((1, n, Hkv, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    rng = np.random.default_rng(6)
    at = n - 40
    kb, vb, qb = (bits(rng, (40, Hkv, d)) for _ in range(3))
    k[0, at:], v[0, at:] = dev(kb), dev(vb)
    cache = vc.Cache(k, v)
    heads = [0, 1, 255, 511]
    f64 = O.bf16_to_f64
    q = dev(qb[:3])[None]
    for T in (1, 3):
        out, lse = vc.vitcop_window_attn(q[:, :T], cache, n - T, window=30)
        start = 40 - T
        want = S.attend(f64(qb[:T, heads]), f64(kb[:, heads]), f64(vb[:, heads]), S.window_sees(start, T, 40, 30, 0))
        want["keys"] = 40
        check(host_f64(out)[0][:, heads], host_f64(lse)[0][heads], want, T, f"T={T}")
    sinks = vc.vitcop_window_attn(q[:, :1], cache, n - 1, window=5, sinks=2)[0]      # zeros among the keys: it differs
    assert torch.isfinite(sinks).all()
    out, _ = vc.vitcop_tree_attn(q[:, :2], cache.k[:, at:at + 2].contiguous(), cache.v[:, at:at + 2].contiguous(),
                                 torch.tensor([1, 3], device="cuda"), cache, n)
    total = np.concatenate([np.zeros((n - 40, len(heads), d)), f64(kb[:, heads]), f64(kb[:2, heads])])
    vals = np.concatenate([np.zeros((n - 40, len(heads), d)), f64(vb[:, heads]), f64(vb[:2, heads])])
    want = S.attend(f64(qb[:2, heads]), total, vals, S.tree_sees(n, 2, [1, 3]))
    want["keys"] = n + 2
    check(host_f64(out)[0][:, heads], None, want, 2, "tree")


def test_another_stream_and_a_graph(vc):
    """Captured calls go by what the device arrays hold at the replay, each graph with a workspace of its own."""
    B, T, n, Hq, Hkv, d = 3, 4, 900, 8, 2, 128
    rng = np.random.default_rng(7)
    k, v = (dev(bits(rng, (B, n + T, Hkv, d))) for _ in range(2))
    q, dk, dv = (dev(bits(rng, (B, T, h, d))) for h in (Hq, Hkv, Hkv))
    starts, counts = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    tree = torch.tensor([1, 3, 5, 9], device="cuda")
    cache = vc.Cache(k, v)

    def calls(out):
        return [vc.vitcop_window_attn(q, cache, n, 300, 4, starts, counts, out=out[0]),
                vc.vitcop_tree_attn(q, dk, dv, tree, cache, n, starts, counts, out=out[1])]

    def fresh():
        return [(torch.zeros((B, T, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((B, Hq, T), device="cuda"))
                for _ in range(2)]

    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        out = fresh()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            calls(out)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            calls(out)
        graphs.append((g, out))
    for s, c in (([900, 1, 450], [4, 4, 1]), ([0, 899, 300], [1, 0, 4]), ([900, 900, 900], [4, 4, 4])):
        starts.copy_(torch.tensor(s, dtype=torch.int32))
        counts.copy_(torch.tensor(c, dtype=torch.int32))
        for g, out in graphs:
            for o, e in out:
                o.zero_()
                e.zero_()
            g.replay()
        want = calls(fresh())
        torch.cuda.synchronize()
        for _, out in graphs:
            for (o, e), (wo, we) in zip(out, want):
                assert torch.equal(o, wo) and torch.equal(e, we)


def test_many_rows_on_two_streams_at_once_and_in_a_graph(vc):
    """Questions of many rows: two streams at once, each with its own workspace, and replays that go by the lengths."""
    B, T, n, Hq, Hkv, d = 3, 150, 700, 8, 2, 128
    rng = np.random.default_rng(13)
    k, v = (dev(bits(rng, (B, n + T, Hkv, d))) for _ in range(2))
    q = dev(bits(rng, (B, T, Hq, d)))
    starts, counts = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    cache = vc.Cache(k, v)

    def fresh():
        return torch.zeros((B, T, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((B, Hq, T), device="cuda")

    def call(window, out):
        return vc.vitcop_window_attn(q, cache, n, window, 4, starts, counts, out=out)

    starts.copy_(torch.tensor([700, 20, 333], dtype=torch.int32))
    counts.copy_(torch.tensor([150, 1, 70], dtype=torch.int32))
    want = [call(w, fresh()) for w in (0, 90)]
    outs = [[fresh() for _ in range(4)] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(4):
        for j, side in enumerate(streams):
            with torch.cuda.stream(side):
                call((0, 90)[j], outs[j][i])
    torch.cuda.synchronize()
    for j in range(2):
        for o, e in outs[j]:
            assert torch.equal(o, want[j][0]) and torch.equal(e, want[j][1])
    out = fresh()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(90, out)
    for s, c in (([700, 0, 5], [150, 150, 0]), ([0, 699, 350], [149, 2, 128]), ([700, 700, 700], [1, 150, 33])):
        starts.copy_(torch.tensor(s, dtype=torch.int32))
        counts.copy_(torch.tensor(c, dtype=torch.int32))
        for t in out:
            t.zero_()
        g.replay()
        o, e = call(90, fresh())
        torch.cuda.synchronize()
        assert torch.equal(out[0], o) and torch.equal(out[1], e)


def test_calls_repeat_bit_for_bit(vc):
    c = Case(vc, 11, 2, 20, 1500, 8, 2, 128)
    a = [t.clone() for t in c.window(0, 0)]
    b = c.window(0, 0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_without_lse_and_with_a_workspace(vc):
    c = Case(vc, 12, 1, 1, 2000, 4, 4, 128)
    cache = vc.Cache(dev(c.k), dev(c.v))
    need = vc.lib.vitcop_window_attn_workspace_bytes(1, 1, 2000, 4, 4, 128, 0, 0)
    assert need > 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    out, lse = vc.vitcop_window_attn(c.qd, cache, 2000, want_lse=False, ws=ws)
    assert lse is None and torch.equal(out, vc.vitcop_window_attn(c.qd, cache, 2000)[0])
    with pytest.raises(vc.VitcopError):
        vc.vitcop_window_attn(c.qd, cache, 2000, ws=ws[:need - 256])


def test_no_tokens(vc):
    cache = vc.Cache(*[torch.zeros((2, 8, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)])
    q = torch.zeros((2, 0, 4, 64), dtype=torch.bfloat16, device="cuda")
    out, lse = vc.vitcop_window_attn(q, cache, 3)
    assert out.shape == (2, 0, 4, 64) and lse.shape == (2, 4, 0)
    assert math.prod(vc.vitcop_tree_attn(q, q[:, :, :2], q[:, :, :2], torch.zeros((2, 0), dtype=torch.int64, device="cuda"),
                                         cache, 3)[0].shape) == 0


def test_refusals_of_the_binding(vc):
    B, T, Hq, Hkv, d = 2, 3, 4, 2, 64
    k = torch.zeros((B, 9, Hkv, d), dtype=torch.bfloat16, device="cuda")
    cache = vc.Cache(k, k.clone())
    q, dk = (torch.zeros((B, T, h, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv))
    tree = torch.zeros((B, T), dtype=torch.int64, device="cuda")
    counts = torch.zeros(B, dtype=torch.int32, device="cuda")
    for bad in (q.cpu(), q[:1], q.float(), q[..., :32], q[:, :, ::2], q[0], q.transpose(1, 2)):
        with pytest.raises((ValueError, vc.VitcopError)):
            vc.vitcop_window_attn(bad, cache, 0)
        with pytest.raises((ValueError, vc.VitcopError)):
            vc.vitcop_tree_attn(bad, dk, dk, tree, cache, 0)
    for kw in (dict(start=2 ** 31), dict(start=7), dict(start=-1), dict(start=0, window=-1), dict(start=0, sinks=2 ** 40),
               dict(start=0, start_samples=counts.long()), dict(start=0, n_samples=counts[:1]), dict(start=0, n_samples=counts.cpu()),
               dict(start=0, scale=float("nan")), dict(start=0, out=(q.float(), None)), dict(start=0, ws=counts)):
        with pytest.raises((ValueError, vc.VitcopError)):
            vc.vitcop_window_attn(q, cache, **kw)
    for bad in (dict(k=dk[:, :2]), dict(v=dk.half()), dict(tree=tree.int()), dict(tree=tree[:, :2]), dict(tree=tree.t()),
                dict(start=10), dict(k=dk.expand(B, T, Hkv, d)[:, :1].expand(B, T, Hkv, d))):
        with pytest.raises((ValueError, vc.VitcopError)):
            vc.vitcop_tree_attn(**dict(dict(q=q, k=dk, v=dk, tree=tree, cache=cache, start=0), **bad))
    for make in (lambda: vc.Cache(k, k[:, :8]), lambda: vc.Cache(k.cpu(), k.cpu()), lambda: vc.Cache(k[:, ::2], k[:, ::2]),
                 lambda: vc.Cache(k[0], k[0]), lambda: vc.Cache(k, k.float())):
        with pytest.raises(ValueError):
            make()
    with pytest.raises(AttributeError):
        cache.k = k
