"""vitcop_window_attn and vitcop_tree_attn where offsets pass 31 and 32 bits.  Bounds as in test_gpu_span_attn.py."""
import numpy as np
import pytest
import torch

from gpu_util import dev, host_f64
from oracle import span_oracle as S
from oracle import vitcop_oracle as O
from test_gpu_span_attn import bits, trees, vc  # noqa: F401

pytestmark = pytest.mark.gpu

PERIOD = 1031                      # query heads repeat after so many: one that is read in another's place is seen


def bounds(want, d, keys):
    """Of outputs [n,Hq,d] and of lse [n,Hq], where more than 32 query rows read a KV head."""
    e = (d + 4) * 2.0 ** -24 * want["reach"]
    out = 2.0 ** -8 * np.abs(want["out"]) + (2.0 ** -8 + 2 * e[..., None] + 2.0 ** -21 + keys * 2.0 ** -24) * want["mass"] * 1.01
    return out, 1.01 * e + 2.0 ** -21 + keys * 2.0 ** -24 + 2.0 ** -22 * np.abs(want["lse"].T)


def assert_heads(out, lse, q, k, v, keys):
    """out [Hkv,G,d] and lse [Hkv,G] of one token, head g of each being q[g % PERIOD], over k, v [keys,Hkv,d]."""
    f64 = O.bf16_to_f64
    Hkv, G, d = out.shape
    for hk in sorted({0, 1, Hkv - 1} & set(range(Hkv))):
        want = S.attend(f64(q)[None], f64(k[:, hk:hk + 1]), f64(v[:, hk:hk + 1]), np.ones((1, keys), bool))
        ob, lb = (torch.from_numpy(x[0]).cuda() for x in bounds(want, d, keys))
        wo, wl = torch.from_numpy(want["out"][0]).cuda(), torch.from_numpy(want["lse"][:, 0]).cuda()
        for first in range(0, G, 256 * PERIOD):
            n = min(256 * PERIOD, G - first)
            at = torch.arange(n, device="cuda") % PERIOD
            assert bool(((out[hk, first:first + n].double() - wo[at]).abs() <= ob[at]).all()), (hk, first)
            assert bool(((lse[hk, first:first + n].double() - wl[at]).abs() <= lb[at]).all()), (hk, first)


def heads(q, n):
    tile = dev(q)
    return tile.repeat((n + PERIOD - 1) // PERIOD, 1)[:n]


def test_query_heads_past_31_bits(vc):  # noqa: F811
    """A token of more than 2^24 query heads of 128 channels: a head's offset in its row passes 2^31."""
    d, n, G = 128, 70, (1 << 24) + 200
    rng = np.random.default_rng(1)
    q, k, v = bits(rng, (PERIOD, d)), bits(rng, (n + 1, 1, d)), bits(rng, (n + 1, 1, d))
    qd = heads(q, G).view(1, 1, G, d)
    cache = vc.Cache(dev(k)[None], dev(v)[None])
    out, lse = vc.vitcop_window_attn(qd, cache, n)
    assert_heads(out.view(1, G, d), lse.view(1, G), q, k, v, n + 1)
    out.fill_(7.5)
    k2, v2 = (dev(x[n:]).view(1, 1, 1, d) for x in (k, v))
    vc.vitcop_tree_attn(qd, k2, v2, torch.ones((1, 1), dtype=torch.int64, device="cuda"), cache, n, out=(out, lse))
    assert_heads(out.view(1, G, d), lse.view(1, G), q, k, v, n + 1)


def test_query_heads_past_31_bits_over_4_gib_of_cache(vc):  # noqa: F811
    """The same where the cache's rows leave the kernel of many query rows out; few of the rows are there."""
    d, n, Hkv, G, start = 128, 70, 16, (1 << 20) + 40, 1 << 20
    rng = np.random.default_rng(2)
    q, k, v = bits(rng, (PERIOD, d)), bits(rng, (n + 1, Hkv, d)), bits(rng, (n + 1, Hkv, d))
    qd = heads(q, G)[None].expand(Hkv, G, d).reshape(1, 1, Hkv * G, d)
    kc, vcache = (torch.empty((1, start + 1, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kc[0, :n + 1], vcache[0, :n + 1] = dev(k), dev(v)
    cache, at = vc.Cache(kc, vcache), torch.tensor([n], dtype=torch.int32, device="cuda")
    out, lse = vc.vitcop_window_attn(qd, cache, start, start_samples=at)
    assert_heads(out.view(Hkv, G, d), lse.view(Hkv, G), q, k, v, n + 1)
    out.fill_(7.5)
    k2, v2 = (dev(x[n:]).view(1, 1, Hkv, d) for x in (k, v))
    vc.vitcop_tree_attn(qd, k2, v2, torch.ones((1, 1), dtype=torch.int64, device="cuda"), cache, start, start_samples=at,
                        out=(out, lse))
    assert_heads(out.view(Hkv, G, d), lse.view(Hkv, G), q, k, v, n + 1)


# Rows of 128 KiB, 512 KV heads of one query head each: 32400 of them end 14 MB below 2^32 bytes with the kernel's margin of 256 rows.
HKV, D, ROWS, NEAR = 512, 128, 40000, 32400
HEADS = [0, 1, 255, 511]


@pytest.fixture(scope="module")
def large(vc):  # noqa: F811
    torch.manual_seed(3)
    k, v = (torch.randn((1, ROWS, HKV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.randn((1, 70, HKV, D), dtype=torch.bfloat16, device="cuda")
    some = [host_f64(t[0][:, HEADS].contiguous()) for t in (q, k, v)]
    return vc.Cache(k, v), q, some


def assert_rows(out, lse, q, k, v, sees, where):
    """out [T,Hq,d], lse [Hq,T] of all heads; q, k, v of those looked at."""
    n, keys = sees.shape
    want = S.attend(q[:n], k[:keys], v[:keys], sees)
    ob, lb = bounds(want, D, keys)
    assert (np.abs(host_f64(out)[:n, HEADS] - want["out"]) <= ob).all(), where
    assert (np.abs(host_f64(lse)[HEADS, :n] - want["lse"]) <= lb.T).all(), where


# T, start, window, sinks, tokens: rows past 2^31 bytes in the kernel of many query rows (NEAR and fewer rows), rows past 2^32 in the
# other, three blocks of 32 query rows of it, the last one of six, or the later ones empty
@pytest.mark.parametrize("T,start,window,sinks,tokens", [
    (70, NEAR - 70, 0, 0, None), (70, NEAR - 70, 20000, 17000, None), (70, ROWS - 70, 32300, 40, None),
    (70, ROWS - 70, 0, 0, None), (70, ROWS - 70, 33000, 3, None), (70, ROWS - 70, 0, 0, 32), (70, ROWS - 70, 33000, 3, 41)])
def test_rows_past_31_and_32_bits(vc, large, T, start, window, sinks, tokens):  # noqa: F811
    cache, q, (qh, kh, vh) = large
    n = T if tokens is None else tokens
    counts = None if tokens is None else torch.tensor([tokens], dtype=torch.int32, device="cuda")
    out = torch.full((1, T, HKV, D), 7.5, dtype=torch.bfloat16, device="cuda"), torch.full((1, HKV, T), 7.5, device="cuda")
    vc.vitcop_window_attn(q[:, :T], cache, start, window, sinks, n_samples=counts, out=out)
    assert_rows(out[0][0], out[1][0], qh, kh, vh, S.window_sees(start, n, start + n, window, sinks), "window")
    assert bool((out[0][:, n:] == 7.5).all()) and bool((out[1][:, :, n:] == 7.5).all())


@pytest.mark.parametrize("T,start,tokens", [(64, NEAR - 64, None), (64, ROWS - 64, None), (45, ROWS - 45, 20), (45, ROWS - 64, None)])
def test_trees_past_31_and_32_bits(vc, large, T, start, tokens):  # noqa: F811
    """The drafts are rows of the cache behind the first `start`."""
    cache, q, (qh, kh, vh) = large
    n = T if tokens is None else tokens
    counts = None if tokens is None else torch.tensor([tokens], dtype=torch.int32, device="cuda")
    masks = trees(np.random.default_rng(T), 1, T)[0]
    signed = torch.tensor([m - 2 ** 64 if m >= 2 ** 63 else m for m in masks], device="cuda")
    out = torch.full((1, T, HKV, D), 7.5, dtype=torch.bfloat16, device="cuda"), torch.full((1, HKV, T), 7.5, device="cuda")
    vc.vitcop_tree_attn(q[:, :T], cache.k[:, start:start + T], cache.v[:, start:start + T], signed, cache, start, n_samples=counts,
                        out=out)
    assert_rows(out[0][0], out[1][0], qh, kh, vh, S.tree_sees(start, n, masks), "tree")
    assert bool((out[0][:, n:] == 7.5).all()) and bool((out[1][:, :, n:] == 7.5).all())


@pytest.mark.parametrize("T,G,n,row", [(64, 1, 70, 6144), (33, 2, 0, 6144), (64, 1, 70, (1 << 24) - 8), (20, 1, 70, (1 << 24) - 8),
                                       (5, 1, 0, (1 << 24) - 8)])
@pytest.mark.parametrize("d", [64, 128])
def test_drafts_of_wide_rows_that_no_token_sees(vc, T, G, n, row, d):  # noqa: F811
    """Keys and values of drafts in rows of `row` elements, up to the longest that there may be; every third draft is seen by none
    and holds NaN and infinities, and so does what lies beside them."""
    rng = np.random.default_rng(T)
    f64 = O.bf16_to_f64
    q, k, v = bits(rng, (T, G, d)), bits(rng, (n + T, 1, d)), bits(rng, (n + T, 1, d))
    hidden = sum(1 << j for j in range(1, T, 3))
    masks = [((2 << t) - 1) & ~hidden for t in range(T)]
    k2, v2 = k[n:].copy(), v[n:].copy()
    k2[1::3], v2[1::3] = 0xFF80, 0x7FC0
    views = []
    for x in (k2, v2):
        wide = torch.empty((T - 1) * row + 2 * d, dtype=torch.bfloat16, device="cuda")
        wide[:2 * d], wide[-2 * d:] = float("nan"), float("nan")
        view = wide[d:].as_strided((1, T, 1, d), (T * row, row, d, 1))
        view.copy_(dev(x)[None])
        views.append(view)
    cache = vc.Cache(dev(k[:n])[None], dev(v[:n])[None])
    signed = torch.tensor([m - 2 ** 64 if m >= 2 ** 63 else m for m in masks], device="cuda")
    out, lse = vc.vitcop_tree_attn(dev(q)[None], *views, signed, cache, n)
    want = S.attend(f64(q), f64(k), f64(v), S.tree_sees(n, T, masks))
    ob, lb = bounds(want, d, n + T)
    assert (np.abs(host_f64(out)[0] - want["out"]) <= ob).all() and (np.abs(host_f64(lse)[0] - want["lse"]) <= lb.T).all()
