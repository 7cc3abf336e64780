"""How many bits of a probability reach the products with V: 24 of up to 16 query rows of a KV head, 16 of up to 32.

Two keys whose values cancel but for some 2^-11 to 2^-15: V is 1 and -top, the scores 0 and s = ln(1/top) + ln(1 + delta), so the
output is (1 - top p) / (1 + p), p = e^s, about -delta / (1 + 1/top), and an error of p shows in it undiminished.  Products and
sums before the exponential are exact (q is s in three bf16, K ones); all other keys have a score of -200 and no probability that
fp32 holds.  In units of 2^-24: s in powers of two (1.6 at most) is off by two roundings of itself, 2 * 1.6 * ln 2 = 2.2 of p; the
exponential by two (one step); with top p about 1 and three for the products' sum that is 7.2 of the numerator, and 5.4 of the
quotient, 1 + p being 4/3 and more: 8 units are 2^-21.  Half a step of bf16 is 2^-8 of the value: a probability in two is off by
2^-16 of itself at most, and so is top p / (1 + p) < 1 of the output.  Tolerance: half a step of the output, 2^-21, and with
17 to 32 rows 2^-16."""
import numpy as np
import pytest
import torch

import vitcop_inputs as I
from oracle import vitcop_oracle as O


def f32_bits(x):
    return int(I.f32_to_bf16_bits(np.array([x], np.float32))[0])


def in_bf16(x, parts):
    """The bits of so many bf16, each the nearest to what those before leave of x, and their sum."""
    left, bits = np.array(x, np.float64), []
    for _ in range(parts):
        bits.append(O.f64_to_bf16_bits(left))
        left = left - O.bf16_to_f64(bits[-1])
    return bits, sum(O.bf16_to_f64(b) for b in bits)


def tolerance(want, rows):
    return 2.0 ** -8 * np.abs(want) + 2.0 ** -21 + (2.0 ** -16 if rows > 16 else 0.0)


def scores(rng, shape, top):
    """(three bf16 of the score of the second key, p, the output)"""
    delta = np.exp2(rng.uniform(-15, -11, shape)) * rng.choice([-1.0, 1.0], shape)
    parts, s = in_bf16(np.log(1 / top) + np.log1p(delta), 3)
    p = np.exp(s)
    return parts, p, (1 - top * p) / (1 + p)


# B, T, G, Hkv
ROWS = [(6, 1, 16, 1), (4, 4, 4, 2), (6, 16, 1, 1), (12, 1, 7, 1), (5, 1, 17, 1), (3, 4, 7, 2), (3, 32, 1, 1), (3, 2, 16, 1)]


@pytest.mark.parametrize("B,T,G,Hkv", ROWS)
@pytest.mark.parametrize("top", [1.5, 3.0])
def test_the_tolerance_tells_a_part_less(B, T, G, Hkv, top):
    """The kernels' arithmetic but for the order of sums: within the tolerance with their number of parts, past it with one less."""
    _, p, want = scores(np.random.default_rng(B * T), (B, T, G * Hkv), top)
    p = p.astype(np.float32).astype(np.float64)
    parts = 3 if T * G <= 16 else 2
    for n, holds in ((parts, True), (parts - 1, False)):
        sent = in_bf16(p, n)[1]
        got = O.bf16_to_f64(O.f64_to_bf16_bits((1 - top * sent) / (1 + p)))
        assert (np.abs(got - want) <= tolerance(want, T * G)).all() == holds


def window(vc, q, k, v, T):
    return vc.vitcop_window_attn(q, vc.Cache(k, v), k.shape[1] - T, scale=1.0)


def tree(vc, q, k, v, T):
    """The last T rows of the keys are drafts, all of them seen by each."""
    n = k.shape[1] - T
    masks = torch.tensor([2 ** T - 1] * T, device="cuda")
    return vc.vitcop_tree_attn(q, k[:, n:], v[:, n:], masks, vc.Cache(k[:, :n].contiguous(), v[:, :n].contiguous()), n, scale=1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,G,Hkv", ROWS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,at", [                       # (the two in the same 32 keys: in one wavefront's sums)
    (45, (33, 44)), (900, (611, 620)), (8500, (5003, 5022))])
@pytest.mark.parametrize("call", [window, tree])
def test_a_probability_keeps_its_bits(B, T, G, Hkv, d, n, at, call):
    from gpu_util import dev, host_f64
    from paper_2601_17818_amd import binding as vc
    for top in (1.5, 3.0):
        parts, p, want = scores(np.random.default_rng(B * T), (B, T, G * Hkv), top)
        q = np.zeros((B, T, G * Hkv, d), np.uint16)
        for c in range(3):
            q[..., c] = parts[c]
        q[..., 3] = f32_bits(-100.0)
        k = np.zeros((B, n + T, Hkv, d), np.uint16)
        v = np.full((B, n + T, Hkv, d), f32_bits(1.0), np.uint16)
        k[..., 3] = f32_bits(2.0)
        k[:, at[0], :, 3] = k[:, at[1], :, 3] = 0
        k[:, at[1], :, :3] = f32_bits(1.0)
        v[:, at[1]] = f32_bits(-top)
        out, lse = call(vc, dev(q), dev(k), dev(v), T)
        off = np.abs(host_f64(out) - want[..., None])
        assert (off <= tolerance(want, T * G)[..., None]).all(), (top, off.max())
        assert np.abs(lse.cpu().numpy().transpose(0, 2, 1) - np.log(1 + p)).max() <= 2.0 ** -21


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,G", [(4, 4), (16, 1), (8, 3), (32, 1)])
def test_a_probability_of_a_draft_keeps_its_bits(T, G, d):
    """The two keys are drafts 0 and T - 1 that every token sees."""
    from gpu_util import dev, host_f64
    from paper_2601_17818_amd import binding as vc
    B, n = 8, 70
    for top in (1.5, 3.0):
        parts, p, want = scores(np.random.default_rng(T), (B, T, G), top)
        q = np.zeros((B, T, G, d), np.uint16)
        for c in range(3):
            q[..., c] = parts[c]
        q[..., 3] = f32_bits(-100.0)
        k = np.zeros((B, n + T, 1, d), np.uint16)
        v = np.full((B, n + T, 1, d), f32_bits(1.0), np.uint16)
        k[..., 3] = f32_bits(2.0)
        k[:, n, :, 3] = k[:, -1, :, 3] = 0
        k[:, -1, :, :3] = f32_bits(1.0)
        v[:, -1] = f32_bits(-top)
        out, _ = tree(vc, dev(q), dev(k), dev(v), T)
        off = np.abs(host_f64(out) - want[..., None])
        assert (off <= tolerance(want, T * G)[..., None]).all(), (top, off.max())
