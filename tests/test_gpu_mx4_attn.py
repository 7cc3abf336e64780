"""GPU parity: what attention over a cache in 4 bits holds in 32 bits, and its plans of slices and wavefronts."""
import numpy as np
import pytest
import torch

import vitcop_inputs as I
from oracle import mx4_oracle as X
from oracle import vitcop_oracle as O
from gpu_util import dev, host_f64

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def vc():
    from paper_2601_17818_amd import binding
    return binding


def f32_bits(x):
    return I.f32_to_bf16_bits(np.asarray(x, dtype=np.float32))


def in_three(x):
    """x as the sum of three bf16 (their bits), and that sum."""
    bits, left = [], np.asarray(x, dtype=np.float64)
    for _ in range(3):
        bits.append(O.f64_to_bf16_bits(left))
        left = left - O.bf16_to_f64(bits[-1])
    return bits, sum(O.bf16_to_f64(b) for b in bits)


# Two keys whose values cancel but for some 2^-11 to 2^-15: V is 1 and -top, the scores 0 and s = ln(1/top) + ln(1 + delta), so
# the output is (1 - top p) / (1 + p), p = e^s, about -delta / (1 + 1/top), and an error of p shows in it undiminished.  All
# products and sums before the exponential are exact (q is s in three bf16, K ones).  In units of 2^-24: s in powers of two
# (1.6 at most) is off by two roundings of itself, 2 * 1.6 * ln 2 = 2.2 of p; the exponential by two (one step); with top p about
# 1 and three for the products' sum that is 7.2 of the numerator, and 5.4 of the quotient, 1 + p being 4/3 and more.
# Tolerance: half a step of the output, and 8.  (A probability rounded to 16 bits is off by up to 256 of itself.)
@pytest.mark.parametrize("B,N,Hq,Hkv,d,at", [
    (4, 2, 16, 1, 64, (0, 1)), (4, 45, 16, 2, 128, (33, 44)), (3, 900, 32, 2, 128, (601, 620)), (40, 1700, 32, 8, 64, (7, 31)),
    (31, 8500, 16, 1, 64, (5003, 5022)), (5, 24001, 16, 4, 128, (0, 24000))])
@pytest.mark.parametrize("top", [1.5, 3.0])
def test_a_probability_keeps_its_bits(vc, B, N, Hq, Hkv, d, at, top):
    rng = np.random.default_rng(N + d)
    delta = np.exp2(rng.uniform(-15, -11, (B, Hq))) * rng.choice([-1.0, 1.0], (B, Hq))
    parts, s = in_three(np.log(1 / top) + np.log1p(delta))
    q = np.zeros((B, Hq, d), np.uint16)
    for c in range(3):
        q[..., c] = parts[c]
    q[..., 3] = f32_bits(-100.0)
    k, v = np.zeros((1, N, Hkv, d), np.uint16), np.full((1, N, Hkv, d), f32_bits(1.0), np.uint16)
    k[..., 3] = f32_bits(2.0)                                             # the others: a score of -200, a probability of 0
    k[:, at[0], :, 3] = k[:, at[1], :, 3] = 0
    k[:, at[1], :, :3] = f32_bits(1.0)
    v[:, at[1]] = f32_bits(-top)
    cache = vc.CacheMx4.empty(B, N, Hkv, d)
    vc.vitcop_cache_mx4_write(cache, dev(k).expand(B, N, Hkv, d), dev(v).expand(B, N, Hkv, d))
    p = np.exp(s)
    want = ((1 - top * p) / (1 + p))[..., None]
    got, lse = vc.vitcop_decode_attn_mx4(dev(q), cache, N, scale=1.0)
    off = np.abs(host_f64(got) - want)
    assert (off <= 2.0 ** -8 * np.abs(want) + 2.0 ** -21).all(), (off.max(), (off > 2.0 ** -8 * np.abs(want) + 2.0 ** -21).mean())
    assert np.abs(lse.cpu().numpy() - np.log(1 + p)).max() <= 2.0 ** -21
    # and against the framework's attention over the values read back
    kk, vv = vc.vitcop_cache_mx4_read(cache, N)
    other, other_lse = vc.vitcop_decode_attn(dev(q), kk, vv, scale=1.0)
    assert (np.abs(host_f64(other) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -21).all()
    assert torch.equal(torch.isnan(got), torch.isnan(other)) and (lse - other_lse).abs().max() <= 2.0 ** -20


# Every number of wavefronts, sliced and not, and of products with V (up to 5, 8 and 16 query heads a pass; 17: two passes).
# Samples attend over all rows, none, a third (so that slices, and wavefronts of a slice, have no key) and 33 of them.
@pytest.mark.parametrize("B,N,Hq,Hkv,d", [
    (4, 50, 12, 1, 64), (4, 60, 8, 1, 128), (4, 61, 9, 1, 128), (4, 100, 6, 1, 64), (4, 110, 32, 2, 64), (4, 300, 14, 2, 64),
    (4, 300, 6, 1, 128), (4, 1100, 8, 1, 64), (4, 1100, 22, 2, 64), (4, 1030, 7, 1, 128), (31, 8500, 3, 1, 64), (31, 8500, 7, 1, 64),
    (31, 8500, 17, 1, 64), (7, 9500, 4, 4, 128), (7, 9500, 28, 4, 128), (31, 8500, 17, 1, 128), (15, 9300, 30, 2, 64)])
def test_slices_and_wavefronts(vc, B, N, Hq, Hkv, d):
    rows = [I.normal_bf16(N + Hq, i, (4, N, Hkv, d)) for i in range(2)]
    q4 = I.normal_bf16(N + Hq, 2, (4, Hq, d))
    of = np.arange(B) % 4
    q = dev(np.ascontiguousarray(q4[of]))
    cache = vc.CacheMx4.empty(B, N, Hkv, d)
    vc.vitcop_cache_mx4_write(cache, dev(rows[0])[of], dev(rows[1])[of])
    kv = [X.round_trip(x).transpose(0, 2, 1, 3) for x in rows]
    for lens in (None, [N, 0, N // 3, 33]):
        if lens is not None:
            for b in range(B):
                for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
                    t[b, :, lens[b % 4]:] = 255                          # not a number, and not looked at
        n = None if lens is None else torch.tensor([lens[b % 4] for b in range(B)], dtype=torch.int32, device="cuda")
        o, lse = vc.vitcop_decode_attn_mx4(q, cache, N, n)
        ref, ref_lse, spread, size = (x[of] for x in X.decode_attention(q4, kv[0], kv[1], lens))
        # a score is off by (d + 4) 2^-24 of its products' magnitudes, a probability by that and the exponential's last bits
        p_off = (d + 4) * EPS * size + 2.0 ** -20 + N * EPS
        got, got_lse, live = host_f64(o), lse.cpu().numpy().astype(np.float64), ~np.isneginf(ref_lse)
        assert np.array_equal(np.isneginf(got_lse), ~live) and not got[~live].any()
        assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2 * p_off[..., None] * spread)[live].all()
        assert (np.abs(got_lse[live] - ref_lse[live]) <= p_off[live] + 2.0 ** -22 * (1 + np.abs(ref_lse[live]))).all()
        first, first_lse = o[:4].clone(), lse[:4].clone()
        for b in range(4, B):                                             # equal samples, equal results
            assert torch.equal(o[b], first[b % 4]) and torch.equal(lse[b], first_lse[b % 4])
