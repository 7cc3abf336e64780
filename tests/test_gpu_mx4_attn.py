"""GPU parity: what attention over a cache in 4 bits holds in 32 bits, and its plans of slices and wavefronts."""
import numpy as np
import pytest
import torch

import vitcop_inputs as I
from oracle import vitcop_oracle as O
from gpu_util import dev, host_f64

pytestmark = pytest.mark.gpu


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
# Tolerance: half a step of the output, and 8.  (A probability rounded to 16 bits is off by up to 64 of itself.)
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
